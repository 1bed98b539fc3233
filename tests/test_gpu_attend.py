"""GPU parity of attention over pages against the oracle in float64: head layouts, page sizes, lengths from nothing to
several tiles, several query tokens, E4M3 keys, shared prefixes; everything that is not held is NaN."""
import numpy as np
import pytest
import torch

from paper_2601_07667_b200 import binding as B

from pages_check import Both, check_attention, ints, queries

pytestmark = pytest.mark.gpu

HEADS = [(8, 2), (32, 8), (28, 4), (5, 5), (32, 1), (40, 1), (64, 8), (128, 1)]


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("page,fp8", [(16, False), (32, True), (64, False), (128, True), (128, False), (16, True)])
def test_single_tokens(heads, page, fp8):
    lens = [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 200, 333]
    both = Both(kv_heads=heads[1], page=page, n_pages=140, max_seqs=len(lens), max_pages=-(-333 // page), fp8=fp8, seed=heads[0])
    both.fill(lens)
    slots = [int(x) for x in np.random.default_rng(1).permutation(len(lens))]
    check_attention(both, 0, slots, list(range(len(lens) + 1)), heads[0], share=False)
    check_attention(both, 0, slots, list(range(len(lens) + 1)), heads[0], share=2, want_lse=False)


@pytest.mark.parametrize("heads", [(8, 2), (28, 4), (32, 1), (6, 6)])
@pytest.mark.parametrize("page,fp8", [(16, True), (64, False)])
def test_several_tokens_of_a_sequence(heads, page, fp8):
    """Causal among themselves; as many as the sequence has; none; a free slot and padding; rows behind the last."""
    lens = [5, 9, 64, 70, 130, 0, 300, 40]
    counts = [5, 2, 33, 1, 9, 2, 17, 0]
    both = Both(kv_heads=heads[1], page=page, n_pages=60, max_seqs=9, max_pages=-(-300 // page), fp8=fp8, seed=7)
    both.fill(lens + [0])
    slots = [0, 1, 2, 3, 4, 5, 6, 7, -1, 99]
    cu = np.concatenate([[0], np.cumsum(counts + [3, 2])]).tolist()
    check_attention(both, 0, slots, cu, heads[0], share=2, n_tokens=cu[-1] + 4)


def test_keys_that_are_not_seen_may_hold_anything():
    """A later token of the same sequence with NaN and infinities in K and V changes nothing for the tokens before it."""
    both = Both(kv_heads=2, page=16, n_pages=30, max_seqs=2, max_pages=8)
    both.fill([70, 35])
    cu, slots = [0, 6, 9], [0, 1]
    q = queries(both.rng, 9, 8)
    _, clean, lse = check_attention(both, 0, slots, cu, 8, share=False, q=q)
    for s, n in ((0, 70), (1, 35)):
        p, r = int(both.oracle.table[s, (n - 1) // 16]), (n - 1) % 16
        both.cache.k[0, p, :, r] = float("nan")
        both.cache.v[0, p, :, r, ::2] = float("inf")
        both.cache.v[0, p, :, r, 1::2] = float("nan")
    batch = both.cache.batch(ints(slots), ints(cu), n_tokens=9, n_q_heads=8)
    both.cache.plan(batch)
    out = both.cache.attend(0, batch, q[0])
    for last in (5, 8):
        assert torch.isnan(out[last]).any()
    keep = [0, 1, 2, 3, 4, 6, 7]
    assert torch.equal(out[keep], clean[keep])


def test_logits_of_any_size():
    """Keys far along the query: one weight is 1; equal keys: all weights are; logits of -inf leave their keys out."""
    both = Both(kv_heads=1, page=16, n_pages=20, max_seqs=1, max_pages=16)
    both.fill([200])
    o = both.oracle
    big = lambda x: torch.full((128,), x).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)   # noqa: E731
    for pos, val in ((3, 40.0), (70, -40.0), (150, 39.75)):
        both.oracle.put(0, 0, pos, 0, big(val), o.v[0, o.table[0, pos // 16], 0, pos % 16].copy())
    both.cache.k.copy_(both.dev(o.k))
    q = torch.full((1, 4, 128), 3.0)
    q[0, 1], q[0, 2], q[0, 3] = 0.0, -3.0, 0.001
    q = q.to(torch.bfloat16)
    check_attention(both, 0, [0], [0, 1], 4, share=False, q=(q.cuda(), q.double().numpy()))
    # a key of -infinity where the query is positive: its weight is zero for that row
    both.cache.k[0, int(o.table[0, 1]), 0, 5] = float("-inf")
    batch = both.cache.batch(ints([0]), ints([0, 1]), n_tokens=1, n_q_heads=4)
    both.cache.plan(batch)
    out = both.cache.attend(0, batch, q.cuda())
    assert torch.isfinite(out[0, 0]).all() and torch.isnan(out[0, 1]).all()         # 0 x inf is NaN, as it is in a product


def test_strided_queries_and_layers():
    both = Both(kv_heads=4, page=32, n_pages=40, max_seqs=3, max_pages=10, layers=3, seed=9)
    both.fill([100, 7, 290])
    wide = torch.randn((5, 3, 20, 128), device="cuda").to(torch.bfloat16)           # q between other tensors of a fused projection
    for layer in range(3):
        q = wide[:, layer, 4:16]
        check_attention(both, layer, [2, 0, 1], [0, 2, 3, 5], 12, share=2, q=(q, q.double().cpu().numpy()))


def test_the_same_bits_every_time():
    both = Both(kv_heads=2, page=16, n_pages=300, max_seqs=2, max_pages=140)
    both.fill([2100, 900])
    q = queries(both.rng, 2, 8)
    _, out, lse = check_attention(both, 0, [0, 1], [0, 1, 2], 8, share=False, q=q)
    for _ in range(5):
        _, again, lse2 = check_attention(both, 0, [0, 1], [0, 1, 2], 8, share=False, q=q)
        assert torch.equal(out, again) and torch.equal(lse, lse2)


def test_a_workspace_without_a_plan_is_refused():
    both = Both(kv_heads=2, page=16, n_pages=20, max_seqs=2, max_pages=8)
    both.fill([20, 30])
    batch = both.cache.batch(ints([0, 1]), ints([0, 1, 2]), n_tokens=2, n_q_heads=4)
    batch.workspace.zero_()
    out = torch.full((2, 4, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    both.cache.attend(0, batch, torch.ones_like(out), out)
    assert B.asl_pages_status(both.cache.ctx, both.cache.pages) == (B.ASL_ERR_WORKSPACE, -1)
    assert (out == 7.0).all()


def forked(heads, page, prompts, tails, *, fp8=False, layers=1, seed=0):
    """(cache, slots): for each prompt of that many tokens a parent and its forks, each with a tail of its own."""
    n = sum(len(t) for t in tails)
    need = sum(-(-p // page) + sum(2 + -(-t // page) for t in ts) for p, ts in zip(prompts, tails))
    longest = max(p + max(ts) for p, ts in zip(prompts, tails))
    P = len(prompts)
    both = Both(kv_heads=heads[1], page=page, n_pages=need + 3, max_seqs=P + n, max_pages=-(-longest // page), layers=layers, fp8=fp8, seed=seed)
    both.fill(list(prompts) + [0] * n)
    parent, want = [-1] * P, [-1] * P
    for i, ts in enumerate(tails):
        parent += [i] * len(ts)
        want += [prompts[i] + t for t in ts]
    both.fork(parent)
    both.fill(want)
    return both, list(range(P, P + n))


@pytest.mark.parametrize("heads", [(8, 2), (28, 4), (32, 1), (3, 3), (128, 1), (64, 8)])
@pytest.mark.parametrize("page,fp8", [(16, False), (32, True), (64, False), (128, True), (128, False)])
def test_a_shared_prefix(heads, page, fp8):
    """Nine sequences on one prompt whose last page is not full and whose last tile is not either."""
    prompt = 128 * 5 + max(page, 48) + 5
    both, slots = forked(heads, page, [prompt], [[1, 2, 15, 60, 64, 65, 130, 7, 1]], fp8=fp8, seed=page)
    check_attention(both, 0, slots, list(range(10)), heads[0], share=2)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("heads,n", [((8, 2), 31), ((8, 2), 32), ((8, 2), 33), ((8, 2), 64), ((8, 2), 65), ((14, 2), 37), ((16, 1), 40), ((2, 2), 300)])
def test_rows_around_a_chunk(heads, n, fp8):
    """Rows of a prefix below, at and above 128 and 256."""
    both, slots = forked(heads, 32, [1056], [[1 + (i * 7) % 40 for i in range(n)]], fp8=fp8, seed=n)
    check_attention(both, 0, slots, list(range(n + 1)), heads[0], share=2)


@pytest.mark.parametrize("fp8", [False, True])
def test_several_prompts_and_several_tokens(fp8):
    """Prompts of different lengths, some too short to share; sequences of other prompts between them; padding inside a group;
    drafts of several tokens; one prompt's own slot beside its forks."""
    prompts, tails = [700, 2000, 40, 1300], [[5, 9, 30], [3, 17, 100, 64], [6, 8], [5, 5, 5, 5, 5]]
    both, s = forked((28, 4), 16, prompts, tails, fp8=fp8, layers=2, seed=5)
    slots = s[:3] + [1] + s[3:5] + [-1] + s[5:7] + s[7:9] + [2] + s[9:] + [3]
    counts = [5, 3, 1, 2, 3, 3, 4, 5, 5, 2, 2, 1, 5, 5, 1, 5, 5, 7]
    cu = np.concatenate([[0], np.cumsum(counts)]).tolist()
    for layer in range(2):
        check_attention(both, layer, slots, cu, 28, share=2, n_tokens=cu[-1] + 3)
    order = [slots[i] for i in (9, 0, 17, 4, 1, 8, 12)]
    check_attention(both, 0, order, list(range(len(order) + 1)), 28, share=2)


@pytest.mark.parametrize("groups,n,prompt", [(1, 2, 40000), (3, 40, 5000), (16, 3, 1100), (40, 2, 600)])
def test_long_prompts_split_over_blocks(groups, n, prompt):
    """Stretches that begin and end inside chunks of one and two rows of accumulators."""
    heads = (8, 2)
    both, slots = forked(heads, 64, [prompt + 33 * i for i in range(groups)], [[1 + (i * 5 + g) % 20 for i in range(n)] for g in range(groups)], seed=groups)
    check_attention(both, 0, slots, list(range(len(slots) + 1)), heads[0], share=2)


def test_a_shared_prefix_of_any_size_of_logits():
    """Maxima that grow from tile to tile, fall, jump by more than the reference may lag, and a NaN that stays one."""
    both, slots = forked((4, 1), 16, [1600], [[3, 4, 5, 6]], seed=1)
    o = both.oracle
    big = lambda x: torch.full((128,), x).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)   # noqa: E731
    for pos, val in ((1, 1.0), (140, 2.0), (141, -30.0), (300, 2.5), (500, 11.0), (900, 40.0), (1000, 39.0), (1400, -50.0)):
        o.put(0, 0, pos, 0, big(val), o.v[0, o.table[0, pos // 16], 0, pos % 16].copy())
    both.cache.k.copy_(both.dev(o.k))
    q = torch.randn((4, 4, 128)) * 0.3 + torch.tensor([1.0, -1.0, 0.0, 0.05])[None, :, None]
    q = q.to(torch.bfloat16)
    check_attention(both, 0, slots, [0, 1, 2, 3, 4], 4, share=2, q=(q.cuda(), q.double().numpy()))
    for pool, value in ((both.cache.k, float("nan")), (both.cache.v, float("nan")), (both.cache.k, float("inf"))):
        keep = pool[0, int(o.table[0, 20]), 0, 3].clone()
        pool[0, int(o.table[0, 20]), 0, 3] = value
        batch = both.cache.batch(ints(slots), ints([0, 1, 2, 3, 4]), n_tokens=4, n_q_heads=4)
        both.cache.plan(batch, share=2)
        # (a key of infinity against queries that are all negative is a logit of -inf: a weight of zero)
        zero_weight = (q.double() * float("inf")).sum(-1).cuda() == float("-inf") if value == float("inf") else torch.zeros((4, 4), dtype=bool, device="cuda")
        assert torch.equal(torch.isnan(both.cache.attend(0, batch, q.cuda())), ~zero_weight[:, :, None].expand(4, 4, 128))
        pool[0, int(o.table[0, 20]), 0, 3] = keep


def test_shared_and_alone_agree_and_repeat():
    both, slots = forked((32, 8), 64, [3000], [[1 + i for i in range(20)]], seed=3)
    q = queries(both.rng, 20, 32)
    _, alone, _ = check_attention(both, 0, slots, list(range(21)), 32, share=False, q=q)
    _, out, lse = check_attention(both, 0, slots, list(range(21)), 32, share=2, q=q)
    for _ in range(3):
        _, again, lse2 = check_attention(both, 0, slots, list(range(21)), 32, share=2, q=q)
        assert torch.equal(out, again) and torch.equal(lse, lse2)


def test_a_plan_that_shares_wants_its_prefixes_read():
    """A plan with shared prefixes and an attention told that nothing is: refused, nothing written."""
    both, slots = forked((8, 2), 16, [1600], [[3, 4, 5, 6]], seed=1)
    batch = both.cache.batch(ints(slots), ints([0, 1, 2, 3, 4]), n_tokens=4, n_q_heads=8)
    out = torch.full((4, 8, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    both.cache.plan(batch, share=2)
    batch.share = 0
    both.cache.attend(0, batch, torch.ones_like(out), out)
    assert B.asl_pages_status(both.cache.ctx, both.cache.pages) == (B.ASL_ERR_WORKSPACE, -1)
    assert (out == 7.0).all()
    for share in (-1, 3):
        with pytest.raises(B.AslError):
            both.cache.plan(batch, share=share)


def test_sharing_where_it_saves_enough():
    """share = 1: nothing is told apart by the results, whether the prefix is read once (32 MB or more saved) or by each."""
    for prompt, n in ((600, 5), (2100, 40)):
        both, slots = forked((32, 8), 64, [prompt], [[1 + i % 7 for i in range(n)]], seed=n)
        check_attention(both, 0, slots, list(range(n + 1)), 32, share=1)
