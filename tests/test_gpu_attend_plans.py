"""Plans that do not belong to the call that meets them: of another cache, of an earlier owner of the workspace's memory; and
tables that name pages which the pool does not have."""
import pytest
import torch

from paper_2601_07667_b200 import binding as B

from pages_check import Both, check_attention, ints, queries

pytestmark = pytest.mark.gpu


def left_alone(cache, batch, heads):
    out = torch.full((batch.n_tokens, heads, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((batch.n_tokens, heads), 7.0, device="cuda")
    cache.attend(0, batch, torch.ones_like(out), out, lse)
    assert B.asl_pages_status(cache.ctx, cache.pages) == (B.ASL_ERR_WORKSPACE, -1)
    assert (out == 7.0).all() and (lse == 7.0).all()


def forked(**sizes):
    """A prompt of 90 tokens in the last slots but five and five forks of it behind it."""
    both = Both(kv_heads=2, **sizes)
    n = sizes["max_seqs"]
    both.fill([0] * (n - 6) + [90] + [0] * 5)
    both.fork([-1] * (n - 6) + [-1] + [n - 6] * 5)
    both.fill([-1] * (n - 5) + [91, 95, 99, 100, 92])
    return both


@pytest.mark.parametrize("share", [0, 2])
@pytest.mark.parametrize("other", [dict(page=64), dict(max_seqs=7), dict(max_pages=8), dict()])
def test_a_plan_of_another_cache_is_refused(other, share):
    """The plan names slots that the other cache's table may not have, and prefixes of whole pages of another size: refused by
    what differs, or, where all sizes agree, by the table that it was made from."""
    sizes = dict(page=16, n_pages=80, max_seqs=40, max_pages=12)
    a, b = forked(**sizes), forked(**{**sizes, **other})
    batch = a.cache.batch(ints(range(34, 40)), ints(range(7)), n_tokens=6, n_q_heads=8)
    a.cache.plan(batch, share=share)
    left_alone(b.cache, batch, 8)
    n = b.cache.len.numel()
    check_attention(b, 0, list(range(n - 6, n)), list(range(7)), 8, share=share)
    check_attention(a, 0, list(range(34, 40)), list(range(7)), 8, share=share)


def test_a_batch_may_serve_several_caches():
    """Rows appended and attention planned anew for each of two caches with the same slots."""
    sizes = dict(page=16, n_pages=80, max_seqs=40, max_pages=12)
    a, b = forked(**sizes), forked(**sizes, seed=1)
    batch = a.cache.batch(ints(range(34, 40)), ints(range(7)), n_tokens=6, n_q_heads=8)
    q = torch.randn((6, 8, 128), device="cuda").to(torch.bfloat16)
    for both in (a, b):
        both.cache.plan(batch, share=2)
        out = both.cache.attend(0, batch, q)
        both.cache.check()
        o, _, tol, _ = both.expect(0, list(range(34, 40)), list(range(7)), q.double().cpu().numpy(), 8)
        assert (abs(out.double().cpu().numpy() - o) <= tol).all()


def test_a_plan_that_an_earlier_batch_left_is_none():
    """A batch whose workspace lies where another's did, plan and all."""
    both = forked(page=16, n_pages=80, max_seqs=40, max_pages=12)
    slots, cu = ints(range(34, 40)), ints(range(7))
    batch = both.cache.batch(slots, cu, n_tokens=6, n_q_heads=8)
    both.cache.plan(batch)
    at = batch.ws
    del batch
    batch = both.cache.batch(slots, cu, n_tokens=6, n_q_heads=8)
    assert batch.ws == at
    left_alone(both.cache, batch, 8)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("page,prompt", [(16, 90), (16, 1500), (128, 300)])
@pytest.mark.parametrize("wrong", [-1, "n_pages", 1 << 30, -2 ** 31])
def test_page_numbers_that_the_pool_does_not_have(page, prompt, wrong, fp8):
    """A spoiled entry of the table, in a tail or in the pages that a prompt's forks share (the first ones or far behind them): noted
    with a slot that holds it; what does not read it is as it was."""
    n_pages = 6 + -(-prompt // page) + 5 * 3 + 2
    both = Both(kv_heads=2, page=page, n_pages=n_pages, max_seqs=8, max_pages=-(-prompt // page) + 2, fp8=fp8, seed=3)
    both.fill([prompt, 0, 0, 0, 0, 0, 40, 0])
    both.fork([-1, 0, 0, 0, 0, 0, -1, -1])
    both.fill([-1] + [prompt + 1 + i for i in range(5)] + [-1, -1])
    slots, cu = list(range(1, 7)), list(range(7))
    q = queries(both.rng, 6, 8)
    clean = {share: check_attention(both, 0, slots, cu, 8, share=share, q=q)[1] for share in (0, 2)}
    batch = both.cache.batch(ints(slots), ints(cu), n_tokens=6, n_q_heads=8)
    wrong = n_pages if wrong == "n_pages" else wrong
    table, last = both.cache.table.clone(), prompt // page
    for spoiled, column in (([3], last), ([1, 2, 3, 4, 5], 0), ([1, 2, 3, 4, 5], last - 1), ([6], 0)):
        both.cache.table[torch.tensor(spoiled), column] = wrong
        for share in (0, 2):
            both.cache.plan(batch, share=share)
            out = both.cache.attend(0, batch, q[0])
            st, slot = B.asl_pages_status(both.cache.ctx, both.cache.pages)
            assert st == B.ASL_ERR_INVALID and slot in spoiled
            for i, s in enumerate(slots):
                if s not in spoiled:
                    assert torch.equal(out[i], clean[share][i]) or both_close(both, s, out[i], q[1][i])
        both.cache.table.copy_(table)


def both_close(both, slot, out, q):
    """Neighbours that no longer share what they did are read in other parts, and still within the tolerance."""
    o, _, tol, _ = both.expect(0, [slot], [0, 1], q[None], 8)
    return (abs(out[None].double().cpu().numpy() - o) <= tol).all()


@pytest.mark.parametrize("fp8", [False, True])
def test_steps_back_to_back_read_what_was_just_written(fp8):
    """Rows appended, queries changed and attention over a shared prefix and tails, call behind call without a wait: the same bits as
    with a wait behind each.  The word by which one kernel lets the next one read is taken back every time."""
    n, L = 24, 2
    both = Both(kv_heads=4, page=16, n_pages=400, max_seqs=n + 1, max_pages=80, layers=L, fp8=fp8, seed=9)
    both.fill([1030] + [0] * n)
    both.fork([-1] + [0] * n)
    both.fill([-1] + [1031 + 7 * i % 60 for i in range(n)])
    c = both.cache
    batch = c.batch(ints(range(1, n + 1)), ints(range(n + 1)), n_tokens=n, n_q_heads=16)
    steps = [([both.dev(x) for x in both.new_rows(n, 4, 128)], queries(both.rng, n, 16)[0]) for _ in range(12)]
    word = batch.workspace[128:132].view(torch.int32)

    def go(wait):
        got = []
        for (k, v), q in steps:
            for layer in range(L):
                c.append(layer, batch, k, v)
                if wait:
                    torch.cuda.synchronize()
            c.plan(batch, share=2)
            for layer in range(L):
                got.append(c.attend(layer, batch, q))
                if wait:
                    torch.cuda.synchronize()
                    assert word.item() == 0
        return got
    waited = go(True)
    for _ in range(8):
        for a, b in zip(waited, go(False)):
            assert torch.equal(a, b)
    c.check()


def test_scales_may_change_from_call_to_call():
    """Key scales written by the kernel just before: the calls behind it use them."""
    both = Both(kv_heads=2, page=16, n_pages=200, max_seqs=9, max_pages=44, fp8=True, seed=2)
    both.fill([600] + [0] * 8)
    both.fork([-1] + [0] * 8)
    both.fill([-1] + [601 + 9 * i for i in range(8)])
    slots, cu, q = list(range(1, 9)), list(range(9)), queries(both.rng, 8, 8)
    batch = both.cache.batch(ints(slots), ints(cu), n_tokens=8, n_q_heads=8)
    first = both.scale.copy()
    for share in (0, 2):
        both.cache.plan(batch, share=share)
        outs = []
        for times in (1.0, 2.0, 0.5, 1.5):
            both.cache.k_scale.copy_(torch.from_numpy(first).cuda() * times)
            outs.append((times, both.cache.attend(0, batch, q[0])))
        for times, out in outs:
            both.scale = first * times
            o, _, tol, _ = both.expect(0, slots, cu, q[1], 8)
            assert (abs(out.double().cpu().numpy() - o) <= tol).all()
    both.cache.check()
