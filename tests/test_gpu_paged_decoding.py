"""A prompt's way through the paged cache as a user goes it: prefill layers pruned into pages, forks, steps of decoding with
copies on write, pruning once more, freeing; and the calls under CUDA graphs, on other streams and at far offsets."""
import numpy as np
import pytest
import torch

from oracle import asl_oracle as O
from paper_2601_07667_b200 import binding as B
from paper_2601_07667_b200 import inputs as I

from asl_check import make_path, to_dev
from pages_check import Both, bits, check_attention, ints, queries

pytestmark = pytest.mark.gpu


def step(both, slots, n_q_heads, counts, share=2):
    """One decoding step of `counts` tokens for each slot: grow, append on every layer, attend on every layer."""
    want = [-1] * len(both.oracle.len)
    for s, c in zip(slots, counts):
        want[s] = int(both.oracle.len[s]) + c
    both.reserve(want)
    cu = np.concatenate([[0], np.cumsum(counts)])
    batch = both.cache.batch(ints(slots), ints(cu), n_tokens=int(cu[-1]))
    for layer in range(both.layers):
        k, v = both.new_rows(int(cu[-1]), both.kv_heads, 128)
        both.cache.append(layer, batch, both.dev(k), both.dev(v))
        for i, s in enumerate(slots):
            for t in range(counts[i]):
                for h in range(both.kv_heads):
                    both.oracle.put(layer, s, int(both.oracle.len[s]) - counts[i] + t, h, k[cu[i] + t, h], v[cu[i] + t, h])
        check_attention(both, layer, slots, cu.tolist(), n_q_heads, share=share)


def test_prefill_fork_decode_prune_free():
    """Two prompts of three layers; kept rows go into pages as the layers run; samples of both decode side by side, single
    tokens and drafts; then one sample's cache is pruned into another slot, the rest is freed, and the pool is whole again."""
    wl = I.workload("C1", seqlens=(2500, 1700), budgets=(1111, 640), layers=3)
    path, H, Hq = make_path(wl), wl.n_kv_heads, wl.n_q_heads
    both = Both(kv_heads=H, page=32, n_pages=150, max_seqs=12, max_pages=48, layers=3, seed=1)
    both.reserve([-1, 1111, -1, 640] + [-1] * 8)
    path.store_into(both.cache, ints([1, 3]))
    alive = []
    for layer in range(3):
        x = I.layer_inputs(wl, layer, seed=9)
        args = [to_dev(x[n]) for n in ("q_obs", "k", "v")]
        alive.append(args)
        path.run_layer(*args, layer)
        path.join()
        idx = path.idx.cpu().numpy()
        for b, (slot, m, off, tok) in enumerate(((1, 1111, 0, 0), (3, 640, 1111, 2500))):
            for h in range(H):
                for r in range(m):
                    t = tok + idx[h, off + r]
                    both.oracle.put(layer, slot, r, h, x["k"][t, h], x["v"][t, h])
    both.cache.check()
    both.same_rows()
    both.fork([-1, -1, 1, -1, 1, 1, 1, 1, 3, 3, -1, -1])
    slots = [2, 4, 5, 6, 7, 1, 8, 9]
    for counts in ([1] * 8, [1] * 8, [3, 1, 5, 1, 2, 1, 4, 4], [30] * 8):
        step(both, slots, Hq, counts)
        both.same_books()
    both.same_rows()
    # sample 5 goes on with 200 rows per head
    both.reserve([-1] * 10 + [200, -1])
    for layer in range(3):
        keep = np.stack([np.sort(both.rng.choice(int(both.oracle.len[5]), 200, replace=False)) for _ in range(H)])
        both.cache.compact(layer, ints([5]), ints([10]), ints([0, 200]), torch.from_numpy(keep.astype(np.int32)).cuda(), max_kept=200)
        for h in range(H):
            k, v = both.oracle.rows(both.oracle.k, layer, 5, h).copy(), both.oracle.rows(both.oracle.v, layer, 5, h).copy()
            for r in range(200):
                both.oracle.put(layer, 10, r, h, k[keep[h, r]], v[keep[h, r]])
    both.trim([0] * 10 + [-1, 0])
    both.same_books()
    step(both, [10], Hq, [1])
    both.trim([0] * 12)
    both.same_books()
    assert both.cache.refs.abs().sum().item() == 0
    both.cache.check()
    path.close()


def test_a_decoding_step_replayed():
    """Grow, append, plan and attend captured once and replayed with other lengths, rows and batches (slots put in place
    of padding between replays); two graphs share one workspace; an eager call between them."""
    H, Hq, L = 2, 8, 2
    both = Both(kv_heads=H, page=16, n_pages=200, max_seqs=8, max_pages=60, layers=L, seed=4)
    both.fill([700, 0, 0, 0, 50, 3, 0, 0])
    both.fork([-1, 0, 0, 0, -1, -1, -1, -1])
    cache = both.cache
    slots, cu, want = ints([1, 2, 3, -1, 4, 5]), ints([0, 1, 2, 3, 4, 5, 6]), ints([-1] * 8)
    batch = cache.batch(slots, cu, n_tokens=6, n_q_heads=Hq)
    k_new = torch.zeros((L, 6, H, 128), dtype=torch.bfloat16, device="cuda")
    v_new, q, out = torch.zeros_like(k_new), torch.zeros((L, 6, Hq, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros((L, 6, Hq, 128), dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros((L, 6, Hq), device="cuda")

    def one(layers):
        cache.reserve(want)
        for layer in layers:
            cache.append(layer, batch, k_new[layer], v_new[layer])
        cache.plan(batch, share=2)
        for layer in layers:
            cache.attend(layer, batch, q[layer], out[layer], lse[layer])

    # Sets everything up; nothing grows, so that the forks' rows are refused (their last page is shared) and the others' land on
    # the last tokens, from where the oracle's are put back.
    one(range(L))
    assert B.asl_pages_status(cache.ctx, cache.pages)[0] == B.ASL_ERR_INVALID
    cache.k.copy_(both.dev(both.oracle.k)), cache.v.copy_(both.dev(both.oracle.v))
    torch.cuda.synchronize()
    graphs = []
    for layers in (range(L), range(L)):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, capture_error_mode="thread_local"):
            one(layers)
        graphs.append(g)
    for n, entries in enumerate(([1, 2, 3, -1, 4, 5], [1, 2, 3, 0, 4, 5], [2, -1, 3, 0, -1, 1], [-1, -1, -1, -1, -1, 4])):
        slots.copy_(ints(entries))
        new = [-1] * 8
        for s in entries:
            if s >= 0:
                new[s] = int(both.oracle.len[s]) + 1
        both.oracle.reserve(new)
        want.copy_(ints(new))
        k, v = both.new_rows(L, 6, H, 128)
        k_new.copy_(both.dev(k)), v_new.copy_(both.dev(v))
        qs = torch.from_numpy(both.rng.standard_normal((L, 6, Hq, 128))).to(torch.bfloat16)
        q.copy_(qs)
        out.fill_(7.0)
        graphs[n % 2].replay()
        torch.cuda.synchronize()
        for layer in range(L):
            for i, s in enumerate(entries):
                if s >= 0:
                    for h in range(H):
                        both.oracle.put(layer, s, int(both.oracle.len[s]) - 1, h, k[layer, i, h], v[layer, i, h])
            o, z, tol, tol_lse = both.expect(layer, entries, list(range(7)), qs[layer].double().numpy(), Hq)
            got, ok = out[layer].double().cpu().numpy(), ~np.isnan(z)
            assert (got[~ok] == 7.0).all()
            assert (np.abs(got[ok] - o[ok]) <= tol[ok]).all()
            assert (np.abs(lse[layer].double().cpu().numpy()[ok] - z[ok]) <= tol_lse[ok]).all()
        cache.check()
        both.same_books()
    both.same_rows()


def test_two_caches_on_two_streams():
    """Attention of two caches at once, each on a stream of its own that is not the current one's default."""
    a = Both(kv_heads=8, page=64, n_pages=120, max_seqs=20, max_pages=30, seed=1)
    b = Both(kv_heads=4, page=16, n_pages=200, max_seqs=5, max_pages=60, fp8=True, seed=2)
    a.fill([1200] + [0] * 19)
    a.fork([-1] + [0] * 19)
    a.fill([-1] + [1200 + 3 * i + 1 for i in range(19)])
    b.fill([900, 5, 77, 300, 64])
    work = []
    for both, heads, n in ((a, 32, 20), (b, 28, 5)):
        q = queries(both.rng, n, heads)
        slots, cu = list(range(n)), list(range(n + 1))
        work.append((both, heads, q, slots, cu, both.cache.batch(ints(slots), ints(cu), n_tokens=n, n_q_heads=heads), torch.cuda.Stream()))
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(8):
        for i, (both, heads, q, slots, cu, batch, stream) in enumerate(work):
            with torch.cuda.stream(stream):
                both.cache.plan(batch, share=2)
                outs[i].append(both.cache.attend(0, batch, q[0]))
    torch.cuda.synchronize()
    for i, (both, heads, q, slots, cu, batch, stream) in enumerate(work):
        both.cache.check()
        o, z, tol, _ = both.expect(0, slots, cu, q[1], heads)
        for out in outs[i]:
            assert (np.abs(out.double().cpu().numpy() - o) <= tol).all()


def test_pages_far_into_a_large_pool():
    """Rows beyond 4 GB of K and of V: pages at the end of a pool of 5 GB, shared and not, appended and pruned there."""
    H, page, n_pages = 8, 128, 20000
    shape = (1, n_pages, H, page, 128)
    k, v = torch.empty(shape, dtype=torch.bfloat16, device="cuda"), torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    table, length = torch.zeros((9, 12), dtype=torch.int32, device="cuda"), torch.zeros(9, dtype=torch.int32, device="cuda")
    refs = torch.ones(n_pages, dtype=torch.int32, device="cuda")
    refs[-60:] = 0
    cache = B.PagedCache(page_size=page, k=k, v=v, table=table, length=length, refs=refs)
    n = 1100
    cache.reserve(ints([n] + [-1] * 8))
    cache.fork(ints([-1] + [0] * 7 + [-1]))
    batch = cache.batch(ints([0]), ints([0, n]), n_tokens=n)
    g = torch.Generator(device="cuda").manual_seed(1)
    rows = [torch.randn((n, H, 128), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2)]
    cache.trim(ints([-1] + [0] * 7 + [-1]))                    # (appending wants the pages for itself)
    cache.append(0, batch, *rows)
    cache.fork(ints([-1] + [0] * 7 + [-1]))
    cache.reserve(ints([n + 1] * 8 + [100]))
    one = cache.batch(ints(range(8)), ints(range(9)), n_tokens=8, n_q_heads=32)
    tail = [torch.randn((8, H, 128), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2)]
    cache.append(0, one, *tail)
    q = torch.randn((8, 32, 128), generator=g, device="cuda").to(torch.bfloat16)
    assert int(table[0, 0]) >= n_pages - 60
    cache.plan(one, share=2)
    out = cache.attend(0, one, q)
    cache.plan(one, share=False)
    alone = cache.attend(0, one, q)
    idx = torch.arange(0, 1100, 11, dtype=torch.int32, device="cuda").repeat(H, 1).contiguous()
    cache.compact(0, ints([3]), ints([8]), ints([0, 100]), idx, max_kept=100)
    cache.check()
    for s in range(8):
        kk = torch.cat([rows[0], tail[0][s:s + 1]]).double().repeat_interleave(4, dim=1)
        vv = torch.cat([rows[1], tail[1][s:s + 1]]).double().repeat_interleave(4, dim=1)
        w = torch.softmax(torch.einsum("hd,nhd->hn", q[s].double(), kk) / 128 ** 0.5, dim=1)
        ref, scale = torch.einsum("hn,nhd->hd", w, vv), torch.einsum("hn,nhd->hd", w, vv.abs())
        # weights and the result rounded to bf16 (2^-8 each); fp32 sums over 1101 keys
        tol = 2.0 ** -8 * ref.abs() + scale * (2.0 ** -8 + 1101 * 2.0 ** -24 + 2.0 ** -10)
        assert ((out[s].double() - ref).abs() <= tol).all() and ((alone[s].double() - ref).abs() <= tol).all()
    got = k[0, table[8, 0].long(), :, :100].transpose(0, 1)
    assert torch.equal(got, rows[0][::11])


def test_as_many_sequences_as_a_batch_has():
    """4096 sequences of a few tokens each, half of them forks of one another."""
    n = 4096
    both = Both(kv_heads=1, page=16, n_pages=5000, max_seqs=n, max_pages=3)
    want = [(i % 40) + 1 if i % 2 == 0 else 0 for i in range(n)]
    both.fill(want)
    both.fork([i - 1 if i % 2 else -1 for i in range(n)])
    check_attention(both, 0, list(range(n)), list(range(n + 1)), 2, share=2)


def test_batches_that_are_not_ascending_are_refused():
    both = Both(kv_heads=2, page=16, n_pages=20, max_seqs=4, max_pages=8)
    both.fill([20, 30, 40, 50])
    for cu in ([0, 4, 0, 4, 4], [0, 1, 2, 3, 9], [-1, 0, 1, 2, 3]):
        batch = both.cache.batch(ints([0, 1, 2, 3]), ints(cu), n_tokens=4, n_q_heads=4)
        out = torch.full((4, 4, 128), 7.0, dtype=torch.bfloat16, device="cuda")
        both.cache.plan(batch)
        both.cache.attend(0, batch, torch.ones_like(out), out)
        assert B.asl_pages_status(both.cache.ctx, both.cache.pages) == (B.ASL_ERR_INVALID, -1)
        assert (out == 7.0).all()


def test_arguments_that_the_binding_refuses():
    both = Both(kv_heads=2, page=16, n_pages=20, max_seqs=4, max_pages=8)
    c = both.cache
    batch = c.batch(ints([0]), ints([0, 1]), n_tokens=1, n_q_heads=4)
    q = torch.zeros((1, 4, 128), dtype=torch.bfloat16, device="cuda")
    for call in (lambda: c.reserve(ints([1, 2])), lambda: c.reserve(torch.zeros(4, device="cuda")), lambda: c.fork(torch.zeros(4, dtype=torch.int32)),
                 lambda: c.batch(ints([0, 1]), ints([0, 1]), n_tokens=1), lambda: c.attend(0, batch, q[:, :3]), lambda: c.attend(0, batch, q.float()),
                 lambda: c.attend(1, batch, q), lambda: c.attend(0, batch, q.transpose(1, 2)), lambda: c.attend(0, batch, q, q[:, :2]),
                 lambda: c.attend(0, batch, q, None, torch.zeros((1, 3), device="cuda")),
                 lambda: c.append(0, batch, q, q), lambda: c.compact(0, ints([0]), ints([1]), ints([0]), ints([0])[None], max_kept=1),
                 lambda: B.PagedCache(page_size=16, n_kv_heads=2, n_pages=4, max_seqs=0, max_pages=1),
                 lambda: B.PagedCache(page_size=16, n_kv_heads=2, n_pages=4, max_seqs=1, max_pages=1, k_dtype=B.ASL_K_FP8_E4M3),
                 lambda: B.PagedCache(page_size=24, n_kv_heads=2, n_pages=4, max_seqs=1, max_pages=1)):
        with pytest.raises(B.AslError) as e:
            call()
        assert e.value.status in (B.ASL_ERR_INVALID, B.ASL_ERR_UNSUPPORTED)


def test_finished_requests_keep_their_pages():
    """Under the latching controller a request that has selected keeps what its selection layer stored."""
    wl = I.workload("C1", seqlens=(600,), budgets=(100,), layers=4, l_min=1, l_obs=2, tau=2.0)     # selects at its first evaluated layer
    path = make_path(wl)
    path.set_controller(B.ASL_CONTROLLER_LATCH)
    cache = B.PagedCache(page_size=16, n_layers=4, n_kv_heads=wl.n_kv_heads, n_pages=8, max_seqs=1, max_pages=8)
    cache.reserve(ints([100]))
    path.store_into(cache, ints([0]))
    for layer in range(4):
        x = I.layer_inputs(wl, layer, seed=2)
        path.run_layer(*[to_dev(x[n]) for n in ("q_obs", "k", "v")], layer, overlap=False)
    torch.cuda.synchronize()
    stat = path.read_stat()[0]
    assert stat["selected"] and stat["layer_idx"] == 1
    cache.check()
    filled = [bool((cache.v[layer] != 0).any()) for layer in range(4)]
    assert filled == [True, True, False, False]
    path.close()
