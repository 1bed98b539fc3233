"""GPU parity of the pages' operations: bookkeeping exact against the oracle's, rows bit for bit, refusals left alone."""
import numpy as np
import pytest
import torch

from oracle import pages_oracle as P
from paper_2601_07667_b200 import binding as B
from paper_2601_07667_b200 import inputs as I

from asl_check import make_path, to_dev, with_fp8_keys
from pages_check import Both, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("page,layers,fp8", [(16, 1, False), (32, 3, False), (64, 2, True), (128, 1, False)])
def test_a_random_history(page, layers, fp8):
    """Slots grow, fork, are cut and freed at random: table, lengths, counts and every copied row as the oracle has them."""
    slots, max_pages = 13, 9
    both = Both(kv_heads=2, page=page, n_pages=75, max_seqs=slots, max_pages=max_pages, layers=layers, fp8=fp8, seed=page)
    rng = np.random.default_rng(page + 1)
    for step in range(40):
        o = both.oracle
        what = step % 4
        if what in (0, 2):
            want = [int(n) + int(rng.choice([-1, 0, 1, page - 1, page, 2 * page + 3])) for n in o.len]
            want = [min(w, max_pages * page) if rng.random() < 0.6 else -1 for w in want]
            try:
                both.fill(want)
            except P.OutOfPages as e:
                both.cache.reserve(ints(want))
                assert B.asl_pages_status(both.cache.ctx, both.cache.pages) == (B.ASL_ERR_PAGES, e.missing)
        elif what == 1:
            free = [s for s in range(slots) if o.len[s] == 0]
            held = [s for s in range(slots) if o.len[s] > 0]
            parent = [-1] * slots
            for s in free[:5]:
                if held:
                    parent[s] = int(rng.choice(held))
            both.fork(parent)
        else:
            both.trim([int(rng.integers(0, n + 1)) if n and rng.random() < 0.4 else -1 for n in o.len])
        both.same_books()
        both.same_rows()
    both.trim([0] * slots)
    both.same_books()
    assert both.cache.refs.sum().item() == 0
    both.cache.check()


@pytest.mark.parametrize("n_pages,slots", [(31, 3), (1000, 40), (70001, 70), (1 << 20, 2100)])
def test_pages_of_any_pool(n_pages, slots):
    """Odd pools and the largest, more slots than a block has threads, one slot that takes many pages."""
    k = torch.zeros((1, n_pages, 1, 16, 128), dtype=torch.uint8, device="cuda")
    v = torch.empty((1, n_pages, 1, 16, 128), dtype=torch.bfloat16, device="cuda")
    table = torch.zeros((slots, 2048), dtype=torch.int32, device="cuda")
    length, refs = torch.zeros(slots, dtype=torch.int32, device="cuda"), torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    rng = np.random.default_rng(n_pages)
    held = rng.random(n_pages) < 0.3
    refs.copy_(torch.from_numpy(held.astype(np.int32)))
    cache = B.PagedCache(page_size=16, k=k, v=v, table=table, length=length, refs=refs, k_scale=torch.ones((1, 1)))
    free = np.flatnonzero(~held)
    want = rng.integers(1, 40, slots)
    want[1] = min(2048 * 16, 16 * (len(free) // 2))
    while (-(-want // 16)).sum() > len(free):
        want = np.maximum(1, want // 2)
    cache.reserve(ints(want))
    cache.check()
    at, tab = 0, table.cpu().numpy()
    for s, w in enumerate(want):
        m = -(-int(w) // 16)
        assert tab[s, :m].tolist() == free[at:at + m].tolist()
        at += m
    held[free[:at]] = True
    assert (refs.cpu().numpy() == held).all() and length.tolist() == want.tolist()
    # too many: nothing changes
    left = int((~held).sum())
    more = [-1] * slots
    more[0], more[2] = 2048 * 16, int(want[2]) + 16
    if left < 2048 - -(-int(want[0]) // 16) + 1:
        cache.reserve(ints(more))
        missing = 2048 - -(-int(want[0]) // 16) + 1 - left
        assert B.asl_pages_status(cache.ctx, cache.pages) == (B.ASL_ERR_PAGES, missing)
        assert (refs.cpu().numpy() == held).all() and length.tolist() == want.tolist()


def test_wants_and_forks_that_do_not_fit():
    both = Both(kv_heads=1, page=16, n_pages=40, max_seqs=6, max_pages=4)
    both.fill([20, 5, 0, 0, 0, 0])
    both.cache.reserve(ints([-1, 65, 3, -1, -1, -1]))                 # slot 1: more than its row of the table holds
    assert B.asl_pages_status(both.cache.ctx, both.cache.pages) == (B.ASL_ERR_INVALID, 1)
    both.same_books()
    # into a held slot, from a slot that is itself forked, from itself, from no slot; the fork that fits is made
    both.oracle.fork([-1, 0, 0, 2, 4, 99])
    both.cache.fork(ints([-1, 0, 0, 2, 4, 99]))
    st, slot = B.asl_pages_status(both.cache.ctx, both.cache.pages)
    assert st == B.ASL_ERR_INVALID and slot in (1, 3, 4, 5)
    both.same_books()
    assert both.cache.len.tolist() == [20, 5, 20, 0, 0, 0]


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("page", [16, 64])
def test_append_of_packed_and_strided_rows(page, fp8):
    """Tokens of several sequences, none for one of them, padding, rows behind the last; K and V inside a wider tensor."""
    H, layers = 4, 2
    both = Both(kv_heads=H, page=page, n_pages=60, max_seqs=7, max_pages=8, layers=layers, fp8=fp8, seed=3)
    both.fill([30, 0, 70, 1, 16, 0, 0])
    both.fork([-1, 0, -1, -1, -1, 2, -1])
    counts, slots = [3, 1, 0, 40, 2, 17], [1, 5, 3, 0, -1, 4]
    want = [-1] * 7
    for s, c in zip(slots, counts):
        if s >= 0:
            want[s] = int(both.oracle.len[s]) + c
    both.reserve(want)
    cu = np.concatenate([[0], np.cumsum(counts)])
    n_tokens = int(cu[-1]) + 5
    batch = both.cache.batch(ints(slots), ints(cu), n_tokens=n_tokens)
    for layer in range(layers):
        k, v = both.new_rows(n_tokens, 3 * H, 128)
        both.cache.append(layer, batch, both.dev(k)[:, H:2 * H], both.dev(v)[:, 2 * H:])
        for i, s in enumerate(slots):
            for t in range(counts[i] if s >= 0 else 0):
                for h in range(H):
                    both.oracle.put(layer, s, int(both.oracle.len[s]) - counts[i] + t, h, k[cu[i] + t, H + h], v[cu[i] + t, 2 * H + h])
    both.cache.check()
    both.same_books()
    both.same_rows()


def test_append_leaves_shared_pages_and_missing_rows_alone():
    both = Both(kv_heads=2, page=16, n_pages=10, max_seqs=3, max_pages=4)
    both.fill([20, 0, 2])
    both.fork([-1, 0, -1])
    k, v = both.new_rows(5, 2, 128)
    batch = both.cache.batch(ints([1, 2]), ints([0, 1, 5]), n_tokens=5)    # slot 1's last page is shared; slot 2 has 2 tokens, not 4
    both.cache.append(0, batch, both.dev(k), both.dev(v))
    st, slot = B.asl_pages_status(both.cache.ctx, both.cache.pages)
    assert st == B.ASL_ERR_INVALID and slot in (1, 2)
    for t in (2, 3):
        for h in range(2):
            both.oracle.put(0, 2, t - 2, h, k[1 + t, h], v[1 + t, h])
    both.same_rows()


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("page", [16, 128])
def test_store_of_a_prefills_kept_rows(page, fp8):
    """asl_pages_store against asl_compact_kv on the same lists; K and V rows bit for bit, slots out of order."""
    w = 32
    seqlens, kept = (65, 80, 200, 300, 500), (64, 65, 127, 193, 500)
    wl = I.workload("C3", n_q_heads=16, n_kv_heads=4, window=w, seqlens=seqlens, budgets=kept, layers=1, l_min=1, l_obs=2)
    x = I.layer_inputs(wl, 0, seed=3)
    launch = {}
    if fp8:
        x = with_fp8_keys(x)
        launch = dict(k_dtype=B.ASL_K_FP8_E4M3, k_scale=[float(s) for s in x["k_scale"]])
    path = make_path(wl, **launch)
    both = Both(kv_heads=4, page=page, n_pages=90, max_seqs=6, max_pages=40, fp8=fp8)
    rng, cu = np.random.default_rng(4), wl.cu_seqlens()
    idx = np.stack([np.concatenate([np.sort(rng.choice(n, m, replace=False)) for n, m in zip(seqlens, kept)]) for _ in range(4)])
    slots = [5, 0, 2, 1, 4]
    want = [-1] * 6
    for s, m in zip(slots, kept):
        want[s] = m
    both.reserve(want)
    both.cache.store(0, path, to_dev(x["k"]), to_dev(x["v"]), torch.from_numpy(idx.astype(np.int32)).cuda(), ints(slots))
    both.cache.check()
    at = 0
    for b, m in enumerate(kept):
        for h in range(4):
            for r in range(m):
                t = cu[b] + idx[h, at + r]
                both.oracle.put(0, slots[b], r, h, x["k"][t, h], x["v"][t, h])
        at += m
    both.same_rows()
    path.close()


def test_layers_of_a_prompt_straight_into_pages():
    """run_layer with store_into: the pages hold what k_out and v_out would, two layers in flight."""
    wl = I.workload("C1", seqlens=(700, 900), budgets=(100, 333), layers=3)
    dense, paged = make_path(wl), make_path(wl)
    H = wl.n_kv_heads
    cache = B.PagedCache(page_size=32, n_layers=3, n_kv_heads=H, n_pages=20, max_seqs=3, max_pages=11)
    slots = ints([2, 0])
    cache.reserve(ints([333, -1, 100]))
    paged.store_into(cache, slots)
    want, alive = [], []
    for layer in range(3):
        x = I.layer_inputs(wl, layer, seed=5)
        args = [to_dev(x[n]) for n in ("q_obs", "k", "v")]
        alive.append(args)
        dense.run_layer(*args, layer)
        dense.join()
        want.append((dense.k_out.clone(), dense.v_out.clone()))
        paged.run_layer(*args, layer)
    paged.join()
    cache.check()
    table = cache.table.cpu().numpy()
    for layer in range(3):
        for pool, ref in zip((cache.k, cache.v), want[layer]):
            for b, (slot, m, off) in enumerate(((2, 100, 0), (0, 333, 100))):
                ids = torch.from_numpy(table[slot, :-(-m // 32)].astype(np.int64)).cuda()
                got = pool[layer, ids].transpose(0, 1).reshape(H, -1, 128)[:, :m]
                assert torch.equal(got.view(torch.int16), ref[:, off:off + m].view(torch.int16)), (layer, b)
    assert torch.equal(dense.stat, paged.stat)
    paged.store_into(None)
    paged.run_layer(*alive[-1], 3, overlap=False)
    dense.run_layer(*alive[-1], 3, overlap=False)
    assert torch.equal(paged.k_out.view(torch.int16), dense.k_out.view(torch.int16))
    dense.close(), paged.close()


@pytest.mark.parametrize("fp8", [False, True])
def test_cached_sequences_pruned_into_other_slots(fp8):
    """From shared pages, lists of 1 to all tokens, one empty; then the old slots are freed."""
    H, layers, page = 3, 2, 32
    both = Both(kv_heads=H, page=page, n_pages=60, max_seqs=9, max_pages=12, layers=layers, fp8=fp8, seed=2)
    both.fill([100, 0, 333, 64, 0, 0, 0, 0, 0])
    both.fork([-1, 0, -1, -1, -1, -1, -1, -1, -1])
    both.fill([-1, 110, -1, -1, -1, -1, -1, -1, -1])
    src, dst, m = [1, 2, 3, 0], [5, 4, 8, 7], [65, 200, 64, 0]
    want = [-1] * 9
    for d, n in zip(dst, m):
        want[d] = n
    both.reserve(want)
    off = np.concatenate([[0], np.cumsum(m)])
    for layer in range(layers):
        idx = np.stack([np.concatenate([np.sort(both.rng.choice(int(both.oracle.len[s]), n, replace=False)) for s, n in zip(src, m)]) for _ in range(H)])
        both.cache.compact(layer, ints(src), ints(dst), ints(off), torch.from_numpy(idx.astype(np.int32)).cuda(), max_kept=max(m))
        for j, (s, d) in enumerate(zip(src, dst)):
            for h in range(H):
                k, v = both.oracle.rows(both.oracle.k, layer, s, h).copy(), both.oracle.rows(both.oracle.v, layer, s, h).copy()
                for r in range(m[j]):
                    t = int(idx[h, off[j] + r])
                    both.oracle.put(layer, d, r, h, k[t], v[t])
    both.cache.check()
    both.same_rows()
    both.trim([0, 0, 0, 0, -1, -1, -1, -1, -1])
    both.same_books()


def test_pruning_leaves_out_what_does_not_fit():
    """A slot onto itself, positions that a sequence does not have, rows that no page was reserved for, shared pages."""
    both = Both(kv_heads=1, page=16, n_pages=30, max_seqs=8, max_pages=4)
    both.fill([40, 0, 0, 20, 0, 0, 0, 0])
    both.fork([-1, -1, -1, -1, 3, -1, -1, -1])
    both.reserve([-1, 10, 10, -1, -1, -1, -1, -1])
    src, dst, m = [0, 0, 0, 0, 0], [0, 1, 2, 4, 77], [5, 10, 12, 20, 3]
    off = np.concatenate([[0], np.cumsum(m)])
    idx = np.arange(off[-1]) % 40
    idx[off[1] + 4] = 40                                          # one past the end
    idx[off[1] + 5] = -3
    both.cache.compact(0, ints(src), ints(dst), ints(off), ints(idx)[None], max_kept=20)
    assert B.asl_pages_status(both.cache.ctx, both.cache.pages)[0] == B.ASL_ERR_INVALID
    k, v = both.oracle.rows(both.oracle.k, 0, 0, 0).copy(), both.oracle.rows(both.oracle.v, 0, 0, 0).copy()
    for j, d, rows in ((1, 1, [0, 1, 2, 3, 6, 7, 8, 9]), (2, 2, range(10))):
        for r in rows:
            both.oracle.put(0, d, r, 0, k[idx[off[j] + r]], v[idx[off[j] + r]])
    both.same_rows()
    both.same_books()
    assert B.asl_pages_status(both.cache.ctx, both.cache.pages) == (B.ASL_OK, 0)
