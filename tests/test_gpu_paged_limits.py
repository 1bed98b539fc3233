"""The paged cache at its limits: sizes around what a kernel's shared memory holds by default, steps and lists without rows, lists
and slots that do not fit."""
import numpy as np
import pytest
import torch

from paper_2601_07667_b200 import binding as B
from paper_2601_07667_b200 import inputs as I

from asl_check import make_path, to_dev
from pages_check import Both, check_attention, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_pages", [392064, 392065, 392500, 393216, 393217])
def test_a_pool_whose_books_are_about_48_kb(n_pages):
    """Each pool on a context of its own: slots grow over what is free, with a copy of a shared last page."""
    k = torch.zeros((1, n_pages, 1, 16, 128), dtype=torch.uint8, device="cuda")
    v = torch.zeros((1, n_pages, 1, 16, 128), dtype=torch.bfloat16, device="cuda")
    table, length = torch.zeros((3, 64), dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    refs = torch.ones(n_pages, dtype=torch.int32, device="cuda")
    free = [5, 70000, 392000, 392063, n_pages - 2, n_pages - 1]
    free = sorted(set(free))
    refs[torch.tensor(free, device="cuda")] = 0
    cache = B.PagedCache(page_size=16, k=k, v=v, table=table, length=length, refs=refs, k_scale=torch.ones((1, 1)))
    cache.reserve(ints([20, -1, -1]))
    cache.fork(ints([-1, 0, -1]))
    cache.reserve(ints([-1, 21, -1]))
    cache.check()
    assert length.tolist() == [20, 21, 0]
    assert table[0, :2].tolist() == free[:2] and table[1, :2].tolist() == [free[0], free[2]]
    assert [int(refs[p]) for p in free[:4]] == [2, 1, 1, 0]
    cache.close()


@pytest.mark.parametrize("n", [1019, 1020, 1021, 1022, 1023, 1024, 1025])
def test_a_batch_whose_plan_is_about_48_kb(n):
    """Each batch on a context of its own; every third sequence a fork of the one before it, one free slot."""
    both = Both(kv_heads=1, page=16, n_pages=2 * n, max_seqs=n, max_pages=3, seed=n)
    both.fill([(i % 40) + 1 if i % 3 and i != 7 else 0 for i in range(n)])
    both.fork([i - 1 if i % 3 == 0 and i else -1 for i in range(n)])
    check_attention(both, 0, list(range(n)), list(range(n + 1)), 2, share=2)
    both.cache.close()


def test_a_step_without_tokens():
    """Every sequence has ended: a batch of padding and of free slots without a token, through every call of a step."""
    both = Both(kv_heads=2, page=16, n_pages=20, max_seqs=4, max_pages=8)
    both.fill([20, 0, 40, 0])
    c = both.cache
    batch = c.batch(ints([-1, 0, 1]), ints([0, 0, 0, 0]), n_tokens=0, n_q_heads=4)
    rows, q = torch.empty((0, 2, 128), dtype=torch.bfloat16, device="cuda"), torch.empty((0, 4, 128), dtype=torch.bfloat16, device="cuda")
    c.append(0, batch, rows, rows)
    for share in (0, 1, 2):
        c.plan(batch, share=share)
        out = c.attend(0, batch, q, lse=torch.empty((0, 4), device="cuda"))
        assert out.shape == (0, 4, 128)
    c.check()
    both.same_books()
    both.same_rows()


@pytest.mark.parametrize("off,max_kept", [([-2, 3, 6], 6), ([0, 3, 7], 6), ([0, 4, 2], 6), ([3, 9, 6], 6), ([0, 0, 2 ** 31 - 1], 6), ([-2 ** 31, 3, 6], 6)])
def test_lists_that_are_not_there_are_noted(off, max_kept):
    """A job whose list begins or ends outside all lists is left out and noted; the other one, where its list is good, is done."""
    both = Both(kv_heads=1, page=16, n_pages=30, max_seqs=6, max_pages=4, seed=1)
    both.fill([40, 30, 0, 0, 0, 0])
    both.reserve([-1, -1, 10, 10, -1, -1])
    idx = [3, 5, 9, 11, 17, 29]
    both.cache.compact(0, ints([0, 1]), ints([2, 3]), ints(off), ints(idx)[None], max_kept=max_kept)
    st, slot = B.asl_pages_status(both.cache.ctx, both.cache.pages)
    good = [0 <= off[j] <= off[j + 1] <= 6 for j in range(2)]
    assert st == B.ASL_ERR_INVALID and slot in [s for s, ok in zip((2, 3), good) if not ok]
    for j, (s, d) in enumerate(((0, 2), (1, 3))):
        if good[j]:
            k, v = both.oracle.rows(both.oracle.k, 0, s, 0).copy(), both.oracle.rows(both.oracle.v, 0, s, 0).copy()
            for r, t in enumerate(idx[off[j]:off[j + 1]]):
                both.oracle.put(0, d, r, 0, k[t], v[t])
    both.same_rows()


def test_nothing_kept_of_any_sequence():
    both = Both(kv_heads=2, page=16, n_pages=30, max_seqs=4, max_pages=4, seed=1)
    both.fill([40, 30, 0, 0])
    none = torch.empty((2, 0), dtype=torch.int32, device="cuda")
    both.cache.compact(0, ints([0, 1]), ints([2, 3]), ints([0, 0, 0]), none, max_kept=0)
    both.cache.check()
    both.cache.compact(0, ints([0, 1]), ints([2, 3]), ints([0, 0, 1]), none, max_kept=0)
    assert B.asl_pages_status(both.cache.ctx, both.cache.pages) == (B.ASL_ERR_INVALID, 3)
    both.same_rows()
    both.same_books()


@pytest.mark.parametrize("n_jobs", [4, 300])
def test_slots_that_another_job_needs_are_left_alone(n_jobs):
    """Jobs run side by side: one that would write a slot whose rows another reads, or that another writes too, is left out and
    noted; those of other slots are done, and a slot may be read by several."""
    both = Both(kv_heads=2, page=16, n_pages=700, max_seqs=n_jobs + 6, max_pages=4, seed=2)
    both.fill([40, 30, 20, 50] + [0] * (n_jobs + 2))
    both.reserve([-1] * 4 + [10] * (n_jobs + 2))
    src, dst = [0, 1, 1, 3] + [0] * (n_jobs - 4), [1, 4, 5, 5] + list(range(6, n_jobs + 2))
    if n_jobs > 4:
        src[-1], dst[-1] = 9, n_jobs + 4               # reads what another job writes: that one is left out
    done = [j for j in range(n_jobs) if j not in (0, 2, 3) and not (n_jobs > 4 and dst[j] == 9)]
    idx = np.stack([np.concatenate([np.sort(both.rng.choice(10, 5, replace=False)) for _ in range(n_jobs)]) for _ in range(2)])
    both.cache.compact(0, ints(src), ints(dst), ints(range(0, 5 * n_jobs + 1, 5)), torch.from_numpy(idx.astype(np.int32)).cuda(), max_kept=5)
    st, slot = B.asl_pages_status(both.cache.ctx, both.cache.pages)
    assert st == B.ASL_ERR_INVALID and slot in (1, 5, 9)
    for j in done:
        for h in range(2):
            k, v = both.oracle.rows(both.oracle.k, 0, src[j], h).copy(), both.oracle.rows(both.oracle.v, 0, src[j], h).copy()
            for r in range(5):
                both.oracle.put(0, dst[j], r, h, k[idx[h, 5 * j + r]], v[idx[h, 5 * j + r]])
    both.same_rows()


def test_a_job_without_rows_takes_no_slot_from_another():
    """Empty lists read and write nothing: their slots may be anybody's."""
    both = Both(kv_heads=1, page=16, n_pages=20, max_seqs=4, max_pages=4, seed=2)
    both.fill([40, 30, 0, 0])
    both.reserve([-1, -1, 10, -1])
    k, v = both.oracle.rows(both.oracle.k, 0, 0, 0).copy(), both.oracle.rows(both.oracle.v, 0, 0, 0).copy()
    both.cache.compact(0, ints([0, 2, 1]), ints([2, 0, 2]), ints([0, 3, 3, 3]), ints([7, 8, 30])[None], max_kept=3)
    both.cache.check()
    for r, t in enumerate((7, 8, 30)):
        both.oracle.put(0, 2, r, 0, k[t], v[t])
    both.same_rows()


def test_requests_that_share_a_slot_are_not_stored():
    wl = I.workload("C3", n_q_heads=8, n_kv_heads=2, window=32, seqlens=(100, 200, 150), budgets=(64, 64, 64), layers=1, l_min=1, l_obs=2)
    x = I.layer_inputs(wl, 0, seed=3)
    path = make_path(wl)
    both = Both(kv_heads=2, page=16, n_pages=30, max_seqs=3, max_pages=6)
    both.reserve([64, 64, -1])
    idx = np.stack([np.concatenate([np.sort(both.rng.choice(n, 64, replace=False)) for n in (100, 200, 150)]) for _ in range(2)])
    both.cache.store(0, path, to_dev(x["k"]), to_dev(x["v"]), torch.from_numpy(idx.astype(np.int32)).cuda(), ints([1, 0, 1]))
    assert B.asl_pages_status(both.cache.ctx, both.cache.pages) == (B.ASL_ERR_INVALID, 1)
    for h in range(2):
        for r in range(64):
            t = 100 + idx[h, 64 + r]
            both.oracle.put(0, 0, r, h, x["k"][t, h], x["v"][t, h])
    both.same_rows()
    path.close()


@pytest.mark.parametrize("slots,each", [(3, 1 << 20), (40, 1 << 20), (1100, 3000), (2100, 1 << 20)])
def test_how_many_pages_are_missing(slots, each):
    """Wants of far more pages than any pool has are counted to the last page (2^31 - 1 stands for all above)."""
    k = torch.zeros((1, 50, 1, 16, 128), dtype=torch.bfloat16, device="cuda")
    length, refs = torch.zeros(slots, dtype=torch.int32, device="cuda"), torch.zeros(50, dtype=torch.int32, device="cuda")
    cache = B.PagedCache(page_size=16, k=k, v=k.clone(), table=torch.zeros((slots, each), dtype=torch.int32, device="cuda"), length=length, refs=refs)
    cache.reserve(ints([20] + [-1] * (slots - 1)))
    cache.fork(ints([-1, 0] + [-1] * (slots - 2)))
    cache.reserve(ints([each * 16] * slots))
    # the first two need a page for the copy of what they share besides, and hold two already
    missing = min(slots * each - 4 + 2 - 48, 2 ** 31 - 1)
    assert B.asl_pages_status(cache.ctx, cache.pages) == (B.ASL_ERR_PAGES, missing)
    assert length[:3].tolist() == [20, 20, 0] and refs.sum().item() == 4


def test_the_smallest_cache():
    """One page, one slot, one head: every call, up to the page's end and over it."""
    both = Both(kv_heads=1, page=16, n_pages=1, max_seqs=1, max_pages=1)
    both.fill([1])
    check_attention(both, 0, [0], [0, 1], 1, share=2)
    both.fill([16])
    check_attention(both, 0, [0], [0, 16], 1, share=1)
    both.cache.reserve(ints([17]))
    assert B.asl_pages_status(both.cache.ctx, both.cache.pages) == (B.ASL_ERR_INVALID, 0)
    both.trim([15])
    both.same_books()
    check_attention(both, 0, [0], [0, 2], 3, share=2)
    both.trim([0])
    both.same_books()
    check_attention(both, 0, [0], [0, 1], 1, share=2)


@pytest.mark.parametrize("kv_heads,group,page,fp8", [(300, 1, 16, False), (257, 3, 16, True), (40, 128, 32, False)])
def test_many_heads(kv_heads, group, page, fp8):
    both = Both(kv_heads=kv_heads, page=page, n_pages=30, max_seqs=6, max_pages=10, layers=2, fp8=fp8, seed=1)
    both.fill([150, 0, 0, 0, 5, 0])
    both.fork([-1, 0, 0, 0, -1, -1])
    both.fill([-1, 151, 155, 152, -1, -1])
    both.reserve([-1] * 5 + [9])
    for share in (0, 2):
        check_attention(both, 1, [1, 2, 3, 4], [0, 1, 3, 4, 5], kv_heads * group, share=share)
    idx = np.stack([np.sort(both.rng.choice(150, 9, replace=False)) for _ in range(kv_heads)])
    both.cache.compact(1, ints([0]), ints([5]), ints([0, 9]), torch.from_numpy(idx.astype(np.int32)).cuda(), max_kept=9)
    for h in range(kv_heads):
        k, v = both.oracle.rows(both.oracle.k, 1, 0, h).copy(), both.oracle.rows(both.oracle.v, 1, 0, h).copy()
        for r in range(9):
            both.oracle.put(1, 5, r, h, k[idx[h, r]], v[idx[h, r]])
    both.cache.check()
    both.same_rows()
    both.same_books()


def test_as_many_slots_as_a_cache_has():
    """65536 slots: the last ones and some between grow, fork, are cut and freed."""
    n = 65536
    both = Both(kv_heads=1, page=16, n_pages=3000, max_seqs=n, max_pages=5, seed=1)
    some = [0, 1023, 1024, 30000, n - 2]
    want = [-1] * n
    for i, s in enumerate(some):
        want[s] = 20 + i
    both.fill(want)
    parent = [-1] * n
    for i in range(1000):
        parent[40000 + i] = some[i % 5]
    parent[n - 1] = n - 2
    both.fork(parent)
    want = [-1] * n
    for i in list(range(40000, 41000)) + [n - 1]:
        want[i] = 40
    both.reserve(want)
    both.same_books()
    both.same_rows()
    both.trim([0 if i % 3 else -1 for i in range(n)])
    both.same_books()
    both.cache.check()
