"""The paged cache's entry points by their plain functions, one for each, on a stream that is named: the same books, rows and results as
by PagedCache's calls."""
import torch

import pytest

from paper_2601_07667_b200 import binding as B

from pages_check import Both, ints, queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fp8", [False, True])
def test_a_round_by_plain_functions(fp8):
    a, b = (Both(kv_heads=2, page=16, n_pages=120, max_seqs=8, max_pages=30, layers=2, fp8=fp8, seed=4) for _ in range(2))
    for both in (a, b):
        both.fill([200, 33] + [0] * 6)
    cache, ctx, pages, stream = b.cache, b.cache.ctx, b.cache.pages, torch.cuda.Stream()
    parent, want, to = ints([-1, -1, 0, 0, 0, 1, -1, -1]), ints([-1, -1, 203, 201, 209, 34, 50, -1]), ints([-1] * 5 + [0, -1, -1])
    slots, cu = ints([2, 3, 4, 5]), ints([0, 3, 4, 13, 14])
    k, v = a.new_rows(2, 14, 2, 128)
    k, v = a.dev(k), a.dev(v)
    q = queries(a.rng, 14, 8)[0]
    idx = torch.stack([torch.arange(h, 200, 4) for h in range(2)]).to(torch.int32).cuda()

    a.cache.fork(parent)
    a.cache.reserve(want)
    batch = a.cache.batch(slots, cu, n_tokens=14, n_q_heads=8)
    outs, lses = [], []
    for layer in range(2):
        a.cache.append(layer, batch, k[layer], v[layer])
    a.cache.plan(batch, share=2)
    for layer in range(2):
        lses.append(torch.empty((14, 8), device="cuda"))
        outs.append(a.cache.attend(layer, batch, q, lse=lses[-1]))
        a.cache.compact(layer, ints([3]), ints([6]), ints([0, 50]), idx, max_kept=50)
    a.cache.trim(to)
    a.cache.check()

    torch.cuda.synchronize()
    rows = (2 * 128, 128)
    B.asl_pages_fork(ctx, pages, parent, stream)
    B.asl_pages_reserve(ctx, pages, want, stream)
    step = B.AslBatch(4, 14, slots.data_ptr(), cu.data_ptr())
    for layer in range(2):
        B.asl_pages_append(ctx, pages, layer, step, k[layer], v[layer], rows, rows, stream)
    size = B.asl_attend_workspace(ctx, pages, step, 8)
    workspace = torch.zeros(size, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    B.asl_attend_plan(ctx, pages, step, 8, 2, workspace, size, stream)
    off, src, dst = ints([0, 50]), ints([3]), ints([6])
    got = [(torch.empty_like(outs[0]), torch.empty_like(lses[0])) for _ in range(2)]
    torch.cuda.synchronize()
    for layer in range(2):
        B.asl_attend(ctx, pages, layer, step, 8, 2, q, (8 * 128, 128), got[layer][0], got[layer][1], workspace, size, stream)
        B.asl_pages_compact(ctx, pages, layer, src, dst, off, 1, idx, 50, 50, stream)
    B.asl_pages_trim(ctx, pages, to, stream)
    assert B.asl_pages_status(ctx, pages, stream) == (B.ASL_OK, 0)
    assert B.asl_device_status(ctx, stream)[0] == B.ASL_OK

    for layer in range(2):
        assert torch.equal(got[layer][0], outs[layer]) and torch.equal(got[layer][1], lses[layer])
    for x, y in zip((a.cache.len, a.cache.refs, a.cache.k, a.cache.v), (cache.len, cache.refs, cache.k, cache.v)):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    with pytest.raises(B.AslError) as e:
        B.asl_attend(ctx, pages, 0, step, 8, 2, q, (8 * 128, 128), got[0][0], None, workspace, size - 1, stream)
    assert e.value.status == B.ASL_ERR_WORKSPACE
