"""Calls of the paged cache at the same time and captured: attention of several batches of one cache on streams of their own, a prompt's
layers captured into pages; tokens that stand before their sequence's beginning."""
import numpy as np
import pytest
import torch

from paper_2601_07667_b200 import binding as B
from paper_2601_07667_b200 import inputs as I

from asl_check import make_path, to_dev, with_fp8_keys
from pages_check import Both, check_attention, ints, queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fp8", [False, True])
def test_batches_of_one_cache_on_streams_of_their_own(fp8):
    """asl_attend only reads the cache: three batches at once, shared prefixes and not, each with the bits that it has alone."""
    both = Both(kv_heads=4, page=16, n_pages=500, max_seqs=24, max_pages=90, layers=2, fp8=fp8, seed=3)
    both.fill([1200] + [0] * 15 + [700, 30, 900, 64, 1, 333, 80, 1000])
    both.fork([-1] + [0] * 15 + [-1] * 8)
    both.fill([-1] + [1201 + 5 * i for i in range(15)] + [-1] * 8)
    c, work = both.cache, []
    for slots, share in ((list(range(1, 16)), 2), (list(range(16, 24)), 0), (list(range(8, 20)), 2)):
        n = len(slots)
        batch = c.batch(ints(slots), ints(range(n + 1)), n_tokens=n, n_q_heads=16)
        c.plan(batch, share=share)
        q, exact = queries(both.rng, n, 16)
        alone = [c.attend(layer, batch, q) for layer in range(2)]
        o, _, tol, _ = both.expect(0, slots, list(range(n + 1)), exact, 16)
        assert (np.abs(alone[0].double().cpu().numpy() - o) <= tol).all()
        work.append((batch, q, alone, torch.cuda.Stream()))
    torch.cuda.synchronize()
    got = [[] for _ in work]
    for _ in range(10):
        for i, (batch, q, _, stream) in enumerate(work):
            with torch.cuda.stream(stream):
                got[i] += [c.attend(layer, batch, q) for layer in range(2)]
    torch.cuda.synchronize()
    for (_, _, alone, _), outs in zip(work, got):
        assert all(torch.equal(out, alone[j % 2]) for j, out in enumerate(outs))
    c.check()


@pytest.mark.parametrize("fp8", [False, True])
def test_a_prompts_layers_captured_into_pages(fp8):
    """run_layer with store_into under a graph, replayed with other keys and values and into other slots."""
    wl = I.workload("C3", n_q_heads=16, n_kv_heads=4, window=32, seqlens=(700, 900), budgets=(100, 333), layers=2)
    xs = [[I.layer_inputs(wl, layer, seed=seed) for layer in range(2)] for seed in (5, 6)]
    launch = {}
    if fp8:
        xs = [[with_fp8_keys(x) for x in two] for two in xs]
        launch = dict(k_dtype=B.ASL_K_FP8_E4M3, k_scale=[float(s) for s in xs[0][0]["k_scale"]])
    path, dense = make_path(wl, **launch), make_path(wl, **launch)
    cache = B.PagedCache(page_size=16, n_layers=2, n_kv_heads=4, n_pages=60, max_seqs=4, max_pages=21, k_dtype=B.ASL_K_FP8_E4M3 if fp8 else B.ASL_K_BF16,
                         k_scale=torch.ones((2, 4)) if fp8 else None)
    cache.reserve(ints([333, 100, 333, 100]))
    slots = ints([1, 0])
    path.store_into(cache, slots)
    names = ("q_obs", "k", "v")
    held = [[to_dev(x[n]) for n in names] for x in xs[0]]
    for layer in range(2):
        path.run_layer(*held[layer], layer)
    path.join()
    graph = path.capture([(*held[layer], layer) for layer in range(2)])
    for x, at in ((xs[1], [3, 2]), (xs[0], [1, 2]), (xs[1], [1, 0])):
        slots.copy_(ints(at))
        for layer in range(2):
            for t, n in zip(held[layer], names):
                t.copy_(to_dev(x[layer][n]))
        path.reset()
        cache.k.zero_(), cache.v.zero_()
        graph.replay()
        cache.check()
        dense.reset()
        for layer in range(2):
            dense.run_layer(*held[layer], layer)
            dense.join()
            for pool, ref in ((cache.k, dense.k_out), (cache.v, dense.v_out)):
                for slot, m, off in ((at[0], 100, 0), (at[1], 333, 100)):
                    got = pool[layer, cache.table[slot, :-(-m // 16)].long()].transpose(0, 1).reshape(4, -1, 128)[:, :m]
                    assert torch.equal(got.view(torch.uint8), ref[:, off:off + m].view(torch.uint8)), (layer, slot)
    path.close(), dense.close()


@pytest.mark.parametrize("page,fp8", [(16, False), (64, True)])
def test_tokens_before_their_sequences_beginning(page, fp8):
    """More tokens than a sequence holds: the first ones see no key, whatever lies in its pages, beside sequences that share a prompt."""
    lens = [3, 1, 0, 40]
    both = Both(kv_heads=2, page=page, n_pages=60, max_seqs=9, max_pages=-(-330 // page), fp8=fp8, seed=7)
    both.fill(lens + [300, 0, 0, 0, 0])
    both.fork([-1] * 5 + [4] * 4)
    both.fill([-1] * 5 + [301, 302, 310, 305])
    slots = [0, 5, 6, 1, 7, 8, 2, 3]
    counts = [7, 1, 2, 33, 3, 1, 4, 41]
    cu = np.concatenate([[0], np.cumsum(counts)]).tolist()
    for share in (0, 2):
        check_attention(both, 0, slots, cu, 8, share=share)


def spoil(n_bytes, count):
    """Takes as much of the allocator's memory as `count` tensors of that size and fills it."""
    return [torch.full((n_bytes,), 0xff, dtype=torch.uint8, device="cuda") for _ in range(count)]


def test_a_batch_dropped_while_another_stream_is_at_work():
    """The batch belongs to one stream's memory and is used on another: what it held is not given away before that one has read it."""
    both = Both(kv_heads=2, page=16, n_pages=60, max_seqs=6, max_pages=12, seed=5)
    both.fill([100, 30, 64, 1, 17, 90])
    c, q = both.cache, queries(both.rng, 6, 8)
    k, v = [both.dev(x) for x in both.new_rows(6, 2, 128)]
    batch = c.batch(ints(range(6)), ints(range(7)), n_tokens=6, n_q_heads=8)
    c.append(0, batch, k, v)
    c.plan(batch)
    right = c.attend(0, batch, q[0])
    c.check()
    page, side = int(both.oracle.table[0, 99 // 16]), torch.cuda.Stream()
    for _ in range(3):
        batch = c.batch(ints(range(6)), ints(range(7)), n_tokens=6, n_q_heads=8)
        c.k[0, page, :, 99 % 16] = 0
        torch.cuda.synchronize()
        size = batch.ws_bytes
        with torch.cuda.stream(side):
            c.plan(batch)
            torch.cuda._sleep(200_000_000)
            c.append(0, batch, k, v)
            out = c.attend(0, batch, q[0])
        del batch
        held = spoil(size, 1) + spoil(64, 3000)
        torch.cuda.synchronize()
        c.check()
        del held
        assert torch.equal(c.k[0, page, :, 99 % 16].view(torch.int16), k[0].view(torch.int16))
        assert torch.equal(out, right)


def test_slots_replaced_while_a_layer_is_stored():
    """store_into's slots are read on a side stream, which may be behind when the path is given others."""
    wl = I.workload("C3", n_q_heads=8, n_kv_heads=2, window=32, seqlens=(100, 200), budgets=(64, 64), layers=1, l_min=1, l_obs=2)
    x = I.layer_inputs(wl, 0, seed=3)
    path, dense = make_path(wl), make_path(wl)
    args = [to_dev(x[n]) for n in ("q_obs", "k", "v")]
    dense.run_layer(*args, 0)
    dense.join()
    cache = B.PagedCache(page_size=64, n_kv_heads=2, n_pages=4, max_seqs=2, max_pages=2)
    cache.reserve(ints([64, 64]))
    path.run_layer(*args, 0)
    path.join()
    path.reset()
    for _ in range(3):
        cache.k.zero_()
        path.store_into(cache, ints([1, 0]))
        torch.cuda.synchronize()
        with torch.cuda.stream(path.side2):
            torch.cuda._sleep(200_000_000)
        path.run_layer(*args, 0)
        path.store_into(None)
        held = spoil(8, 3000)
        path.join()
        torch.cuda.synchronize()
        cache.check()
        del held
        for b, slot in ((0, 1), (1, 0)):
            got = cache.k[0, int(cache.table[slot, 0])]
            assert torch.equal(got.view(torch.int16), dense.k_out[:, 64 * b:64 * b + 64].view(torch.int16))
        path.reset()
    path.close(), dense.close()
