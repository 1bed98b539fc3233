"""Attention over long shared prefixes: pages compared by a kernel of their own, groups of several chunks whose keys are cut into
stripes of several tiles, prefixes that part far behind their beginning."""
import numpy as np
import pytest
import torch

from pages_check import Both, check_attention, ints, queries
from test_gpu_attend import forked

pytestmark = pytest.mark.gpu

SMS = 148


def stretches(heads, n, pfx):
    """(tiles of a stripe, tiles) of one group of n tokens, as the plan deals them out."""
    G = heads[0] // heads[1]
    tiles, whole, rest = -(-pfx // 128), n // (256 // G), n % (256 // G) * G
    cost = tiles * (2 * whole + (0 if rest == 0 else 2 if rest > 128 else 1)) * heads[1]
    each = max(2, -(-cost // SMS))
    return (each + 1) // 2, tiles


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("heads,n,prompt,page", [((64, 8), 40, 8205, 16), ((16, 1), 72, 9000, 16), ((32, 2), 100, 9100, 32), ((64, 8), 33, 8205, 16),
                                                  ((12, 1), 150, 7777, 16)])
def test_stripes_of_several_tiles(heads, n, prompt, page, fp8):
    """More than 256 rows on a long prompt: stripes of two tiles and more, the last one shorter, chunks of a stripe over two blocks."""
    stripe, tiles = stretches(heads, n, prompt // page * page)
    assert stripe >= 2 and tiles % stripe and n * heads[0] // heads[1] > 256
    both, slots = forked(heads, page, [prompt], [[1 + i % 7 for i in range(n)]], fp8=fp8, seed=n)
    assert n * both.cache.table.shape[1] > 16384                    # (compared by the kernel of its own)
    q = queries(both.rng, n, heads[0])
    for share in (1, 2):
        check_attention(both, 0, slots, list(range(n + 1)), heads[0], share=share, q=q)


def test_several_tokens_on_stripes():
    """Drafts of three tokens, two prompts, a chunk that ends inside a sequence's tokens; queries that lie head by head."""
    both, slots = forked((28, 4), 16, [6001, 9009], [[5, 9, 30, 4, 7] * 6, [3, 17, 100, 64, 3] * 5], seed=5)
    n = len(slots)
    bits = torch.from_numpy(both.rng.standard_normal((28, 3 * n, 128))).to(torch.bfloat16).cuda()
    q = bits.transpose(0, 1)
    for share in (1, 2):
        check_attention(both, 0, slots, list(range(0, 3 * n + 1, 3)), 28, share=share, q=(q, q.double().cpu().numpy()))


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("part", [2047, 2048, 2049, 2125, 2249])
def test_prefixes_that_part_behind_2048_pages(part, wide):
    """Neighbours that hold the same pages up to one of the 2048th or after, compared by the plan or, where the table is wide, by the kernel
    of its own (2048 pages at a time)."""
    page, n = 16, 36003
    both = Both(kv_heads=1, page=page, n_pages=2251 + 3 * 210 + 20, max_seqs=6, max_pages=4500 if wide else 2300, seed=part)
    both.fill([n, 0, 0, 0, 0, 0])
    both.fork([-1, 0, 0, 0, 0, -1])
    both.trim([-1, -1, -1, part * page, part * page, -1])
    both.fill([-1, n + 1, n + 20, n + 3, n + 4, 70])
    same = lambda a, b: int(np.argmax(both.oracle.table[a, :2250] != both.oracle.table[b, :2250])) or 2250     # noqa: E731
    assert same(1, 2) == 2250 and same(2, 3) == part and same(3, 4) == part
    q = queries(both.rng, 5, 8)
    for share in (1, 2):
        check_attention(both, 0, [1, 2, 3, 4, 5], list(range(6)), 8, share=share, q=q)
    check_attention(both, 0, [3, 1, 4, 2], list(range(5)), 8, share=2)
