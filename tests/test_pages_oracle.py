"""The paged cache on the CPU: pins of its oracle (attention against a library's softmax, the books against their invariants)
and the refusals of the entry points, which look at their arguments before any device."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import pages_oracle as P
from paper_2601_07667_b200 import binding as B


def test_attention_is_softmax_of_what_is_seen():
    rng = np.random.default_rng(0)
    q, k, v = rng.standard_normal((3, 4, 16)), rng.standard_normal((9, 16)), rng.standard_normal((9, 16))
    out, lse, weight, _ = P.attend(q, k, v)
    for t in range(3):
        see = 9 - 3 + t + 1
        x = torch.from_numpy(q[t] @ k[:see].T / 4.0)
        w = torch.softmax(x, dim=1).numpy()
        assert np.allclose(out[t], w @ v[:see], atol=1e-13) and np.allclose(lse[t], torch.logsumexp(x, 1).numpy(), atol=1e-13)
        assert np.allclose(weight[t], w @ np.abs(v[:see]), atol=1e-13)
    out, lse, _, _ = P.attend(q, k[:1], v[:1])             # two tokens stand before the sequence's beginning
    assert (out[:2] == 0).all() and np.isneginf(lse[:2]).all() and np.allclose(out[2], v[0])


@pytest.mark.parametrize("seed", range(4))
def test_books_of_a_random_history(seed):
    """Counts are what the slots hold, no page that two slots hold is written, a slot's rows never change under it."""
    rng = np.random.default_rng(seed)
    page, n = 4, 7
    k = np.zeros((1, 40, 1, page, 1), dtype=np.int64)
    o = P.Pages(k, k.copy(), n, 10)
    truth = [[] for _ in range(n)]
    mark = 0
    for _ in range(60):
        what = rng.integers(0, 3)
        if what == 0:
            want = [int(x) + int(rng.integers(-1, 9)) for x in o.len]
            want = [min(w, 40) for w in want]
            try:
                o.reserve(want)
            except P.OutOfPages:
                continue
            for s in range(n):
                while len(truth[s]) < o.len[s]:
                    mark += 1
                    assert o.refs[o.table[s, len(truth[s]) // page]] == 1
                    o.put(0, s, len(truth[s]), 0, mark, -mark)
                    truth[s].append(mark)
        elif what == 1:
            free, held = [s for s in range(n) if not o.len[s]], [s for s in range(n) if o.len[s]]
            if free and held:
                parent = [-1] * n
                p = int(rng.choice(held))
                parent[free[0]] = p
                o.fork(parent)
                truth[free[0]] = list(truth[p])
        else:
            to = [int(rng.integers(0, x + 1)) if x and rng.random() < 0.4 else -1 for x in o.len]
            o.trim(to)
            truth = [t if c < 0 else t[:c] for t, c in zip(truth, to)]
        count = np.zeros(40, dtype=np.int64)
        for s in range(n):
            for p in o.pages(s):
                count[p] += 1
            assert o.rows(o.k, 0, s, 0)[:, 0].tolist() == truth[s]
        assert (count == o.refs).all()


def pages(**changed):
    a = 0x1000                                             # an address that is never looked at
    p = B.AslPages(2, 4, 128, 64, 100, 8, 16, B.ASL_K_BF16, a, a, None, a, a, a, a, a, 1 << 20)
    for name, value in changed.items():
        setattr(p, name, value)
    return p


def test_scratch_covers_slots_and_pages():
    assert B.asl_pages_scratch(pages()) >= 4 * (100 + 5 * 8)
    assert C.sizeof(B.AslPages) == 8 * 4 + 9 * 8 and C.sizeof(B.AslBatch) == 24


@pytest.mark.parametrize("changed,status", [
    (dict(k=None), B.ASL_ERR_INVALID), (dict(table=None), B.ASL_ERR_INVALID), (dict(err=None), B.ASL_ERR_INVALID),
    (dict(v=0x1008), B.ASL_ERR_INVALID), (dict(page_size=48), B.ASL_ERR_INVALID), (dict(page_size=256), B.ASL_ERR_INVALID),
    (dict(n_layers=0), B.ASL_ERR_INVALID), (dict(max_seqs=0), B.ASL_ERR_INVALID), (dict(n_pages=0), B.ASL_ERR_INVALID),
    (dict(k_dtype=2), B.ASL_ERR_INVALID), (dict(k_dtype=B.ASL_K_FP8_E4M3), B.ASL_ERR_INVALID), (dict(head_dim=100), B.ASL_ERR_INVALID),
    (dict(head_dim=64), B.ASL_ERR_UNSUPPORTED), (dict(n_pages=(1 << 20) + 1), B.ASL_ERR_UNSUPPORTED),
    (dict(n_pages=1 << 20, n_kv_heads=32), B.ASL_ERR_UNSUPPORTED), (dict(max_seqs=65537), B.ASL_ERR_UNSUPPORTED),
    (dict(max_pages=1 << 25), B.ASL_ERR_UNSUPPORTED)])
def test_descriptions_that_are_refused(changed, status):
    with pytest.raises(B.AslError) as e:
        B.asl_pages_scratch(pages(**changed))
    assert e.value.status == status


def test_calls_that_are_refused():
    lib, p, size = B.library(), pages(), C.c_size_t()
    ctx = C.create_string_buffer(1 << 16)                  # a context that no call gets as far as using
    a, two = 0x1000, (C.c_int64 * 2)(512, 128)
    batch = B.AslBatch(3, 4, a, a)
    ws = lambda b, hq: lib.asl_attend_workspace(ctx, C.byref(p), C.byref(b), hq, C.byref(size))   # noqa: E731
    assert ws(B.AslBatch(0, 4, a, a), 8) == B.ASL_ERR_INVALID
    assert ws(B.AslBatch(3, -1, a, a), 8) == B.ASL_ERR_INVALID
    assert ws(B.AslBatch(3, 4, None, a), 8) == B.ASL_ERR_INVALID
    assert ws(batch, 6) == B.ASL_ERR_INVALID               # not a multiple of H_k
    assert ws(batch, 4 * 129) == B.ASL_ERR_UNSUPPORTED
    assert ws(B.AslBatch(4097, 4, a, a), 8) == B.ASL_ERR_UNSUPPORTED
    assert lib.asl_attend_workspace(None, C.byref(p), C.byref(batch), 8, C.byref(size)) == B.ASL_ERR_INVALID
    assert lib.asl_attend_workspace(ctx, C.byref(p), C.byref(batch), 8, None) == B.ASL_ERR_INVALID
    for call in (lib.asl_pages_reserve, lib.asl_pages_fork, lib.asl_pages_trim):
        assert call(None, C.byref(p), a, None) == B.ASL_ERR_INVALID
    assert lib.asl_pages_store(None, C.byref(p), 0, a, a, a, a, None) == B.ASL_ERR_INVALID
    assert lib.asl_pages_compact(None, C.byref(p), 0, a, a, a, 1, a, 1, 1, None) == B.ASL_ERR_INVALID
    assert lib.asl_pages_append(None, C.byref(p), 0, C.byref(batch), a, a, two, two, None) == B.ASL_ERR_INVALID
    assert lib.asl_attend(None, C.byref(p), 0, C.byref(batch), 8, 1, a, two, a, a, a, 1 << 30, None) == B.ASL_ERR_INVALID
    assert lib.asl_pages_status(None, C.byref(p), None, None) == B.ASL_ERR_INVALID
    assert "pages" in B.asl_strerror(B.ASL_ERR_PAGES)
