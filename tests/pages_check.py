"""Shared by the tests of the paged cache: caches with everything unheld set to NaN, and the comparison with the oracle."""
import numpy as np
import torch

from oracle import asl_oracle as O
from oracle import pages_oracle as P
from paper_2601_07667_b200 import binding as B

D = 128
NAN_BITS = 0x7fc0


def ints(x):
    return torch.tensor(list(map(int, x)), dtype=torch.int32, device="cuda")


def bits(t):
    """The raw elements of a bf16 or one-byte tensor."""
    t = t.contiguous()
    return t.cpu().numpy() if t.element_size() == 1 else t.view(torch.int16).cpu().numpy().view(np.uint16)


def codes_to_float(codes):
    return torch.from_numpy(np.ascontiguousarray(codes)).view(torch.float8_e4m3fn).double().numpy()


class Both:
    """A cache on the device and the oracle's, moved by the same calls.  Rows that nothing has written are NaN (bf16) or the
    largest code (E4M3)."""

    def __init__(self, *, kv_heads, page, n_pages, max_seqs, max_pages, layers=1, fp8=False, seed=0):
        shape = (layers, n_pages, kv_heads, page, D)
        self.rng = np.random.default_rng(seed)
        self.scale = self.rng.uniform(0.01, 0.02, (layers, kv_heads)).astype(np.float32) if fp8 else None
        self.cache = B.PagedCache(page_size=page, n_layers=layers, n_kv_heads=kv_heads, n_pages=n_pages, max_seqs=max_seqs, max_pages=max_pages,
                                  k_dtype=B.ASL_K_FP8_E4M3 if fp8 else B.ASL_K_BF16, k_scale=self.scale)
        self.fp8, self.layers, self.kv_heads, self.page = fp8, layers, kv_heads, page
        k = np.full(shape, 0x7e if fp8 else NAN_BITS, dtype=np.uint8 if fp8 else np.uint16)
        v = np.full(shape, NAN_BITS, dtype=np.uint16)
        self.cache.k.copy_(self.dev(k)), self.cache.v.copy_(self.dev(v))
        self.oracle = P.Pages(k, v, max_seqs, max_pages)

    def dev(self, x):
        x = np.ascontiguousarray(x)
        return torch.from_numpy(x).cuda() if x.dtype == np.uint8 else torch.from_numpy(x.view(np.int16)).cuda().view(torch.bfloat16)

    def new_rows(self, *shape):
        """Random K (bits or codes) and V bits."""
        to = lambda x: torch.from_numpy(x).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)   # noqa: E731
        v = to(self.rng.standard_normal(shape))
        if self.fp8:
            k = torch.from_numpy(self.rng.standard_normal(shape) * 60).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
        else:
            k = to(self.rng.standard_normal(shape))
        return k, v

    def reserve(self, want):
        self.oracle.reserve(want)
        self.cache.reserve(ints(want))

    def fork(self, parent):
        self.oracle.fork(parent)
        self.cache.fork(ints(parent))

    def trim(self, to):
        self.oracle.trim(to)
        self.cache.trim(ints(to))

    def fill(self, want):
        """Slots grow to `want` tokens, the new rows random (written straight into the pools on both sides)."""
        old = self.oracle.len.copy()
        self.reserve(want)
        for s in range(len(want)):
            for pos in range(int(old[s]), int(self.oracle.len[s])):
                k, v = self.new_rows(self.layers, self.kv_heads, D)
                p = self.oracle.table[s, pos // self.page]
                self.oracle.k[:, p, :, pos % self.page] = k
                self.oracle.v[:, p, :, pos % self.page] = v
        self.cache.k.copy_(self.dev(self.oracle.k)), self.cache.v.copy_(self.dev(self.oracle.v))

    def same_books(self):
        o, c = self.oracle, self.cache
        assert c.len.tolist() == o.len.tolist()
        assert c.refs.tolist() == o.refs.tolist()
        table = c.table.cpu().numpy()
        for s in range(len(o.len)):
            assert table[s, :len(o.pages(s))].tolist() == o.pages(s), s

    def same_rows(self):
        """Every row of the pools, held or not."""
        assert (bits(self.cache.k) == self.oracle.k).all()
        assert (bits(self.cache.v) == self.oracle.v).all()

    def key_values(self, codes, layer, h):
        if self.fp8:
            return codes_to_float(codes) * float(self.scale[layer, h])
        return O.widen_bf16(codes).astype(np.float64)

    def expect(self, layer, slots, cu, q, n_q_heads):
        """(out, lse, tolerance of out, of lse) of every token; nobody's tokens NaN."""
        G = n_q_heads // self.kv_heads
        out = np.full(q.shape, np.nan)
        lse = np.full(q.shape[:2], np.nan)
        tol, tol_lse = np.zeros(q.shape), np.zeros(q.shape[:2])
        for i, s in enumerate(slots):
            if not 0 <= s < len(self.oracle.len):
                continue
            a, b = cu[i], cu[i + 1]
            for h in range(self.kv_heads):
                k = self.key_values(self.oracle.rows(self.oracle.k, layer, s, h), layer, h)
                v = O.widen_bf16(self.oracle.rows(self.oracle.v, layer, s, h)).astype(np.float64)
                g = slice(h * G, (h + 1) * G)
                o, z, weight, most = P.attend(q[a:b, g], k, v)
                out[a:b, g], lse[a:b, g] = o, z
                # a logit is a sum of 128 products kept in fp32 (each step half of 2^-23), then one product with the scale;
                # weights are rounded to bf16 (2^-8 each), sums run in fp32 over n terms, 2^x is good to 2^-22, and the
                # result is rounded to bf16 (2^-8)
                x = most * 130 * 2.0 ** -24
                n = max(1, k.shape[0]) * 2.0 ** -24
                tol[a:b, g] = 2.0 ** -8 * np.abs(o) + weight * (2.0 ** -8 + 2 * x[..., None] + n + 2.0 ** -20) * 1.01
                tol_lse[a:b, g] = x + n + 2.0 ** -21 * (2 + np.abs(np.where(np.isfinite(z), z, 0)))
        return out, lse, tol, tol_lse


def queries(rng, n_tokens, n_q_heads):
    bits_ = torch.from_numpy(rng.standard_normal((n_tokens, n_q_heads, D)) * 1.5).to(torch.bfloat16)
    return bits_.cuda(), bits_.double().numpy()


def check_attention(both, layer, slots, cu, n_q_heads, *, share, n_tokens=None, q=None, want_lse=True, marks=True):
    """Runs plan and attend, compares with the oracle; tokens that belong to nobody keep what their rows held."""
    n_tokens = n_tokens if n_tokens is not None else cu[-1]
    dev, exact = q if q is not None else queries(both.rng, n_tokens, n_q_heads)
    batch = both.cache.batch(ints(slots), ints(cu), n_tokens=n_tokens, n_q_heads=n_q_heads)
    out = torch.full((n_tokens, n_q_heads, D), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((n_tokens, n_q_heads), 7.0, device="cuda") if want_lse else None
    both.cache.plan(batch, share=share)
    both.cache.attend(layer, batch, dev, out, lse)
    both.cache.check()
    o, z, tol, tol_lse = both.expect(layer, slots, cu, exact, n_q_heads)
    got = out.double().cpu().numpy()
    nobody = np.isnan(z)
    assert (got[nobody] == 7.0).all()
    ok = ~nobody
    assert np.isfinite(got[ok]).all()
    worst = (np.abs(got[ok] - o[ok]) / np.maximum(tol[ok], 1e-300)).max() if ok.any() else 0.0
    assert worst <= 1.0, worst
    if want_lse:
        l = lse.double().cpu().numpy()
        assert (l[nobody] == 7.0).all()
        empty = ok & np.isneginf(z)
        assert np.isneginf(l[empty]).all() and (got[empty] == 0).all()
        rest = ok & ~empty
        assert (np.abs(l[rest] - z[rest]) <= tol_lse[rest]).all()
    return batch, out, lse
