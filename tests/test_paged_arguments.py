"""Arguments that the paged cache's Python calls refuse, checked on the CPU: the checks look at types, shapes and devices before
anything is called.  (A cache without a device: only what the checks look at.)"""
import pytest
import torch

from paper_2601_07667_b200 import binding as B


def bare(codes=False):
    c = object.__new__(B.PagedCache)
    c.torch, c.dev, c.ctx, c._ref = torch, torch.device("cpu"), 0, None
    k = torch.zeros((1, 4, 2, 16, 128), dtype=torch.uint8 if codes else torch.bfloat16)
    c._look_at(k, torch.zeros((3, 4), dtype=torch.int32))
    c.pages = B.AslPages(1, 2, 128, 16, 4, 3, 4, int(codes), None, None, None, None, None, None, None, None, 0)
    return c


def a_batch(n_tokens=2, n_q_heads=4):
    b = object.__new__(B.Batch)
    b.n_tokens, b.n_q_heads, b.share, b.ws, b.ws_bytes, b.ref, b.device = n_tokens, n_q_heads, 1, 0, 0, None, -1
    b.streams = set()
    return b


def refused(call):
    with pytest.raises(B.AslError) as e:
        call()
    assert e.value.status == B.ASL_ERR_INVALID and "asl_" not in str(e.value)         # (by the checks, not by the library)


@pytest.mark.parametrize("dtype", [torch.float16, torch.int16, torch.uint16, torch.float32, torch.uint8])
def test_rows_that_are_not_bf16(dtype):
    """Elements of two bytes are not all bf16: float16 rows would be read as other numbers."""
    c, b = bare(), a_batch()
    q, rows, out = torch.zeros((2, 4, 128), dtype=torch.bfloat16), torch.zeros((2, 2, 128), dtype=torch.bfloat16), torch.zeros((2, 4, 128), dtype=torch.bfloat16)
    refused(lambda: c.attend(0, b, q.to(dtype)))
    refused(lambda: c.attend(0, b, q, out.to(dtype)))
    refused(lambda: c.append(0, b, rows.to(dtype), rows))
    refused(lambda: c.append(0, b, rows, rows.to(dtype)))
    refused(lambda: bare(codes=True).append(0, b, rows.to(torch.uint8), rows.to(dtype)))


@pytest.mark.parametrize("dtype", [torch.int32, torch.float64, torch.bfloat16])
def test_a_log_sum_that_is_not_fp32(dtype):
    c, b, q = bare(), a_batch(), torch.zeros((2, 4, 128), dtype=torch.bfloat16)
    refused(lambda: c.attend(0, b, q, q.clone(), torch.zeros((2, 4), dtype=dtype)))


OTHER_BYTES = [torch.float8_e5m2, torch.float8_e4m3fnuz, torch.float8_e5m2fnuz, torch.float8_e8m0fnu, torch.bool]


@pytest.mark.parametrize("dtype", OTHER_BYTES)
def test_bytes_that_are_no_e4m3_codes(dtype):
    """Codes come as E4M3 or as their bits; other one-byte types would be read as other numbers."""
    v = torch.zeros((2, 2, 128), dtype=torch.bfloat16)
    refused(lambda: bare(codes=True).append(0, a_batch(), torch.zeros((2, 2, 128), dtype=torch.uint8).view(dtype), v))
    k = torch.zeros((1, 4, 2, 16, 128), dtype=torch.uint8).view(dtype)
    refused(lambda: B.PagedCache(page_size=16, k=k, v=torch.zeros(k.shape, dtype=torch.bfloat16), table=torch.zeros((3, 4), dtype=torch.int32),
                                 length=torch.zeros(3, dtype=torch.int32), refs=torch.zeros(4, dtype=torch.int32), k_scale=torch.ones((1, 2))))


@pytest.mark.parametrize("dtype", [torch.uint8, torch.int8, torch.float8_e4m3fn])
def test_codes_of_any_view(dtype):
    k = torch.zeros((2, 2, 128), dtype=torch.uint8).view(dtype)
    assert list(bare(codes=True)._rows(k, "k_new", 2, 2, True)) == [256, 128]


def a_path():
    p = object.__new__(B.LayerPath)
    p.torch, p.dev, p.batch, p.ctx, p._pages, p.H_k, p.sum_kept = torch, torch.device("cpu"), 2, 0, None, 2, 5
    return p


@pytest.mark.parametrize("slots", [None, torch.tensor([1, 0]), torch.tensor([1.0, 0.0]), torch.tensor([1], dtype=torch.int32), torch.tensor([1, 0, 2], dtype=torch.int32),
                                   torch.tensor([1, 5, 0, 5], dtype=torch.int32)[::2]])
def test_slots_to_store_into(slots):
    """One dense int32 a request on the cache's device: int64 would be read as other slots, a host address not at all."""
    c, p = bare(), a_path()
    refused(lambda: p.store_into(c, slots))
    assert p._pages is None
    good = torch.tensor([1, 0], dtype=torch.int32)
    p.store_into(c, good)
    assert p._pages[0] is c and p._pages[1] is good
    p.store_into(None)
    assert p._pages is None
    c._device = 0                                       # a cache on a device: host memory is not there
    refused(lambda: p.store_into(c, good))
    c, p.dev = bare(), torch.device("cuda", 1)
    refused(lambda: p.store_into(c, good))


def test_a_prefills_rows_to_store():
    """K and V of the cache's types, on its device (how they lie there the path's strides say)."""
    c, p = bare(), a_path()
    kv, idx, slots = torch.zeros((7, 2, 128), dtype=torch.bfloat16), torch.zeros((2, 5), dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    for k, v in ((kv.half(), kv), (kv, kv.half()), (kv.view(torch.uint8), kv), (kv, kv.float())):
        refused(lambda: c.store(0, p, k, v, idx, slots))
    c = bare(codes=True)
    codes = torch.zeros((7, 2, 128), dtype=torch.uint8)
    for k, v in ((kv, kv), (codes.view(torch.float8_e5m2), kv), (codes, codes)):
        refused(lambda: c.store(0, p, k, v, idx, slots))
    c._device = 0
    refused(lambda: c.store(0, p, codes, kv, idx, slots))


def test_a_batch_of_another_device():
    """Its slots and workspace lie where the cache's kernels do not look."""
    c, b = bare(), a_batch()
    q, rows = torch.zeros((2, 4, 128), dtype=torch.bfloat16), torch.zeros((2, 2, 128), dtype=torch.bfloat16)
    b.device = 1
    for call in (lambda: c.append(0, b, rows, rows), lambda: c.plan(b), lambda: c.attend(0, b, q)):
        refused(call)
