"""What the paged cache's entry points launch, checked on the CPU: their built objects linked against a runtime that only logs
launches and refuses those that the real one would (fake_launches.cpp)."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2601_07667_b200 import binding as B
from paper_2601_07667_b200 import build

from test_layer_order import CUDA_INCLUDE

A = 0x1000                                              # an address that is never looked at
NAMES = [n for n in B.EXPORTS if n.startswith(("asl_pages_", "asl_attend"))] + ["asl_create", "asl_destroy"]


@pytest.fixture(scope="module")
def built(tmp_path_factory):
    build.build()
    objects = [os.path.join(build.OBJ_DIR, n) for n in ("pages.o", "attend.o")]
    if not all(os.path.exists(o) for o in objects):
        build.build(force=True)
    so = str(tmp_path_factory.mktemp("fake") / "libasl_launches.so")
    here = os.path.dirname(os.path.abspath(__file__))
    subprocess.run(["g++", "-shared", "-fPIC", "-O1", "-std=c++17", "-Wl,-Bsymbolic", "-I", CUDA_INCLUDE, "-I", build.INCLUDE, "-I", build.CSRC, "-I", here,
                    "-x", "c++", os.path.join(build.CSRC, "asl_api.cu"), os.path.join(here, "fake_launches.cpp"), "-x", "none", *objects, "-o", so],
                   check=True)
    return so


@pytest.fixture
def lib(built, tmp_path):
    """A copy of its own, so that no attribute of a kernel is left from another test."""
    so = str(tmp_path / "lib.so")
    with open(built, "rb") as f, open(so, "wb") as g:
        g.write(f.read())
    fake = C.CDLL(so)
    fake.fake_log.restype = C.c_char_p
    for name in NAMES:
        getattr(fake, name).argtypes = getattr(B.library(), name).argtypes
    fake.fake_fail(b"", 0)
    return fake


class Cache:
    def __init__(self, lib, **sizes):
        self.lib, self.ctx = lib, C.c_void_p()
        assert lib.asl_create(C.byref(self.ctx), 0) == B.ASL_OK
        s = dict(n_layers=2, n_kv_heads=2, page_size=16, n_pages=100, max_seqs=8, max_pages=16, k_dtype=B.ASL_K_BF16)
        s.update(sizes)
        self.pages = B.AslPages(s["n_layers"], s["n_kv_heads"], 128, s["page_size"], s["n_pages"], s["max_seqs"], s["max_pages"], s["k_dtype"],
                                A, A, A, A, A, A, A, A, 1 << 40)
        self.ref = C.byref(self.pages)
        lib.fake_clear()

    def batch(self, n_seqs, n_tokens, n_q_heads=4):
        self.b, size = B.AslBatch(n_seqs, n_tokens, A, A), C.c_size_t()
        assert self.lib.asl_attend_workspace(self.ctx, self.ref, C.byref(self.b), n_q_heads, C.byref(size)) == B.ASL_OK
        return C.byref(self.b), n_q_heads, size.value

    def plan(self, batch, share=1):
        b, heads, size = batch
        return self.lib.asl_attend_plan(self.ctx, self.ref, b, heads, share, A, size, None)

    def launches(self):
        """(kernel, grid, block, dynamic bytes) of every launch since the latest look."""
        got = [l.split() for l in self.lib.fake_log().decode().splitlines()]
        self.lib.fake_clear()
        return [(x[0], *map(int, x[1:])) if x[0] != "run" else tuple(x[1:2]) for x in got]

    def kernels(self):
        return [x[0] for x in self.launches()]


@pytest.mark.parametrize("n_pages", [1, 70001, 392063, 392064, 392065, 392500, 393216, 393217, 1 << 20])
def test_the_books_of_a_pool_of_any_size(lib, n_pages):
    """A bit a page lies in shared memory beside the kernel's own arrays: up to 48 KB together need no leave, more do."""
    c = Cache(lib, n_pages=n_pages, n_layers=64, max_seqs=64)
    assert lib.asl_pages_reserve(c.ctx, c.ref, A, None) == B.ASL_OK
    assert c.kernels() == ["pages_reserve_kernel", "pages_copy_kernel"]


def test_no_copies_behind_books_that_were_not_kept(lib):
    """The copying kernel reads a list that the books' kernel writes: where that one cannot be launched nothing follows it."""
    c = Cache(lib, n_layers=64, max_seqs=64)
    lib.fake_fail(b"pages_reserve_kernel", 1)
    assert lib.asl_pages_reserve(c.ctx, c.ref, A, None) == B.ASL_ERR_CUDA
    assert c.kernels() == []
    assert lib.asl_pages_reserve(c.ctx, c.ref, A, None) == B.ASL_OK
    assert c.kernels() == ["pages_reserve_kernel", "pages_copy_kernel"]


@pytest.mark.parametrize("n_seqs", [1, 1000, 1019, 1020, 1021, 1022, 1023, 1024, 1025, 4096])
def test_a_plan_of_any_batch(lib, n_seqs):
    """Twelve words a sequence in shared memory beside the kernel's own arrays."""
    c = Cache(lib, max_seqs=4096, max_pages=4)
    assert c.plan(c.batch(n_seqs, n_seqs)) == B.ASL_OK
    assert c.kernels() == ["attend_plan_kernel"]


def test_no_plan_from_pages_that_were_not_compared(lib):
    """Many pages are compared by a kernel of its own: where that one cannot be launched the plan does not read its counts."""
    c = Cache(lib, max_seqs=64, max_pages=1 << 14)
    batch = c.batch(64, 64)
    lib.fake_fail(b"attend_same_kernel", 1)
    assert c.plan(batch) == B.ASL_ERR_CUDA
    assert c.kernels() == []
    assert c.plan(batch) == B.ASL_OK
    assert c.kernels() == ["attend_same_kernel", "attend_plan_kernel"]


@pytest.mark.parametrize("sum_kept,max_kept,blocks", [(0, 100, 1), (1000, 1000, 16), (1000, 1, 1), (1000, 64, 1), (1000, 65, 2), (1000, 2 ** 31 - 1, 16), (2 ** 31 - 1, 2 ** 31 - 1, 1 << 23),
                                                      (1 << 40, 2 ** 31 - 1, 1 << 23)])
def test_lists_to_prune_by_of_any_announced_length(lib, sum_kept, max_kept, blocks):
    """No list is longer than all of them together, and the columns of blocks are counted without running over."""
    c = Cache(lib)
    assert lib.asl_pages_compact(c.ctx, c.ref, 0, A, A, A, 3, A, sum_kept, max_kept, None) == B.ASL_OK
    assert c.launches() == [("rows_to_pages_kernel", blocks, 2, 3, 256, 0)]


def test_a_step_without_tokens(lib):
    """Empty tensors have no address: nothing is read, nothing launched, and the other arguments are looked at as ever."""
    c, two = Cache(lib), (C.c_int64 * 2)(512, 128)
    batch, heads, size = c.batch(3, 0)
    assert lib.asl_pages_append(c.ctx, c.ref, 0, batch, None, None, two, two, None) == B.ASL_OK
    assert lib.asl_attend(c.ctx, c.ref, 0, batch, heads, 1, None, two, None, None, A, size, None) == B.ASL_OK
    assert lib.asl_pages_append(c.ctx, c.ref, 2, batch, None, None, two, two, None) == B.ASL_ERR_INVALID
    assert lib.asl_attend(c.ctx, c.ref, 2, batch, heads, 1, None, two, None, None, A, size, None) == B.ASL_ERR_INVALID
    assert lib.asl_attend(c.ctx, c.ref, 0, batch, heads, 1, None, two, None, None, A, size - 1, None) == B.ASL_ERR_WORKSPACE
    batch, heads, size = c.batch(3, 1)
    assert lib.asl_pages_append(c.ctx, c.ref, 0, batch, None, A, two, two, None) == B.ASL_ERR_INVALID
    assert lib.asl_attend(c.ctx, c.ref, 0, batch, heads, 1, None, two, A, None, A, size, None) == B.ASL_ERR_INVALID
    assert c.kernels() == []


def test_no_rows_to_prune_by(lib):
    """Nothing kept of any job: an empty list of positions has no address, and a list that is there all the same is noted by the kernel."""
    c = Cache(lib)
    assert lib.asl_pages_compact(c.ctx, c.ref, 0, A, A, A, 3, None, 0, 0, None) == B.ASL_OK
    assert c.kernels() == ["rows_to_pages_kernel"]
    assert lib.asl_pages_compact(c.ctx, c.ref, 0, A, A, A, 3, None, 1, 0, None) == B.ASL_ERR_INVALID
    assert lib.asl_pages_compact(c.ctx, c.ref, 0, A, A, A, 3, None, 0, -1, None) == B.ASL_ERR_INVALID
    assert lib.asl_pages_compact(c.ctx, c.ref, 0, A, A, None, 3, A, 0, 0, None) == B.ASL_ERR_INVALID
    assert lib.asl_pages_compact(c.ctx, c.ref, 0, A, A, A, 0, A, 0, 0, None) == B.ASL_ERR_INVALID
    assert c.kernels() == []
