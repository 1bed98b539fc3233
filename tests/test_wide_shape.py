"""Where the parts of shared prefixes lie: the arithmetic of csrc/attend.cuh on the CPU, over all sizes (wide_shape.cpp)."""
import os
import subprocess

from paper_2601_07667_b200 import build

from test_layer_order import CUDA_INCLUDE


def test_costs_of_any_group_fit_32_bits(tmp_path):
    here, exe = os.path.dirname(os.path.abspath(__file__)), str(tmp_path / "wide_shape")
    subprocess.run(["g++", "-O1", "-std=c++17", "-fsanitize=signed-integer-overflow", "-fno-sanitize-recover=all", "-I", CUDA_INCLUDE, "-I", build.INCLUDE,
                    "-I", build.CSRC, os.path.join(here, "wide_shape.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
