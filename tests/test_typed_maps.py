"""Tensor maps of the products by vertex type, on the host: rows whose pitch no map can hold go the other way, and where a map cannot be made the call says so
and has enqueued nothing."""
import os
import re
import subprocess

import pytest
import torch

from paper_2607_17374_b200 import build

PROGRAM = r"""
#include <cstdio>
#include <cstring>
#include "typed.cuh"

int main(int argc, char**) {
  // addresses that nothing reads
  char* const p = reinterpret_cast<char*>(1ull << 32);
  const long long most = (1ll << 39) - 8;                  // pitches below 2^40 bytes, a multiple of 16
  if (!tma_rows(p, 64) || !tma_rows(p, most) || tma_rows(p, most + 8) || tma_rows(p, 1ll << 55) || tma_rows(p, 63) || tma_rows(p + 8, 64)) { printf("rows for TMA\n"); return 1; }
  if (argc > 1) return 0;
  // without a driver there are no maps
  const TypedSpaces spaces = {p, p, p, p};
  const long long* const off = reinterpret_cast<const long long*>(p);
  for (int32_t type : {TAURUS_F32, TAURUS_BF16, TAURUS_F16})
    for (int width : {64, 47}) {
      int rc = typed_tc_project(1000, 2, off, p, width, type, p, nullptr, width, width, p, type, width, spaces, nullptr, 148, nullptr);
      if (rc != TAURUS_ERR_CUDA || !strstr(taurus_last_cuda_error(), "cuTensorMapEncodeTiled")) { printf("project %d %d: %d '%s'\n", type, width, rc, taurus_last_cuda_error()); return 1; }
      rc = typed_tc_project_grad(1000, 2, off, p, width, type, p, p, width, width, width, p, width, p, type, reinterpret_cast<float*>(p), spaces, nullptr, 148, nullptr);
      if (rc != TAURUS_ERR_CUDA || !strstr(taurus_last_cuda_error(), "cuTensorMapEncodeTiled")) { printf("gradient %d %d: %d '%s'\n", type, width, rc, taurus_last_cuda_error()); return 1; }
    }
  return 0;
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    d = tmp_path_factory.mktemp("maps")
    src, exe = d / "maps.cu", d / "maps"
    src.write_text(PROGRAM)
    lib = build.build()
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    subprocess.check_call([nvcc, "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I", build.CSRC, "-I", build.INCLUDE, "-o", str(exe), str(src), lib,
                           "-Xlinker", "-rpath", "-Xlinker", os.path.dirname(lib), "-lcudart", "-lcuda"])
    return str(exe)


def test_pitches_that_no_map_holds(program):
    r = subprocess.run([program, "pitches"], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr


@pytest.mark.skipif(torch.cuda.is_available(), reason="needs a machine without a GPU")
def test_a_map_that_cannot_be_made_is_an_error_with_its_text(program):
    r = subprocess.run([program], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr


def test_everything_is_ready_before_the_first_launch():
    text = open(os.path.join(build.CSRC, "kernels_typed_tc.cu")).read()
    bodies = [b for b in re.split(r"\n(?=int typed_tc_)", text) if b.startswith(("int typed_tc_project(", "int typed_tc_project_grad("))]
    assert len(bodies) == 2
    for body in bodies:
        assert max(body.rindex(w) for w in ("ready_rows(", "return TAURUS_ERR_CUDA;")) < min(body.index(w) for w in ("pack_weights(", ".lay_out(", "launch_type<"))
