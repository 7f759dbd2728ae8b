"""A call whose launch (or what comes before it) fails goes no further: a kernel behind it would find in the workspace what stood there before, indexes among it.  The library against a runtime of
the test's own, whose n-th launch fails; no GPU is needed or used."""
import os
import subprocess

from paper_2607_17374_b200 import build

PROGRAM = r"""
#include <cstdio>
#include <cstring>
#include <functional>
#include <cuda_runtime_api.h>
#include "taurus.h"

static int launches = 0, failing = -1;           // number of the launch that fails
static bool attributes_fail = false;
extern "C" {
cudaError_t cudaGetDevice(int* d) { *d = 0; return cudaSuccess; }
cudaError_t cudaDeviceGetAttribute(int* v, enum cudaDeviceAttr, int) { *v = 148; return cudaSuccess; }
cudaError_t cudaPointerGetAttributes(struct cudaPointerAttributes* a, const void* p) {
  memset(a, 0, sizeof *a);
  a->type = cudaMemoryTypeDevice;
  a->devicePointer = const_cast<void*>(p);
  return cudaSuccess;
}
cudaError_t cudaFuncSetAttribute(const void*, enum cudaFuncAttribute, int) { return attributes_fail ? cudaErrorInvalidValue : cudaSuccess; }
cudaError_t cudaOccupancyMaxActiveBlocksPerMultiprocessorWithFlags(int* n, const void*, int, size_t, unsigned) { *n = 2; return cudaSuccess; }
static cudaError_t last = cudaSuccess;
static cudaError_t launch() { return launches++ == failing ? last = cudaErrorMemoryAllocation : cudaSuccess; }
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t*, const void*, void**) { return launch(); }
cudaError_t cudaLaunchKernel(const void*, dim3, dim3, void**, size_t, cudaStream_t) { return launch(); }
cudaError_t cudaMemsetAsync(void*, int, size_t, cudaStream_t) { return cudaSuccess; }
cudaError_t cudaGetLastError(void) { const cudaError_t e = last; last = cudaSuccess; return e; }
}

int main() {
  char* const p = reinterpret_cast<char*>(1ull << 40);                 // addresses that nothing reads
  const auto at = [&](int i) { return static_cast<void*>(p + ((long long)i << 32)); };
  const auto f = [&](int i) { return static_cast<float*>(at(i)); };
  const auto l = [&](int i) { return static_cast<int64_t*>(at(i)); };
  const int64_t space = 1ll << 31;
  struct { const char* name; int launches, attributes; std::function<int()> call; } calls[] = {
      {"residual_norm", 1, 1, [&] { return taurus_residual_norm(100000, 256, at(0), 256, 0, at(1), 256, 0, 0, 1, f(2), 3, l(3), f(4), 1.f, f(5), f(6), 1e-5f, at(7), 256, at(8), 256, f(9), nullptr, nullptr); }},
      {"residual_norm_grad", 2, 1, [&] { return taurus_residual_norm_grad(100000, 256, at(0), 256, 0, at(1), 256, 0, 0, 1, f(2), 3, l(3), f(4), 1.f, f(5), f(9), at(10), 256, at(11), 256, at(12), 256, at(13), 256, f(14), f(15), f(16), f(17), at(18), space, nullptr, nullptr); }},
      {"class_logprob in tiles", 1, 1, [&] { return taurus_class_logprob(100000, 128, at(0), 128, 0, l(1), f(2), f(3), f(4), 16, f(5), l(6), nullptr, 0, nullptr, nullptr); }},
      {"class_logprob in parts", 2, 0, [&] { return taurus_class_logprob(3, 100000, at(0), 100000, 0, l(1), f(2), f(3), f(4), 5, f(5), l(6), at(7), space, nullptr, nullptr); }},
      {"class_logprob_train in parts", 3, 0, [&] { return taurus_class_logprob_train(3, 100000, at(0), 100000, 0, l(1), f(2), f(3), f(4), f(5), f(6), at(8), 100000, at(7), space, nullptr, nullptr); }},
      {"norm_rows", 0, 0, [&] { return taurus_norm_rows(100000, 3, l(0), at(1), 64, 0, 64, 8, f(2), f(3), 1e-5f, 0, at(4), 64, f(5), f(7), at(6), space, nullptr, nullptr); }},
      {"norm_rows_grad", 0, 0, [&] { return taurus_norm_rows_grad(100000, 3, l(0), at(1), 64, 0, 64, 8, f(2), f(3), 0, f(5), f(7), at(8), 64, at(9), 64, f(10), f(11), at(6), space, nullptr, nullptr); }},
      {"embed_grad, few ids", 0, 0, [&] { return taurus_embed_grad(1000, l(0), at(1), 0, 64, 64, 1.f, at(2), 0, 5000, 64, at(3), space, nullptr, nullptr); }},
      {"embed_grad", 0, 0, [&] { return taurus_embed_grad(3000000, l(0), at(1), 0, 64, 64, 1.f, at(2), 0, 10000000, 64, at(3), space, nullptr, nullptr); }},
  };
  for (auto& c : calls) {
    attributes_fail = false;
    failing = -1;
    launches = 0;
    int rc = c.call();
    if (rc != TAURUS_OK || launches == 0 || (c.launches && launches != c.launches)) { printf("%s: %d, %d launches\n", c.name, rc, launches); return 1; }
    const int all = launches;
    for (failing = 0; failing < all; ++failing) {
      launches = 0;
      rc = c.call();
      if (rc != TAURUS_ERR_CUDA || launches != failing + 1) { printf("%s: launch %d of %d fails: %d, %d launches\n", c.name, failing + 1, all, rc, launches); return 1; }
    }
    if (!c.attributes) continue;
    failing = -1;
    attributes_fail = true;
    launches = 0;
    rc = c.call();
    if (rc != TAURUS_ERR_CUDA || launches != 0) { printf("%s: shared memory is refused: %d, %d launches\n", c.name, rc, launches); return 1; }
  }
  return 0;
}
"""


def test_nothing_is_launched_behind_a_launch_that_failed(tmp_path):
    src, exe = tmp_path / "launch.cc", tmp_path / "launch"
    src.write_text(PROGRAM)
    lib = build.build()
    cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-rdynamic", "-I", os.path.join(cuda, "include"), "-I", build.INCLUDE, "-o", str(exe), str(src), lib, "-Wl,-rpath," + os.path.dirname(lib),
                           "-Wl,--unresolved-symbols=ignore-in-shared-libs", "-L", os.path.join(cuda, "lib64"), "-Wl,-rpath," + os.path.join(cuda, "lib64")])
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
