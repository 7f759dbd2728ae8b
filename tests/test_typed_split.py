"""The three bf16 values that the products by vertex type make of an fp32 one, on the host: the code that the kernels use, over every mantissa and at the ends of the
range, against the bounds that its comments state."""
import os
import subprocess

import pytest

from paper_2607_17374_b200 import build

PROGRAM = r"""
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <vector>
#include "typed.cuh"

struct Three { float hi, mid, lo; };
// x beside another value, in any of the four places
static Three split(float x, float beside = 1.f, int place = 0) {
  float v[4] = {beside, beside, beside, beside};
  v[place] = x;
  const Split4 s = split4(v[0], v[1], v[2], v[3]);
  auto get = [&](uint2 p) { const unsigned w = place < 2 ? p.x : p.y; return float_of(place & 1 ? w & 0xFFFF0000u : w << 16); };
  return {get(s.hi), get(s.mid), get(s.lo)};
}
static double left_out(float x, float w) {      // of the product, by what is multiplied: all but mid lo, lo mid and lo lo
  const Three a = split(x), b = split(w);
  const double kept = (double)a.hi * b.hi + ((double)a.hi * b.mid + (double)a.mid * b.hi) + (double)a.mid * b.mid + ((double)a.hi * b.lo + (double)a.lo * b.hi);
  const double p = (double)x * w;
  return std::fabs(kept - p) / std::fabs(p) * 16777216.0;      // in 2^-24
}
#define CHECK(c, ...) do { if (!(c)) { printf(#c ": "); printf(__VA_ARGS__); printf("\n"); return 1; } } while (0)

int main() {
  double mid = 0, lo = 0;
  std::vector<float> worst;
  for (unsigned m = 0; m < 1u << 23; ++m)
    for (int e : {-110, 0, 126}) {
      const float x = float_of(m | (unsigned)(e + 127) << 23);
      const Three s = split(x);
      CHECK((double)s.hi + s.mid + s.lo == x, "%a", x);
      if (e) continue;
      mid = std::fmax(mid, std::fabs(s.mid / x)); lo = std::fmax(lo, std::fabs(s.lo / x));
      if (std::fabs(s.mid) * std::fabs(s.lo) > 0.98 * ldexp(1, -25)) worst.push_back(x);
    }
  CHECK(mid <= ldexp(1, -8) && lo <= ldexp(1, -17), "%g %g", mid, lo);
  CHECK(worst.size() > 10, "%zu", worst.size());
  double most = 0;
  for (float x : worst) for (float w : worst) most = std::fmax(most, left_out(x, w));
  unsigned long long r = 1;
  auto next = [&] { r = r * 6364136223846793005ull + 1442695040888963407ull; return (unsigned)(r >> 40); };
  for (int i = 0; i < 5000000; ++i) most = std::fmax(most, left_out(float_of(0x3F800000u | (next() & 0x7FFFFF)), float_of(0x3F800000u | (next() & 0x7FFFFF))));
  for (int i = 0; i < 5000000; ++i) most = std::fmax(most, left_out(float_of(0x3F800000u | (next() & 0xFFFF)), float_of(0x3F800000u | (next() & 0xFFFF))));
  most = std::fmax(most, left_out(float_of(0x3F80FF80u), float_of(0x3F80FF80u)));
  CHECK(most < 1.0, "%g 2^-24 of a product left out", most);
  // the ends of the range: small values are cut off at 2^-133, large ones stay finite, infinities and NaN are hi alone, whatever stands beside them
  for (int i = 0; i < 1000000; ++i) {
    const float x = float_of(((unsigned)(next() % 17) << 23) | (next() & 0x7FFFFF));
    const Three s = split(x);
    CHECK(std::fabs((double)s.hi + s.mid + s.lo - x) < ldexp(1, -133), "%a", x);
  }
  for (int place = 0; place < 4; ++place)
    for (float beside : {1.f, -3.4e38f, INFINITY, NAN, 0.f}) {
      for (unsigned m = 0x7F7F0000u; m < 0x7F800000u; m += 0x0101u)
        for (unsigned sign : {0u, 0x80000000u}) {
          const float x = float_of(m | sign);
          const Three s = split(x, beside, place);
          CHECK(std::isfinite(s.hi) && (double)s.hi + s.mid + s.lo == x, "%a", x);
        }
      for (float x : {INFINITY, -INFINITY}) { const Three s = split(x, beside, place); CHECK(s.hi == x && s.mid == 0 && s.lo == 0, "%g", x); }
      for (unsigned u : {0x7FC00000u, 0x7F800001u, 0x7FFFFFFFu, 0xFFFFFFFFu, 0xFF800001u}) {
        const Three s = split(float_of(u), beside, place);
        CHECK(std::isnan(s.hi) && s.mid == 0 && s.lo == 0, "%x", u);
      }
      const Three z = split(-0.f, beside, place);
      CHECK(z.hi == 0 && z.mid == 0 && z.lo == 0, "zero");
    }
  return 0;
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    d = tmp_path_factory.mktemp("split")
    src, exe = d / "split.cu", d / "split"
    src.write_text(PROGRAM)
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    subprocess.check_call([nvcc, "-std=c++17", "-O2", "-gencode", "arch=compute_100a,code=sm_100a", "-I", build.CSRC, "-I", build.INCLUDE, "-o", str(exe), str(src), build.build()])
    return str(exe)


def test_what_a_product_leaves_out(program):
    env = dict(os.environ, LD_LIBRARY_PATH=os.path.dirname(build.LIB) + ":" + os.environ.get("LD_LIBRARY_PATH", ""))
    r = subprocess.run([program], capture_output=True, text=True, timeout=300, env=env)
    assert r.returncode == 0, r.stdout + r.stderr
