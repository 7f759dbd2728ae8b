"""The search for a row's group, which the residual norm's kernels use: the header, on the host, over up to 2^30 groups (the most that a call may have), against the definition.  The
offsets are computed as they are asked for, and an index outside [0, groups] is an error."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_17374_b200", "csrc")

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include <initializer_list>
#include "group_search.h"

// Offsets first + step * (g / repeat): groups of `step` rows, each followed by repeat - 1 empty ones.
struct Offsets {
  long long first, step, repeat;
  int groups;
  long long operator[](int g) const {
    if (g < 0 || g > groups) { printf("offset %d of %d groups\n", g, groups); exit(1); }
    return first + step * (g / repeat);
  }
};

int main() {
  long long asked = 0;
  const int most = 1 << 30;
  for (int groups : {1, 2, 3, 7, 8, 1000, (1 << 20) + 1, most - 1, most})
    for (long long first : {0ll, 5ll, 1000ll})
      for (long long step : {1ll, 2ll, 100ll})
        for (long long repeat : {1ll, 2ll, 3ll}) {
          const Offsets o = {first, step, repeat, groups};
          const long long last = o[groups];
          for (long long near : {0ll, first, last / 3, last / 2, last - step, last, last + 10})
            for (long long r = near - 3; r <= near + 3; ++r) {
              if (r < 0) continue;
              // g / repeat <= (r - first) / step
              long long want = 0;
              if (r >= first) { want = ((r - first) / step + 1) * repeat - 1; if (want > groups) want = groups; }
              const int got = last_offset_not_above(o, groups, r);
              if (got != want) { printf("%d groups from %lld by %lld, %lld alike, row %lld: %d, not %lld\n", groups, first, step, repeat, r, got, want); return 1; }
              ++asked;
            }
        }
  // offsets that are no offsets: somewhere inside, and an end
  unsigned long long x = 1;
  for (int i = 0; i < 100000; ++i) {
    long long o[9];
    for (long long& v : o) { x = x * 6364136223846793005ull + 1442695040888963407ull; v = (long long)(x >> 40) % 2000 - 1000; }
    const int got = last_offset_not_above(o, 8, (long long)(x >> 50) % 100);
    if (got < 0 || got > 8) { printf("%d of 8\n", got); return 1; }
  }
  printf("%lld\n", asked);
  return 0;
}
"""


def test_every_number_of_groups(tmp_path):
    src, exe = tmp_path / "groups.cc", tmp_path / "groups"
    src.write_text(PROGRAM)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-I", CSRC, "-o", str(exe), str(src)])
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
    assert int(r.stdout) > 3_000
