"""Host arrays into device memory: what an AdamW list is read from has arrived when its creation returns, whichever stream steps first.  The header that creation uses, against a
model of a device whose copies arrive only when their stream is waited for; and no copy in creation but by it."""
import os
import re
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_17374_b200", "csrc")

PROGRAM = r"""
#include <cstdio>
#include <cstring>
#include <vector>
#include "upload.h"

enum Error { NONE, COPY_FAILED, WAIT_FAILED };
struct Device {                                  // what is copied is staged; it arrives with the wait
  struct Staged { void* to; std::vector<char> bytes; };
  std::vector<Staged> staged;
  int copies = 0, waits = 0, fail_copy = -1, running = 0;
  bool fail_wait = false;
  Error copy(const UploadPart& p) {
    if (copies++ == fail_copy) return COPY_FAILED;
    const char* const from = static_cast<const char*>(p.from);
    staged.push_back({p.to, {from, from + p.bytes}});
    return NONE;
  }
  Error wait() {
    ++waits;
    for (const Staged& s : staged) memcpy(s.to, s.bytes.data(), s.bytes.size());
    staged.clear();
    return fail_wait ? WAIT_FAILED : NONE;
  }
};

int main() {
  for (int count = 0; count <= 37; ++count)
    for (int fail = -1; fail < count; ++fail)
      for (int wait_too = 0; wait_too < 2; ++wait_too) {
        std::vector<std::vector<char>> from(count), to(count);
        std::vector<UploadPart> parts(count);
        for (int i = 0; i < count; ++i) {
          from[i].resize(i * i + 1, (char)(i + 1));
          to[i].resize(i * i + 1);
          parts[i] = {to[i].data(), from[i].data(), from[i].size()};
        }
        Device d;
        d.fail_copy = fail;
        d.fail_wait = wait_too != 0;
        const Error e = upload(parts.data(), count, [&](const UploadPart& p) { return d.copy(p); }, [&] { return d.wait(); });
        const Error want = fail >= 0 ? COPY_FAILED : wait_too ? WAIT_FAILED : NONE;
        if (e != want || d.waits != 1 || !d.staged.empty()) { printf("%d parts, copy %d fails: error %d, %d waits, %zu not there\n", count, fail, e, d.waits, d.staged.size()); return 1; }
        if (fail < 0) for (int i = 0; i < count; ++i) if (to[i] != from[i]) { printf("part %d of %d is not there\n", i, count); return 1; }
      }
  return 0;
}
"""


def test_all_has_arrived(tmp_path):
    src, exe = tmp_path / "upload.cc", tmp_path / "upload"
    src.write_text(PROGRAM)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-I", CSRC, "-o", str(exe), str(src)])
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout


def test_creation_copies_by_it_alone():
    text = open(os.path.join(CSRC, "kernels_adamw.cu")).read()
    assert len(re.findall(r"\bcudaMemcpy\w*\(", text)) == 1
    call = text[text.index("e = upload("):]
    call = call[:call.index(";\n ", call.index("cudaStreamSynchronize"))]
    streams = re.findall(r"cudaStream(?!Synchronize)\w+", call)
    assert len(streams) == 2 and streams[0] == streams[1]              # the stream of the copies is the one that is waited for
