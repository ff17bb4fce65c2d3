"""The C interface where host memory runs out: a status, no exception.  A small program replaces the
allocator with one that fails on demand."""

import os
import subprocess

from paper_2010_14109_amd import ooc

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include <new>
#include "ooc.h"
static bool fail = false;
void* operator new(std::size_t n) {
  void* p = fail ? nullptr : std::malloc(n ? n : 1);
  if (!p) throw std::bad_alloc();
  return p;
}
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, std::size_t) noexcept { std::free(p); }
int main() {
  int64_t slices[2];
  uint64_t part;
  const int64_t odd[6] = {1, 1, 1, 3, 2, 8}, good[6] = {1, 1, 1, 2, 2, 8};
  fail = true;
  const int a = ooc_qknorm_slices(0, slices);
  const int b = ooc_attention_slices(OOC_OP_CROSS_ATTENTION_FWD, odd, 6, slices, &part);
  const int c = ooc_attention_slices(OOC_OP_ADD, good, 6, slices, &part);
  const int d = ooc_run_fn(0, nullptr, OOC_OP_ADD, nullptr, nullptr, nullptr, 3, nullptr, 0);
  fail = false;
  const int e = ooc_attention_slices(OOC_OP_CROSS_ATTENTION_FWD, odd, 6, slices, &part);
  std::printf("%d %d %d %d %d\n", a, b, c, d, e);
}
"""


def test_entries_without_a_context_when_memory_runs_out(tmp_path):
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(PROGRAM)
    here = os.path.dirname(ooc.LIB_PATH)
    subprocess.run(["g++", "-std=c++17", "-rdynamic", "-I" + os.path.join(ROOT, "include"), str(src),
                    "-o", str(exe), ooc.LIB_PATH, "-Wl,-rpath," + here, "-Wl,--allow-shlib-undefined",
                    "-Wl,--unresolved-symbols=ignore-in-shared-libs"], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stderr
    oom = ooc.E_HOST_OOM
    assert r.stdout.split() == [str(oom)] * 4 + [str(ooc.E_INVALID)]
