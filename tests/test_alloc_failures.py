"""Memory that runs out while a layout is built: every allocation in turn fails, and the C entries answer with an error code; no
C++ exception leaves them.  A program of its own, whose operator new throws on demand.  No GPU (host layouts)."""
import os
import shutil
import subprocess

import pytest

from paper_2503_08640_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include <new>

#include "dbsa.h"

static long left = -1;  // allocations that still succeed; below 0: all do
static bool spent() {
  if (left < 0) return false;
  return left-- == 0;
}
void* operator new(std::size_t n) {
  if (spent()) { left = 0; throw std::bad_alloc(); }
  if (void* p = std::malloc(n)) return p;
  throw std::bad_alloc();
}
void* operator new(std::size_t n, const std::nothrow_t&) noexcept {
  if (spent()) { left = 0; return nullptr; }
  return std::malloc(n);
}
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, std::size_t) noexcept { std::free(p); }

// how many allocations failed before the call came through
template <typename F>
static void fail_each(const char* what, F&& build) {
  for (long n = 0;; ++n) {
    dbsa_layout* out = nullptr;
    left = n;
    const int rc = build(&out);
    left = -1;
    if (rc == DBSA_OK) {
      dbsa_layout_destroy(out);
      std::printf("%s %ld\n", what, n);
      return;
    }
    if (out) std::abort();
  }
}

int main() {
  const int32_t demos[] = {4, 104, 254, 300}, groups[] = {0, 1, 3}, cu[] = {0, 5, 305}, ptr[] = {0, 1, 3}, idx[] = {1, 0, 1};
  const int32_t own[] = {50, 400};
  dbsa_pool_desc pool{4, 3, demos, 2, groups, 0};
  dbsa_select_desc sel{2, cu, ptr, idx, 0, nullptr};
  fail_each("pool", [&](dbsa_layout** out) { return dbsa_layout_build(&pool, nullptr, 64, 64, DBSA_LAYOUT_HOST_ONLY, nullptr, out); });
  fail_each("query", [&](dbsa_layout** out) { return dbsa_layout_build(&pool, &sel, 64, 64, DBSA_LAYOUT_HOST_ONLY, nullptr, out); });
  fail_each("append", [&](dbsa_layout** out) { return dbsa_layout_build_append(&pool, 1, 64, 64, DBSA_LAYOUT_HOST_ONLY, nullptr, out); });
  fail_each("chunk", [&](dbsa_layout** out) { return dbsa_layout_build_chunk(&pool, &sel, 8, 2, own, DBSA_LAYOUT_HOST_ONLY, nullptr, out); });
  return 0;
}
"""


@pytest.mark.skipif(not (shutil.which("g++") and os.path.exists(build.LIB_PATH)), reason="needs the built library and g++")
def test_no_exception_leaves_a_build(tmp_path):
    (tmp_path / "program.cpp").write_text(PROGRAM)
    where = os.path.dirname(build.LIB_PATH)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "include"), str(tmp_path / "program.cpp"), "-o", str(tmp_path / "program"),
                    build.LIB_PATH, "-Wl,-rpath," + where, "-Wl,-rpath,/opt/rocm/lib", "-Wl,--allow-shlib-undefined"], check=True)
    done = subprocess.run([str(tmp_path / "program")], capture_output=True, text=True, timeout=60)
    assert done.returncode == 0, done.stderr
    failed = dict(line.split() for line in done.stdout.splitlines())
    assert set(failed) == {"pool", "query", "append", "chunk"} and all(int(n) > 3 for n in failed.values())
