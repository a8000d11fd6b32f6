"""Room in what the host path keeps (csrc/launch_cache.h): every cluster shape that the
library may ask about, the paged attention's among them, and the kernels' shared memory,
whose promise must not depend on how many shapes have been asked about."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = r"""
#include "launch_cache.h"
#include <cstring>
#include <initializer_list>
static sbd::LaunchCache cache;
static const void* fn(int i) { return reinterpret_cast<const void*>((uintptr_t)(0x400000 + 16 * i)); }

static int shapes() {         // all shapes and all kernels' shared memory twice: one query each
  int queries = 0, asked = 0;
  for (int rep = 0; rep < 2; ++rep) {
    asked = 0;
    auto ask = [&](int f, int threads, size_t smem, int cluster) {
      const int want = ++asked;
      cache.allow_smem(fn(f), smem, [](size_t) { return 0; });
      return cache.clusters(fn(f), threads, smem, cluster, [&] { ++queries; return want; }) == want;
    };
    int f = 0;
    for (int e = 0; e < 4; ++e, ++f)                        // bf16 attention
      for (int c = 2; c <= 16; ++c) if (!ask(f, 320, 230400, c)) return 1;
    for (int e = 0; e < 12; ++e, ++f)                       // fp32 attention, dense and paged
      for (int c : {16, 12, 10, 8, 6, 5, 4, 3, 2}) if (!ask(f, 256, 92000, c)) return 2;
    for (int rows = 16; rows <= 160; rows += 16)            // linear
      for (int c = 2; c <= 8; ++c) if (!ask(f, 320, 1024 + 2048 * rows, c)) return 3;
    ++f;
    for (int e = 0; e < 6; ++e, ++f) if (!ask(f, 320, 228352, 2)) return 4;    // CTA pairs
    for (int e = 0; e < 14; ++e, ++f)                       // bf16 attention over the paged cache
      for (int c = 2; c <= 16; ++c) if (!ask(f, 352, 224000, c)) return 5;
    for (int e = 0; e < 40; ++e, ++f) cache.allow_smem(fn(f), 90000, [](size_t) { return 0; });
  }
  if (queries != asked) return 6;
  return 2 * asked > sbd::LaunchCache::kEntries ? 7 : 0;    // and half of the room is left
}

static int smem() {           // with no place left for shapes, limits are still only raised
  for (int i = 0; i < 2 * sbd::LaunchCache::kEntries; ++i)
    cache.clusters(fn(1000 + i), 32, 0, 2, [&] { return i; });
  for (int f = 0; f < 100; ++f) {
    size_t limit = 0;
    auto set = [&](size_t most) { limit = most; return 0; };
    for (size_t need : std::initializer_list<size_t>{60000, 200000, 70000, 1, 200001, 5})
      if (cache.allow_smem(fn(f), need, set) != 0 || limit < need) return 1;
    if (limit != 200001) return 2;
  }
  return 0;
}

int main(int, char** argv) { return !strcmp(argv[1], "shapes") ? shapes() : smem(); }
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    d = tmp_path_factory.mktemp("launch_cache_room")
    src, exe = d / "t.cpp", d / "t"
    src.write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O2", "-pthread",
                    "-I" + os.path.join(ROOT, "paper_2509_04185_gb300", "csrc"), str(src), "-o", str(exe)], check=True)
    return str(exe)


@pytest.mark.parametrize("what", ["shapes", "smem"])
def test_room(program, what):
    r = subprocess.run([program, what], timeout=60)
    assert r.returncode == 0, (what, r.returncode)
