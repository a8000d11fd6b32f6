"""The key ranges of the fp32 paged attention (csrc/key_ranges.h), compiled for the
CPU: they follow one another from the first to the last key, whole granules but for
the end, up to the longest sequence that a call accepts."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = r"""
#include "key_ranges.h"
static int check(uint32_t n, uint32_t splits, uint32_t granule) {
  uint64_t at = 0, most = 0;
  for (uint32_t s = 0; s < splits; ++s) {
    const sbd::KeyRange r = sbd::key_range(n, splits, s, granule);
    if (r.begin > r.end || r.end > n) return 1;
    if (r.begin != at) return 2;
    at = r.end;
    if (s == 0) most = r.end;
    if (r.end - r.begin > most) return 3;
    if (r.end < n && (r.end - r.begin) % granule) return 4;
  }
  // all keys, in ranges no longer than the share asks for
  return at != n ? 5 : most > ((uint64_t)n + splits - 1) / splits + granule - 1 ? 6 : 0;
}
int main() {
  const uint32_t top = 0x7fffffffu;
  for (uint32_t splits = 1; splits <= 16; ++splits)
    for (uint32_t granule = 1; granule <= 16; granule *= 2) {
      for (uint32_t n = 1; n < 700; ++n)
        if (int e = check(n, splits, granule)) return e;
      for (uint32_t back = 0; back < 700; ++back)
        if (int e = check(top - back, splits, granule)) return 10 + e;
      for (uint32_t n = 701; n < top - 12345679; n += 12345678)
        if (int e = check(n, splits, granule)) return 20 + e;
    }
  return 0;
}
"""


def test_ranges_cover_all_keys(tmp_path):
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover", "-Wall", "-Werror",
                    "-I" + os.path.join(ROOT, "paper_2509_04185_gb300", "csrc"), str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], timeout=60)
    assert r.returncode == 0, r.returncode
