"""The host-made divisors of the cache's slot arithmetic, on the CPU."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_23406_amd", "csrc")

SOURCE = r"""
#include "hq_internal.h"
#include <cstdio>
static uint32_t of(hq_divisor d, uint32_t n) { return d.mul ? (uint32_t)(((uint64_t)n * d.mul) >> 32) >> d.shift : n; }
int main() {
  unsigned bad = 0, seen = 0;
  uint32_t x = 1;
  auto check = [&](uint32_t d) {
    const hq_divisor r = hq_divide_by(d);
    for (int k = 0; k < 3000; ++k) {
      x = x * 1664525u + 1013904223u;
      const uint32_t any = x & 0x7FFFFFFFu, at = any / d * d;  // a multiple, and just below the next one
      for (uint32_t n : {any, at, at + (d - 1), (uint32_t)k, 0x7FFFFFFFu - k})
        if (n <= 0x7FFFFFFFu) bad += of(r, n) != n / d, ++seen;
    }
  };
  for (uint32_t d = 1; d < 70000; d += d < 600 ? 1 : 191) check(d);
  for (uint32_t d : {0x3FFFFFFFu, 0x40000000u, 0x40000001u, 0x7FFFFFFEu, 0x7FFFFFFFu}) check(d);
  printf("%u %u\n", bad, seen);
}
"""


def test_divisions_of_31_bit_numbers(tmp_path):
    src = tmp_path / "d.cpp"
    src.write_text("#include <initializer_list>\n" + SOURCE)
    exe = tmp_path / "d"
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", CSRC, "-o", str(exe), str(src)], check=True)
    bad, seen = map(int, subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split())
    assert bad == 0 and seen > 10 ** 6
