"""The division by the page size as the kernels have it: csrc/kv_order.h in a program of its own."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2510_05528_b200", "csrc")
PROGRAM = """#include <cstdio>
#include <initializer_list>
#include "kv_order.h"
static long long wrong = 0, looked_at = 0;
static void one(uint32_t d, uint32_t mul, int shift, long long p) {
  if (p < 0 || p > 0x7fffffffll) return;
  ++looked_at;
  if (kv::quotient((uint32_t)p, mul, shift) != (uint32_t)p / d && wrong++ < 10) std::printf("%lld / %u\\n", p, d);
}
static void size(uint32_t d) {
  uint32_t mul; int shift;
  kv::divisor(d, mul, shift);
  // either side of multiples of d: the first, the last, and some in between; and numbers anywhere
  const long long most = 0x7fffffffll / d;
  for (long long k = 0; k <= most && k < 200; ++k)
    for (int o = -1; o <= 1; ++o) { one(d, mul, shift, k * d + o); one(d, mul, shift, (most - k) * d + o); }
  one(d, mul, shift, 0x7fffffffll);
  uint32_t x = d * 2654435761u + 1;
  for (int i = 0; i < 200; ++i) { x = x * 1664525u + 1013904223u; one(d, mul, shift, x & 0x7fffffffu); one(d, mul, shift, (long long)(x % (most + 1)) * d - 1); }
}
int main() {
  for (uint32_t d = 1; d <= 5000; ++d) size(d);
  for (int s = 1; s < 31; ++s) { size((1u << s) - 1); size(1u << s); size((1u << s) + 1); }
  size(0x7fffffffu);
  uint32_t x = 1;
  for (int i = 0; i < 20000; ++i) { x = x * 1664525u + 1013904223u; size((x >> (x & 15)) & 0x7fffffffu ? (x >> (x & 15)) & 0x7fffffffu : 1); }
  // and every position there is, for some sizes
  for (uint32_t d : {7u, 48u}) {
    uint32_t mul; int shift;
    kv::divisor(d, mul, shift);
    uint32_t q = 0, r = 0;
    for (uint32_t p = 0; p < 0x80000000u; ++p) {
      if (kv::quotient(p, mul, shift) != q && wrong++ < 10) std::printf("%u / %u\\n", p, d);
      if (++r == d) { r = 0; ++q; }
    }
  }
  std::printf("%lld %lld\\n", looked_at, wrong);
}
"""


def test_pages_of_positions(tmp_path):
    (tmp_path / "division.cc").write_text(PROGRAM)
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-I", CSRC, str(tmp_path / "division.cc"), "-o", str(tmp_path / "division")])
    lines = subprocess.check_output([str(tmp_path / "division")], text=True).split("\n")[:-1]
    looked_at, wrong = map(int, lines[-1].split())
    assert looked_at > 10 ** 6 and wrong == 0, lines[:10]


def test_the_kernels_use_it():
    text = open(os.path.join(CSRC, "kv_cache.cuh")).read() + open(os.path.join(CSRC, "kv_cache.cu")).read()
    assert "quotient(p, c.mul, c.shift)" in text and "divisor(c.page_size, c.mul, c.shift)" in text and "uint32_t quotient(" not in text
