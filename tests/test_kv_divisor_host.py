"""The divisions by known divisors that the key-value cache's kernels find pages, rows and shares with, compiled for the host and compared with `/` (no GPU needed)."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_03537_b200", "csrc")

SOURCE = r"""
#include <cstdio>
#include "kv_params.h"

int main() {
  unsigned divisors[4096];
  int n = 0;
  for (unsigned d = 1; d <= 1024; ++d) divisors[n++] = d;   // page sizes, groups, CTAs
  for (unsigned l = 2; l <= 17; ++l)
    for (int off = -2; off <= 2; ++off)
      if ((1u << l) + off <= 131072u) divisors[n++] = (1u << l) + off;   // up to the largest: two rows for each of 65536 heads
  for (unsigned d = 1500; d <= 131072u; d += 997) divisors[n++] = d;
  unsigned long long checked = 0;
  for (int i = 0; i < n; ++i) {
    const unsigned d = divisors[i], most = 0x7FFFFFFFu;
    const comfuse::Divisor by(d);
    auto check = [&](unsigned x) {
      if (x > most) return true;
      ++checked;
      if (by.of(x) == x / d) return true;
      std::printf("%u / %u: %u\n", x, d, by.of(x));
      return false;
    };
    for (unsigned x = 0; x < 3 * d && x < 4000u; ++x)
      if (!check(x)) return 1;
    // around multiples, where a quotient steps, all over the range and at its end
    for (unsigned long long q = 0; q * d <= most; q += 1 + most / d / 512)
      for (int off = -1; off <= 1; ++off)
        if (q * d + off <= most && !check(static_cast<unsigned>(q * d + off))) return 1;
    for (unsigned x = most - 2 * (d < 5000u ? d : 5000u); x < most; ++x)
      if (!check(x)) return 1;
    for (unsigned q = most / d, j = 0; j < 3 && q > j; ++j)
      for (int off = -1; off <= 1; ++off)
        if (!check((q - j) * d + off)) return 1;
    if (!check(most)) return 1;
  }
  std::printf("ok %d %llu\n", n, checked);
  return 0;
}
"""


def test_division_by_a_known_divisor(tmp_path):
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(SOURCE)
    cuda = os.environ.get("CUDA_HOME") or "/usr/local/cuda"
    subprocess.run([os.environ.get("CXX") or "g++", "-std=c++17", "-O2", "-I", CSRC, "-I", os.path.join(ROOT, "include"), "-I", os.path.join(cuda, "include"), str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.startswith("ok "), r.stdout
