"""Division by multiplication (csrc/divisor.hpp) against division, on the host."""

import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2510_18239_amd", "csrc")

PROGRAM = """
#include <cstdio>
#include <initializer_list>
#include "divisor.hpp"
int main() {
  const int64_t last = (int64_t{1} << 31) - 1;
  auto check = [&](uint32_t d) {
    const lime::Divisor by(d);
    int64_t wrong = 0;
    auto at = [&](int64_t n) {
      if (n >= 0 && n <= last && by.divide(static_cast<int>(n)) != static_cast<int>(n / d)) ++wrong;
    };
    for (int64_t n = 0; n < 3000; ++n) at(n), at(last - n);
    for (int64_t q = 0; q <= last / d; q += 1 + last / d / 1000) at(q * d - 1), at(q * d), at(q * d + 1);
    if (wrong) std::printf("%u: %lld wrong\\n", d, static_cast<long long>(wrong));
    return wrong;
  };
  int64_t wrong = 0;
  for (uint32_t d = 1; d < 5000; ++d) wrong += check(d);
  for (int k = 1; k < 31; ++k)
    for (int e : {-1, 0, 1}) wrong += check((uint32_t{1} << k) + e);
  wrong += check(static_cast<uint32_t>(last)) + (lime::Divisor().divide(7) != 7);
  return wrong != 0;
}
"""


def test_divisor(tmp_path):
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
