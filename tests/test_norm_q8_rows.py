"""Which elements the 8-bit norm reads (csrc/layer/q8_rows.cuh, compiled for the host): nothing outside its
operands, whole groups of 8 on 16 bytes, and every element of every row (CPU only)."""
import os
import subprocess

from tests.test_layer_ops_args import ROOT

SRC = r"""
#include <cstdio>
#include "q8_rows.cuh"
using namespace rdn;
// 0, or what is wrong with the reads of `rows` rows of D elements, ld apart
template <int kLie>
static int look(long long rows, int D, long long ld) {
  const long long end = (rows - 1) * ld + D;
  for (long long r = 0; r < rows; ++r) {
    const int off = kLie == kShifted ? (int)(r * D & 7) : 0;
    int seen = 0;
    for (int n = 0; n * 8 < D + 16; ++n) {
      const int i = place<kLie>(n, 0, 1, off);
      const Read how = read_of<kLie>(i, D, r >= rows - near_end_rows(D));
      const int lo = i < 0 ? 0 : i, hi = i + 8 < D ? i + 8 : D;
      if (hi > lo && how == kNothing) return 1;
      if (how == kGroup && (r * ld + i < 0 || r * ld + i + 8 > end)) return 2;
      if (how == kGroup && (r * ld + i) % 8) return 3;
      if (how != kNothing) seen += hi - lo;
      if (whole<kLie>(i, D) && how != kGroup) return 5;
    }
    if (seen != D) return 4;
  }
  return 0;
}
int main() {
  for (int D = 1; D <= 70; ++D)
    for (long long rows = 1; rows <= 60; ++rows)
      for (int gap = 0; gap <= 16; gap += 8) {
        int bad = look<kShifted>(rows, D, D + gap);
        if (!bad && D % 8 == 0) bad = look<kVectors>(rows, D, D + gap);
        if (!bad) bad = look<kSingle>(rows, D, D + gap);
        if (bad) return printf("%d rows of %d, %d apart: %d\n", (int)rows, D, D + gap, bad), 1;
      }
  return 0;
}
"""


def test_reads_stay_in_the_operands(tmp_path):
    c, exe = tmp_path / "look.cpp", tmp_path / "look"
    c.write_text(SRC)
    subprocess.run(["g++", "-std=c++17", "-O1", "-D__host__=", "-D__device__=", "-D__forceinline__=inline", "-I",
                    os.path.join(ROOT, "paper_2509_25223_gb300", "csrc", "layer"), str(c), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout
