"""Kernels read rows that do not start or end on 16-byte boundaries as the aligned packs of 16 bytes that hold them.
Before the first row's first value and after the last row's last one nothing may be read: a tensor may begin or end
there, and so may the memory.  No run shows a read beyond a tensor inside an allocation, so the function that decides
which rows are read with care is compiled for the host and tried for every alignment."""
from __future__ import annotations

import subprocess

PROGRAM = r"""
#include <cstdio>
#include "operators.cuh"

// Reads the packs of a tensor's rows as the embedding gradient's threads do, 8 columns each, and counts the bytes
// outside the tensor, the rows that are read with care and the others.
int main() {
  long outside = 0, careful = 0, plain = 0, needless = 0;
  for (int size = 2; size <= 4; size += 2)
    for (int start = 0; start < 16; start += size)        // the tensor's alignment
      for (int width = 1; width <= 40; ++width)
        for (int ld = width; ld <= width + 9; ++ld)
          for (int workers = 1; workers <= 3; ++workers)
            for (int rows = 1; rows <= 11; rows += 2)
              for (int m = 0; m < workers; ++m)
                for (int c0 = 0; c0 < width; c0 += 8) {
                  const int E = 16 / size, P = 8 / E, total = ((workers * rows - 1) * ld + width) * size;
                  const bool in = start == 0 && ld * size % 16 == 0;
                  const int Q = in ? P : P + 1;
                  const dq::Rows inside = dq::rows_inside(rows, workers, m, dq::rows_near(ld * size), !in && c0 == 0,
                                                          c0 + 16 > width && !(in && width % E == 0));
                  for (int r = 0; r < rows; ++r) {
                    if (r < inside.begin || r >= inside.end) {
                      ++careful;
                      needless += m * rows + r >= 8 && (workers - m) * rows - r > 8;
                      continue;
                    }
                    ++plain;
                    const int first = ((m * rows + r) * ld + c0) * size, s16 = (start + first) % 16;
                    for (int p = 0; p < Q; ++p)
                      if (16 * p < (width - c0) * size + s16)
                        for (int byte = first - s16 + 16 * p; byte < first - s16 + 16 * p + 16; ++byte)
                          outside += byte < 0 || byte >= total;
                  }
                }
  std::printf("%ld %ld %ld %ld\n", outside, careful, plain, needless);
  return outside || needless || careful == 0 || plain < 4 * careful;
}
"""


def test_nothing_outside_a_tensor_is_read(tmp_path):
    from paper_2010_13359_gb300 import build
    source = tmp_path / "row_ends.cu"
    source.write_text(PROGRAM)
    exe = tmp_path / "row_ends"
    subprocess.run([build.nvcc(), *build.ARCH, "-O1", "-std=c++17", "--expt-relaxed-constexpr", "-I", build.INCLUDE, "-I",
                    build.CSRC, str(source), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout
