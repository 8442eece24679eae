// Which elements the quantiser's wide loads read, for every small matrix: none behind the last element of its last row
// (see tests/test_quantize_reads.py).
#include <cstdio>
#include "../../paper_2203_17189_amd/csrc/fp8.h"

int main() {
  long reads = 0, bad = 0;
  for (int size : {2, 4})
    for (int ld = 1; ld <= 300; ++ld) {
      if (!t5mi::quant_in_pieces(nullptr, ld, size)) continue;
      for (int cols = 1; cols <= ld; ++cols)
        for (int rows = 1; rows <= 4; ++rows)
          for (int row = 0; row < rows; ++row)
            for (int c = 0; c < cols; c += 8) {
              if (!t5mi::quant_whole_piece(c, cols, row + 1 < rows)) continue;
              ++reads;
              if ((long)row * ld + c + 8 > (long)(rows - 1) * ld + cols && bad++ < 20)
                std::printf("%d bytes an element, %d x %d, rows %d apart: row %d, columns %d to %d\n", size, rows, cols, ld, row, c, c + 7);
            }
    }
  std::printf("%ld reads, %ld past the end\n", reads, bad);
  return bad || !reads;
}
