"""Host checks on what the product's kernels read and which of them a call runs,
asked from the sources and the built library."""
from test_dispatch_host import _run, needs_build

SCALES = r"""
#include <cstdio>
#include "blocks.hpp"
using namespace spx;

// Lane l of a tile's load of scale bytes takes four from the smaller of 4 l and
// tile_scale_bytes - 4 on, counted from the tile's first row. They have to cover the tile's
// rows at their places, and none may lie behind the multiple of 16 at which the line ends.
int main() {
  long bad = 0, cut = 0;
  for (int rows : {64, 128, 256})
    for (long lines = 1; lines <= 1100; ++lines)
      for (long first = 0; first < lines; first += rows) {
        const long bytes = tile_scale_bytes(rows, first, lines), end = (lines + 15) / 16 * 16;
        const long there = lines - first < rows ? lines - first : rows;
        cut += there < rows;
        for (long lane = 0; lane < 64; ++lane) {
          const long at = 4 * lane < bytes - 4 ? 4 * lane : bytes - 4;
          bad += at < 0 || at % 4 || first + at + 4 > end || (4 * lane < there && at != 4 * lane);
        }
      }
  std::printf("bad %ld cut %ld\n", bad, cut);
  return bad != 0 || cut < 1000;
}
"""


@needs_build
def test_a_tile_reads_no_scale_bytes_behind_a_line(tmp_path):
    _run(SCALES, tmp_path)
