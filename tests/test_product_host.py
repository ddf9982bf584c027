"""Host checks on what the product's kernels read and which of them a call runs,
asked from the sources and the built library."""
import ctypes

from paper_1809_02839_amd import native
from product_shapes import KINDS, SLICED, WHOLE
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


PLANS = r"""
#include <cstdio>
#include "kernels.hpp"
using namespace spx;
int main() {
  const long shapes[][3] = {%s};
  for (const auto& s : shapes)
    for (bool exact : {false, true})
      for (bool reads : {false, true}) {
        const ProductPlan p = product_plan(s[0], s[1], s[2], exact, reads);
        const long blocks = (s[2] + 127) / 128, plane = s[0] * s[1] * 4;
        // every slice has blocks of k, and the workspace holds a plane for each
        if (p.slices > 1 && (p.slices * p.per_slice < blocks || (p.slices - 1) * p.per_slice >= blocks ||
                             product_ws_bytes(s[0], s[1], s[2]) < static_cast<size_t>(p.slices * plane)))
          return 1;
        std::printf("%%d %%d %%d\n", p.tile, p.slices, int(p.slices * p.per_slice > blocks));
      }
}
"""


def _plans(shapes, tmp_path):
    """(tile, slices, whether the last slice is short) of each shape, by kind."""
    out = _run(PLANS % ", ".join("{%d, %d, %d}" % s for s in shapes), tmp_path).splitlines()
    rows = [tuple(map(int, l.split())) for l in out]
    return [rows[i:i + 4] for i in range(0, len(rows), 4)]


@needs_build
def test_the_sliced_shapes_run_the_kernels_they_are_there_for(tmp_path):
    """The cost model may move; then the shapes have to follow, or a kernel goes untested."""
    reached = set()
    for (shape, tiles), plans in zip(SLICED.items(), _plans(SLICED, tmp_path)):
        for kind, tile, plan in zip(KINDS, tiles, plans):
            print(shape, kind, plan)
            assert plan[0] == tile and plan[1] > 1, (shape, kind, plan)
            reached.add((kind, tile, plan[2]))
    for kind in KINDS:
        assert {(t, 1) for t in (64, 128, 256)} <= {(t, short) for k, t, short in reached if k == kind}, kind


@needs_build
def test_the_whole_shapes_run_the_kernels_they_are_there_for(tmp_path):
    for (shape, tile), plans in zip(WHOLE.items(), _plans(WHOLE, tmp_path)):
        assert all(p[:2] == (tile, 1) for p in plans), (shape, plans)


def test_scale_lines_are_taken_up_to_the_stated_size():
    """scales_ld * ceil(k / 128) below 2^31 is accepted, also where 2^31 is no multiple of the blocks of k (a call of no
    rows: the arguments are checked, nothing runs)."""
    blocks, ld = 32760, 65552
    assert blocks * ld < 1 << 31 <= blocks * (ld + 16)
    for side in ("a_scales_ld", "b_scales_ld"):
        for extra, code in ((0, native.OK), (16, native.EINVAL)):
            d = native.ProductDesc(native.ABI_VERSION, native.FP32, native.FP32, 0, 0, 0, 0, 64, 128 * blocks, 1 << 22, 64,
                                   1 << 22, 64, 64, 64)
            setattr(d, side, ld + extra)
            rc = native.lib().spectrain_product(ctypes.byref(d), 4096, 8192, 12288, 16384, None, None, None, None, 0, None)
            assert rc == code, (side, extra, native.lib().spectrain_last_error())
