// Host side of the paged attention's row arithmetic, compiled without device
// code and called through ctypes by test_paged_rules.py.
#include "../paper_2608_23463_amd/csrc/paged.hpp"

using namespace pf;

// What `cols` columns from x0 on see, of a sequence whose new tokens begin at
// row0 and whose table holds `most` rows: first, top, last, the tiles of the
// first rows, the gap behind them, and the number of tiles.
extern "C" void host_sight(int row0, int most, int group, int x0, int cols, int tile_rows, int window, int sinks,
                           int* out) {
  PagedParams p{};
  p.fgroup = FastDiv(group);
  p.window = window;
  p.sinks = sinks;
  Sequence sq{};
  sq.row0 = row0;
  sq.most = most;
  const Sight s(p, sq, x0, cols, tile_rows);
  out[0] = s.first, out[1] = s.top, out[2] = s.last;
  out[3] = s.head_tiles, out[4] = s.gap, out[5] = s.tiles;
}
