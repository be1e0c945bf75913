// Forward products on linear_tile.hpp's tiles: both operands along K, full epilogue.
#include "linear_tile.hpp"

namespace fs {
void launch_tile_forward(const Product& p, const Epilogue& e, const TileGrid& g, int tm, int cus,
                         hipStream_t s) {
  if (tm == 2) return run_tile<true, true, 2, 4, true>(p, e, g, cus, s);
  switch (tm) {
    case 4: run_tile<true, true, 4, 8, true>(p, e, g, cus, s); break;
    case 6: run_tile<true, true, 6, 8, true>(p, e, g, cus, s); break;
    case 7: run_tile<true, true, 7, 8, true>(p, e, g, cus, s); break;
    default: run_tile<true, true, 8, 8, true>(p, e, g, cus, s);
  }
}
}  // namespace fs
