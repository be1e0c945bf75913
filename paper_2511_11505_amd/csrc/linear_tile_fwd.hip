// Forward products on the large tiles: both operands along K, full epilogue.
#include "linear_tile.hpp"

namespace fs {
void launch_tile_forward(const Product& p, const Epilogue& e, const TileGrid& g, int tm, int cus,
                         hipStream_t s) {
  switch (tm) {
    case 4: run_tile<true, true, 4, true>(p, e, g, cus, s); break;
    case 6: run_tile<true, true, 6, true>(p, e, g, cus, s); break;
    case 7: run_tile<true, true, 7, true>(p, e, g, cus, s); break;
    default: run_tile<true, true, 8, true>(p, e, g, cus, s);
  }
}
}  // namespace fs
