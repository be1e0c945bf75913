// Weight gradients on linear_tile.hpp's tiles: both operands across K (the tokens).
#include "linear_tile.hpp"

namespace fs {
void launch_tile_dw(const Product& p, const Epilogue& e, const TileGrid& g, int tm, int cus,
                    hipStream_t s) {
  if (tm == 2) return run_tile<false, false, 2, 4, false>(p, e, g, cus, s);
  switch (tm) {
    case 4: run_tile<false, false, 4, 8, false>(p, e, g, cus, s); break;
    case 6: run_tile<false, false, 6, 8, false>(p, e, g, cus, s); break;
    default: run_tile<false, false, 8, 8, false>(p, e, g, cus, s);
  }
}
}  // namespace fs
