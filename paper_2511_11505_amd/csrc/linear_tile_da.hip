// Input gradients on linear_tile.hpp's tiles: dz along K, the weight across it.
#include "linear_tile.hpp"

namespace fs {
void launch_tile_da(const Product& p, const Epilogue& e, const TileGrid& g, int tm, int cus,
                    hipStream_t s) {
  if (tm == 2) return run_tile<true, false, 2, 4, false>(p, e, g, cus, s);
  switch (tm) {
    case 4: run_tile<true, false, 4, 8, false>(p, e, g, cus, s); break;
    case 6: run_tile<true, false, 6, 8, false>(p, e, g, cus, s); break;
    case 7: run_tile<true, false, 7, 8, false>(p, e, g, cus, s); break;
    default: run_tile<true, false, 8, 8, false>(p, e, g, cus, s);
  }
}
}  // namespace fs
