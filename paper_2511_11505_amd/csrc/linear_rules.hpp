// Which kernel runs a product of the linear.  Plain C++, so that the rules can
// be built and checked without a GPU; cus is the number of compute units.
#pragma once

#include <stdint.h>

#include <algorithm>

namespace fs {
namespace {

inline int64_t cdiv_(int64_t a, int64_t b) { return (a + b - 1) / b; }

// How a product runs: height 0: the 64 x 64 tiles; else the large tiles of
// `height` rows x 256.  K is cut into `slices` of `per` K blocks of 64 (large
// tiles) or elements (64 x 64).
struct ProductPlan {
  int height, slices, per;
};

// What the large tiles ask of an operand: 16-byte chunks that lie whole in
// their row (along: K % 8 == 0; across: its width % 8 == 0), from an aligned
// base and stride, a tile's rows within 32-bit offsets.
inline bool tile_operand(uintptr_t base, int64_t ld, int64_t row_elems) {
  return base % 16 == 0 && ld % 8 == 0 && row_elems % 8 == 0 && ld <= (1 << 22);
}

// Relative time of the large tiles of h rows: rounds over the CUs, half of a
// part-filled one counted (its workgroups run faster, the chip being bound by
// power), each its rows and a fixed part worth about 53.  Ranks the measured
// times of every height (us at 128, 160, 192, 224, 256 rows): 8192 x 8192 outputs,
// K 5120, 528, 518, 500, 484, 463; 8192 x 5120, K 8192, 564, 557, 510, 466, 506;
// 4096 x 2048, K 5632, 73, 76, 82, 91, 104; 4096 x 5632, K 2048, 110, 134, 110,
// 121, 139.
inline int64_t tile_cost(int64_t M, int64_t N, int cus, int h) {
  const int64_t tiles = cdiv_(M, h) * cdiv_(N, 256);
  return (cdiv_(tiles, cus) * cus + tiles) * (h + 53);
}

// The heights that the products have: 128, 192, 224 (not where A lies across K:
// whole panels of 64 rows) and 256 rows (not where K ends inside a block: the
// copies' pointers leave no registers for it).
inline int tile_height(int64_t M, int64_t N, int64_t K, int cus, bool a_along) {
  int best = 192;
  for (const int h : {256, 224, 128})
    if ((a_along || h % 64 == 0) && (h < 256 || K % 64 == 0) &&
        tile_cost(M, N, cus, h) < tile_cost(M, N, cus, best))
      best = h;
  return best;
}

inline ProductPlan product_plan(bool bf16, bool tiles_ok, bool a_along, int64_t M, int64_t N, int64_t K,
                                int cus) {
  if (M <= 0 || N <= 0) return {0, 1, 1 << 30};
  const int64_t np = cdiv_(N, 8) * 8;
  auto fits = [&](int64_t s) { return s * M * np * 4 <= ((int64_t)64 << 20); };   // partial sums
  if (bf16 && tiles_ok && K > 192) {
    const int h = tile_height(M, N, K, cus, a_along);
    const int64_t tiles = cdiv_(M, h) * cdiv_(N, 256), blocks = cdiv_(K, 64);
    if (tiles * 2 >= cus) return {h, 1, (int)blocks};
  }
  // 64 x 64 tiles: enough workgroups for two per CU, at least four K blocks
  // each
  const int64_t tiles = cdiv_(M, 64) * cdiv_(N, 64), bk = bf16 ? 64 : 32;
  int64_t s = std::min<int64_t>({cdiv_(2 * cus, tiles), cdiv_(K, 4 * bk), 32});
  while (s > 1 && !fits(s)) --s;
  s = std::max<int64_t>(s, 1);
  const int64_t per = std::max<int64_t>(cdiv_(cdiv_(K, s), bk) * bk, bk);
  return {0, (int)std::max<int64_t>(1, cdiv_(K, per)), (int)per};
}

// Bytes of partial sums of the plan, whichever kernel the operands' alignment
// leaves.
inline size_t product_ws(bool bf16, bool a_along, int64_t M, int64_t N, int64_t K, int cus) {
  size_t b = 0;
  for (const bool ok : {false, true}) {
    const ProductPlan p = product_plan(bf16, ok, a_along, M, N, K, cus);
    if (p.slices > 1) b = std::max(b, (size_t)p.slices * M * (cdiv_(N, 8) * 8) * 4);
  }
  return b;
}

}  // namespace
}  // namespace fs
