// Which kernel runs a product of the linear.  Plain C++, so that the rules can
// be built and checked without a GPU; cus is the number of compute units.
#pragma once

#include <stdint.h>

#include <algorithm>

namespace fs {
namespace {

inline int64_t cdiv_(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Tiles of the kernel whose waves split K (forward only): tokens x outputs,
// waves.
enum MidShape { MID_NONE, MID_16 /* 16 x 32, 8 */, MID_32 /* 32 x 32, 8 */, MID_64 /* 64 x 32, 8 */, MID_SHAPES };

// How a product runs: height > 0: tiles of `height` x `width` (linear_tile.hpp);
// else mid != MID_NONE: the kernel whose waves split K; else the 64 x 64 tiles.
// K is cut into `slices` of `per` K blocks of 64 (linear_tile.hpp; each at least
// 4, which its copies run ahead) or elements (64 x 64).
struct ProductPlan {
  int height, width, slices, per, mid;
  double us;   // estimated time
};

// What linear_tile.hpp asks of an operand: 16-byte chunks that lie whole in
// their row (along: K % 8 == 0; across: its width % 8 == 0), from an aligned
// base and stride, a tile's rows within 32-bit offsets.
inline bool tile_operand(uintptr_t base, int64_t ld, int64_t row_elems) {
  return base % 16 == 0 && ld % 8 == 0 && row_elems % 8 == 0 && ld <= (1 << 22);
}

// Partial sums of a cut K: at most 64 MB.
inline bool slices_fit(int64_t s, int64_t M, int64_t N) {
  return s == 1 || s * M * (cdiv_(N, 8) * 8) * 4 <= ((int64_t)64 << 20);
}
// Time in us of adding s slices: a second launch, and the sums written and read.
inline double slices_us(int64_t s, int64_t M, int64_t N) {
  return s == 1 ? 0.0 : 4.5 + (double)s * M * N * 8 / 8e6;
}

// The kernels' times in us, fitted to measurements on one MI355X; they only
// have to rank.
//
// Large tiles of h x 256: rounds over the CUs, half of a part-filled one after
// the first counted (its workgroups run faster, the chip being bound by power),
// 0.0047 us per K block and row, and a fixed part worth 53 rows.  Measured (us
// at 128, 192, 224, 256 rows): 8192 x 8192 outputs, K 5120, 528, 500, 484, 463;
// 8192 x 5120, K 8192, 564, 510, 466, 506; 4096 x 2048, K 5632, 73, 82, 91, 104;
// 4096 x 5632, K 2048, 110, 110, 121, 139; 2048 x 2048, K 2048, 32 at 128.
inline double large_us(int64_t M, int64_t N, int64_t K, int cus, int h) {
  const int64_t tiles = cdiv_(M, h) * cdiv_(N, 256), rounds = cdiv_(tiles, cus);
  const double r = rounds == 1 ? 1.0 : 0.5 * (rounds + (double)tiles / cus);
  return 4.0 + cdiv_(K, 64) * r * (h + 53) * 0.0047;
}
// 64 x 128 tiles: a K block 0.43 us while there is a workgroup per CU, 0.70 with
// two.  Measured (us, by slices): 512 x 2048, K 2048, 17.4 (1), 17.9 (2), 20.3
// (4); 128 x 4096, K 4096, 28 (1), 20.5 (2), 17.1 (4), 19.2 (8); 2048 x 2048, K
// 2048, 24.7 (1), 37.8 (2); 64 x 7168, K 2048, 17.1 (1), 14.7 (2), 14.0 (4).  (128 x
// 128 tiles were never better by more than 1 us.)
inline double small_us(int64_t M, int64_t N, int64_t per, int64_t s, int cus) {
  const int64_t wgs = cdiv_(M, 64) * cdiv_(N, 128) * s;
  return 4.0 + per * (wgs <= cus ? 0.43 : 0.70 * cdiv_(wgs, 2 * cus)) + slices_us(s, M, N);
}
// Waves splitting K: a CU gets 35 KB/us from the L2, 2.5 times less from rows
// that 16 bytes do not align, and multiplies fp32 at half an MFMA's rate.
// Measured: 64 x 512, K 512, 4.3 us at 16 x 32, 4.8, 6.0 at 64 x 32; 64 x 7168, K
// 2048, 25, 18.6, 15.0; 200 x 1000, K 2000, 11.7, 9.2, 12.2; 777 x 1001, K 1409
// (unaligned) 90, 65, 55, and 22, 19 from K 1408.
inline double mid_us(int64_t M, int64_t N, int64_t K, int es, bool aligned, int cus, int rows) {
  const double wgs = (double)cdiv_(M, rows) * cdiv_(N, 32) / cus;
  return 3.5 + std::max(wgs, 1.0) * (rows + 32) * K * es * (aligned ? 1.0 : 2.5) / 35e3;
}
// 64 x 64 tiles: a K block of 128 bytes 0.50 us (0.65 from rows that 16 bytes do
// not align, 0.79 in fp32), or 0.26 (0.34, 0.70) per workgroup of the CU.  Measured:
// 512 x 2048, K 2048, 20.0 us; 2048 x 2048, K 2048, 36.7; 777 x 1001, K 1409 (unaligned)
// 18.6 (1 slice), 19.0 (2), 21.6 (4); fp32 512 x 1408, K 2048, 55 (1), 47 (2), 42 (4),
// 1408 x 2048, K 512, 38, 4096 x 4096, K 4096, 1317; rows that 16 bytes do not align,
// by an odd stride (by a base one element off): 4096 x 4096, K 4096, 323 (458), 8192 x
// 8192, K 5120, 1773 (2270).
inline double any_us(int64_t M, int64_t N, int64_t blocks, int64_t s, bool bf16, bool aligned, int cus) {
  const double wgs = (double)(cdiv_(M, 64) * cdiv_(N, 64) * s) / cus;
  const double one = bf16 ? (aligned ? 0.50 : 0.65) : 0.79, each = bf16 ? (aligned ? 0.26 : 0.34) : 0.70;
  return 4.0 + blocks * std::max(one, each * (bf16 ? wgs : (double)(int64_t)(wgs + 0.99))) + slices_us(s, M, N);
}

// The plan of least time.  tiles_ok: the operands suit linear_tile.hpp.
inline ProductPlan product_plan(bool bf16, bool tiles_ok, bool a_along, bool b_along, int64_t M,
                                int64_t N, int64_t K, int cus) {
  ProductPlan best{0, 0, 1, 1 << 30, MID_NONE, 1e30};
  if (M <= 0 || N <= 0) return best;
  auto take = [&](double t, ProductPlan p) {
    p.us = t;
    if (t < best.us) best = p;
  };
  const int64_t blocks = cdiv_(K, 64);
  if (bf16 && tiles_ok && blocks >= 4) {
    // heights: 224 not where A lies across K (whole panels of 64 rows), 256 not
    // where K ends inside a block (the copies' pointers leave no registers)
    for (const int h : {128, 192, 224, 256})
      if ((a_along || h % 64 == 0) && (h < 256 || K % 64 == 0))
        take(large_us(M, N, K, cus, h), {h, 256, 1, (int)blocks, MID_NONE, 0});
    for (int64_t s = 1; s <= 16 && slices_fit(s, M, N); s *= 2) {
      const int64_t per = cdiv_(blocks, s), n = cdiv_(blocks, per);
      if (blocks - per * (n - 1) < 4) continue;
      take(small_us(M, N, per, n, cus), {64, 128, (int)n, (int)per, MID_NONE, 0});
    }
  }
  // (a grid holds fewer than 2^32 threads, 512 of a workgroup here)
  if (a_along && b_along && cdiv_(M, 16) * cdiv_(N, 32) < (1 << 22)) {
    take(mid_us(M, N, K, bf16 ? 2 : 4, tiles_ok, cus, 16), {0, 0, 1, 0, MID_16, 0});
    take(mid_us(M, N, K, bf16 ? 2 : 4, tiles_ok, cus, 32), {0, 0, 1, 0, MID_32, 0});
    take(mid_us(M, N, K, bf16 ? 2 : 4, tiles_ok, cus, 64), {0, 0, 1, 0, MID_64, 0});
  }
  const int64_t bk = bf16 ? 64 : 32;
  for (int64_t s = 1; s <= 32 && slices_fit(s, M, N); s *= 2) {
    const int64_t per = std::max<int64_t>(cdiv_(cdiv_(K, s), bk) * bk, bk);
    const int64_t n = std::max<int64_t>(1, cdiv_(K, per));
    take(any_us(M, N, per / bk, n, bf16, tiles_ok, cus), {0, 0, (int)n, (int)per, MID_NONE, 0});
  }
  return best;
}

// Whether operands that linear_tile.hpp cannot read for their widths (K % 8 !=
// 0 along, M or N % 8 != 0 across) are first copied to rows of whole 16-byte
// chunks (zeros behind the last element): when the tiles' time and the copies'
// are less than the other kernels'.  By the sizes alone, so that the workspace
// is known: an odd stride or base of divisible widths is not copied.  (777 x 1001, K
// 1409: 19 us without, 24 with, of which the copies 10; 4096 x 4096, K 4097, 170 with,
// where K 4096 with stride 4097 takes 323.)
inline bool product_packs(bool bf16, bool a_along, bool b_along, int64_t M, int64_t N, int64_t K, int cus) {
  if (!bf16 || M <= 0 || N <= 0) return false;
  const bool a = (a_along ? K : M) % 8 != 0, b = (b_along ? K : N) % 8 != 0;
  if (!a && !b) return false;
  const ProductPlan tiles = product_plan(true, true, a_along, b_along, M, N, K, cus);
  const double copied = (a ? (double)M * K : 0.0) + (b ? (double)N * K : 0.0);
  return tiles.height &&
         tiles.us + 9.0 + copied * 4 / 5e6 < product_plan(true, false, a_along, b_along, M, N, K, cus).us;
}

// Bytes of partial sums of the plan, whichever kernel the operands' alignment
// leaves.
inline size_t product_ws(bool bf16, bool a_along, bool b_along, int64_t M, int64_t N, int64_t K, int cus) {
  size_t b = 0;
  for (const bool ok : {false, true}) {
    const ProductPlan p = product_plan(bf16, ok, a_along, b_along, M, N, K, cus);
    if (p.slices > 1) b = std::max(b, (size_t)p.slices * M * (cdiv_(N, 8) * 8) * 4);
  }
  return b;
}

}  // namespace
}  // namespace fs
