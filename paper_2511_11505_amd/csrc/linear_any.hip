// The linear's products of any type, alignment, stride and size: tiles of 64 x
// 64, four waves of 32 x 32, staged through registers into LDS.
//
// bf16 multiplies on v_mfma_f32_16x16x32_bf16, fp32 on v_mfma_f32_32x32x2_f32 (on
// one wave per SIMD, register operands only, 143 TFLOP/s against 98 of the 16 x
// 16 x 4 form, whose chains of dependent instructions wait).  A block of one
// workgroup per CU is bound by latency; blocks therefore go through registers
// two ahead of LDS, and the loads' pointers only advance.

#include <type_traits>

#include "linear.hpp"

namespace fs {
namespace {

typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;

// One operand's 64 rows x 128 bytes of K in LDS, as it lies in memory: along,
// 64 rows of 128 bytes; across, BK rows (of k) of 64 elements.  Padding
// spreads the rows over the banks.
template <typename T, bool ALONG>
struct Panel {
  static constexpr int V = 16 / sizeof(T), BK = 128 / sizeof(T);
  static constexpr int ROWS = ALONG ? 64 : BK, PIECES = ALONG ? 8 : 64 / V;
  static constexpr int STRIDE = (ALONG ? 128 : 64 * (int)sizeof(T)) + 16;   // bytes
  static constexpr int BYTES = ROWS * STRIDE;
  // This thread's two 16-byte pieces: where the next whole K block has them,
  // and how many of their elements exist.  (Rows past the end, along, are
  // copies of the last: their outputs are not stored.)
  const T* p[2];
  int n[2];
  int64_t step;
  __device__ __forceinline__ void init(const T* base, int64_t ld, int row0, int rows, int k0) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int q = (int)threadIdx.x + 256 * i, r = q / PIECES, e = (q % PIECES) * V;
      if constexpr (ALONG) {
        p[i] = base + (int64_t)min(row0 + r, rows - 1) * ld + k0 + e;
        n[i] = V;
      } else {
        p[i] = base + (int64_t)(k0 + r) * ld + row0 + e;
        n[i] = rows - row0 - e;
      }
    }
    step = ALONG ? BK : BK * ld;
  }
  // the K block with `left` elements of K
  __device__ __forceinline__ void fetch(int left, uint4 (&st)[2]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      int have = n[i];
      if (left < BK) {   // (uniform; the last block)
        const int q = (int)threadIdx.x + 256 * i;
        if (ALONG) have = left - (q % PIECES) * V;
        else if (q / PIECES >= left) have = 0;
      }
      if (ALONG && left >= BK) st[i] = load16<T>(p[i], V);
      else st[i] = have > 0 ? load16<T>(p[i], have) : make_uint4(0, 0, 0, 0);
      p[i] += step;
    }
  }
  static __device__ __forceinline__ void put(unsigned char* lds, const uint4 (&st)[2]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int q = (int)threadIdx.x + 256 * i;
      st16(lds + (q / PIECES) * STRIDE + (q % PIECES) * 16, st[i]);
    }
  }
  // The fragment of a wave's 32 rows from r0.  bf16: 16 rows from r0, 32 of K
  // per step: lane l row l % 16, k 8 (l / 16) .. + 7; fp32: 32 rows, 8 of K per
  // step: lane l row l % 32, k 4 (l / 32) .. + 3.
  static __device__ __forceinline__ uint4 frag(const unsigned char* lds, int r0, int step) {
    const int lane = threadIdx.x & 63;
    if constexpr (sizeof(T) == 4) {
      const int r = lane & 31, g = lane >> 5;
      if constexpr (ALONG) return *reinterpret_cast<const uint4*>(lds + (r0 + r) * STRIDE + step * 32 + g * 16);
      uint4 f;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        (&f.x)[i] = *reinterpret_cast<const uint32_t*>(lds + (step * 8 + 4 * g + i) * STRIDE + (r0 + r) * 4);
      return f;
    } else {
      const int r = lane & 15, g = lane >> 4;
      if constexpr (ALONG) return *reinterpret_cast<const uint4*>(lds + (r0 + r) * STRIDE + step * 64 + g * 16);
      // a transposing read: in each 16-lane group lane p gives the address
      // of 4 elements of row p / 4, columns 4 (p % 4) .., and gets the 4 rows
      // of column p
      const unsigned char* q = lds + (step * 32 + 8 * g + (r >> 2)) * STRIDE + (r0 + 4 * (r & 3)) * 2;
      const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)q);
      const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(q + 4 * STRIDE));
      const uint2 a = __builtin_bit_cast(uint2, lo), b = __builtin_bit_cast(uint2, hi);
      return make_uint4(a.x, a.y, b.x, b.y);
    }
  }
};

// LDS of a tile: two slots of both operands.
template <typename T, bool LA, bool LB>
constexpr int any_lds() {
  return 2 * (Panel<T, LA>::BYTES + Panel<T, LB>::BYTES);
}

// Tile `tile` of the product, K slice `slice` of kper elements; with more than
// one slice the fp32 sums go to part[slice][M][np].
template <typename T, bool LA, bool LB>
__device__ __forceinline__ void any_tile(const Product& p, const Epilogue& e, int tile, int slice, int kper,
                                         float* __restrict__ part, int np, unsigned char* smem) {
  using PA = Panel<T, LA>;
  using PB = Panel<T, LB>;
  constexpr int BK = 128 / sizeof(T);
  constexpr bool F32 = sizeof(T) == 4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wm = (wave >> 1) * 32, wn = (wave & 1) * 32;
  const int tiles_n = (p.N + 63) / 64;
  const int n0 = tile % tiles_n * 64, m0 = tile / tiles_n * 64;
  const int k0 = slice * kper, kend = min(p.K, k0 + kper);
  floatx4 acc[2][2] = {};
  floatx16 accf = {};
  uint4 ra[2][2], rb[2][2];
  PA pa;
  PB pb;
  pa.init((const T*)p.A, p.lda, m0, p.M, k0);
  pb.init((const T*)p.B, p.ldb, n0, p.N, k0);
  auto fetch = [&](int i, int kb) __attribute__((always_inline)) {
    if (kb < kend) {
      pa.fetch(kend - kb, ra[i]);
      pb.fetch(kend - kb, rb[i]);
    }
  };
  auto block = [&](int i, int kb) __attribute__((always_inline)) {
    unsigned char *sa = smem + i * PA::BYTES, *sb = smem + 2 * PA::BYTES + i * PB::BYTES;
    PA::put(sa, ra[i]);
    PB::put(sb, rb[i]);
    __syncthreads();
    fetch(i, kb + 2 * BK);
    if constexpr (F32) {
#pragma unroll
      for (int step = 0; step < 4; ++step) {
        const uint4 fa = PA::frag(sa, wm, step), fb = PB::frag(sb, wn, step);
#pragma unroll
        for (int k = 0; k < 4; ++k)
          accf = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float((&fb.x)[k]), __uint_as_float((&fa.x)[k]),
                                                      accf, 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int step = 0; step < 2; ++step) {
        uint4 fa[2], fb[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          fa[j] = PA::frag(sa, wm + 16 * j, step);
          fb[j] = PB::frag(sb, wn + 16 * j, step);
        }
        mma_step<T>(fa, fb, acc);
      }
    }
  };
  fetch(0, k0);
  fetch(1, k0 + BK);
  for (int kb = k0; kb < kend; kb += 2 * BK) {
    block(0, kb);
    if (kb + BK < kend) block(1, kb + BK);
  }
  auto finish = [&](int64_t r, int c, float (&v)[8], auto lanes) __attribute__((always_inline)) {
    if (part) {
      if (r < p.M && c < p.N) store8<float>(part + ((int64_t)slice * p.M + r) * np + c, v, 8);
    } else {
      epilogue8<T, decltype(lanes)::value>(e, p.M, p.N, r, c, v, epilogue_bias(e, p.N, c),
                                           epilogue_res<T>(e, p.M, p.N, r, c));
    }
  };
  if constexpr (F32) {
    // element v of lane l is row l % 32 of the tokens, output 8 (v / 4) + 4 (l
    // / 32) + v % 4: through LDS to 8 consecutive outputs per lane
    constexpr int LD = 68;
    static_assert(64 * LD * 4 <= any_lds<T, LA, LB>(), "the tile fits");
    float* t = reinterpret_cast<float*>(smem);
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *reinterpret_cast<floatx4*>(t + (wm + (lane & 31)) * LD + wn + 8 * q + 4 * (lane >> 5)) =
          floatx4{accf[4 * q], accf[4 * q + 1], accf[4 * q + 2], accf[4 * q + 3]};
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int q = (int)threadIdx.x + 256 * i, r = q / 8, c = q % 8 * 8;
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = t[r * LD + c + j];
      finish((int64_t)m0 + r, n0 + c, v, std::integral_constant<int, LANES_NEXT>{});
    }
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float v[8];
      join8(acc[i][0], acc[i][1], v);
      finish((int64_t)m0 + wm + 16 * i + (lane & 15), n0 + wn + col8(lane), v,
             std::integral_constant<int, LANES_APART>{});
    }
  }
}

// Grid (tiles, K slices).
template <typename T, bool LA, bool LB>
__global__ __launch_bounds__(256) void linear_any_kernel(Product p, Epilogue e, int kper,
                                                         float* __restrict__ part, int np) {
  __shared__ __align__(16) unsigned char smem[any_lds<T, LA, LB>()];
  any_tile<T, LA, LB>(p, e, blockIdx.x, blockIdx.y, kper, part, np, smem);
}

// Both products of a small backward pass in one launch: the first `tiles` of the
// grid are da's.
template <typename T>
__global__ __launch_bounds__(256) void linear_any_pair_kernel(Product da, Epilogue eda, int tiles, Product dw,
                                                              Epilogue edw) {
  constexpr int L1 = any_lds<T, true, false>(), L2 = any_lds<T, false, false>();
  __shared__ __align__(16) unsigned char smem[L1 > L2 ? L1 : L2];
  if ((int)blockIdx.x < tiles) any_tile<T, true, false>(da, eda, blockIdx.x, 0, da.K, nullptr, 0, smem);
  else any_tile<T, false, false>(dw, edw, blockIdx.x - tiles, 0, dw.K, nullptr, 0, smem);
}

// Sum of the K slices, in slice order, and the epilogue.  A thread holds 8
// columns, four neighbours a checkpoint's block.
template <typename T>
__global__ __launch_bounds__(256) void linear_reduce_kernel(const float* __restrict__ part, int slices,
                                                            int M, int N, int np, Epilogue e) {
  const int cpr = (N + 31) / 32 * 4;   // chunks of 8 columns per row
  const int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t r = q / cpr;
  const int c = (int)(q - r * cpr) * 8;
  float v[8] = {};
  if (r < M && c < N)
    for (int s = 0; s < slices; ++s) {
      const Raw8<float> x = load8<float>(part + ((int64_t)s * M + r) * np + c, 8);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += x.get(i);
    }
  epilogue8<T, LANES_NEXT>(e, M, N, r, c, v, epilogue_bias(e, N, c), epilogue_res<T>(e, M, N, r, c));
}

int64_t tiles_of(const Product& p) { return cdiv64(p.N, 64) * cdiv64(p.M, 64); }

template <typename T>
void run_any(const Product& p, const Epilogue& e, int slices, int per, float* part, int np, hipStream_t s) {
  const dim3 grid((unsigned)tiles_of(p), (unsigned)slices);
  float* dst = slices > 1 ? part : nullptr;
  if (p.a_along && p.b_along)
    launch_k(linear_any_kernel<T, true, true>, grid, 256, 0, s, p, e, per, dst, np);
  else if (p.a_along)
    launch_k(linear_any_kernel<T, true, false>, grid, 256, 0, s, p, e, per, dst, np);
  else
    launch_k(linear_any_kernel<T, false, false>, grid, 256, 0, s, p, e, per, dst, np);
}

}  // namespace

void launch_any(int dtype, const Product& p, const Epilogue& e, int slices, int per, float* part, int np,
                hipStream_t s) {
  if (dtype == 0) run_any<float>(p, e, slices, per, part, np, s);
  else run_any<bf16_t>(p, e, slices, per, part, np, s);
}

void launch_any_pair(int dtype, const Product& da, const Epilogue& eda, const Product& dw, const Epilogue& edw,
                     hipStream_t s) {
  const int tiles = (int)tiles_of(da);
  const unsigned grid = (unsigned)(tiles + tiles_of(dw));
  if (dtype == 0) launch_k(linear_any_pair_kernel<float>, grid, 256, 0, s, da, eda, tiles, dw, edw);
  else launch_k(linear_any_pair_kernel<bf16_t>, grid, 256, 0, s, da, eda, tiles, dw, edw);
}

void launch_reduce(int dtype, const float* part, int slices, int M, int N, int np, const Epilogue& e,
                   hipStream_t s) {
  const unsigned grid = (unsigned)cdiv64((int64_t)M * ((N + 31) / 32 * 4), 256);
  if (dtype == 0) launch_k(linear_reduce_kernel<float>, grid, 256, 0, s, part, slices, M, N, np, e);
  else launch_k(linear_reduce_kernel<bf16_t>, grid, 256, 0, s, part, slices, M, N, np, e);
}

}  // namespace fs
