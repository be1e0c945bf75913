// Shared by the linear's kernels: the product they compute, and the epilogue
// they all end in.
#pragma once

#include "internal.hpp"
#include "saved.hpp"

namespace fs {

// out[i, j] = sum over k of A(i, k) B(j, k), i < M, j < N.  An operand is
// "along" when k runs along its rows (element (i, k) at i * ld + k), else
// "across" (at k * ld + i).  *_padded: the rows go on to a multiple of 8
// elements, with zeros.  *_pack: room for such a copy, or null.
struct Product {
  const void* A;
  int64_t lda;
  bool a_along, a_padded;
  const void* B;
  int64_t ldb;
  bool b_along, b_padded;
  int M, N, K;
  void *a_pack, *b_pack;
};

// z = product + bias;  out = act(z) + residual, rounded once.  z and out may
// also be kept as checkpoints of their rounded values (scales: null without
// codes).
struct Epilogue {
  const float* bias;
  const void* res;
  int64_t ldr;
  void* out;
  int64_t ldo;
  void* z;
  int64_t ldz;
  uint8_t *z_codes, *z_scales, *out_codes, *out_scales;
  int act;
};

// The large tiles' grid (linear_tile.hpp).
struct TileGrid {
  int tiles_m, tiles_n, slices;
  int kb_per;      // K blocks per slice (the last may have fewer, but 4)
  float* part;     // more than one slice: fp32 sums [slice][M][np]
  int np;
};
// tm: tile height in units of 32 rows, 2 (of 128 columns), 4, 6, 7 or 8 (of 256;
// dw: not 7); cus: compute units to fill.
typedef void TileLaunch(const Product& p, const Epilogue& e, const TileGrid& g, int tm, int cus,
                        hipStream_t s);
TileLaunch launch_tile_forward, launch_tile_da, launch_tile_dw;

// 64 x 64 tiles for everything (linear_any.hip): K in `slices` of `per` elements,
// the sums of more than one to part; both products of a small backward pass in
// one launch; the sum of the slices with the epilogue.
void launch_any(int dtype, const Product& p, const Epilogue& e, int slices, int per, float* part, int np,
                hipStream_t s);
void launch_any_pair(int dtype, const Product& da, const Epilogue& eda, const Product& dw, const Epilogue& edw,
                     hipStream_t s);
void launch_reduce(int dtype, const float* part, int slices, int M, int N, int np, const Epilogue& e,
                   hipStream_t s);

// Forward products of up to kFewTokens rows (linear_few.hip).
constexpr int kFewTokens = 8;
void launch_few(int dtype, const Product& p, const Epilogue& e, int cus, hipStream_t s);

// Forward products on tiles whose waves split K (linear_mid.hip); shape: a
// MidShape of linear_rules.hpp.
void launch_mid(int dtype, const Product& p, const Epilogue& e, int shape, hipStream_t s);

enum { ACT_NONE = 0, ACT_RELU = 1, ACT_GELU = 2, ACT_SILU = 3 };

namespace {

// Logistic function; for bf16 results the hardware exponential and reciprocal
// (about 1 ulp each in fp32).
template <typename T>
__device__ __forceinline__ float logistic(float z) {
  if constexpr (sizeof(T) == 2) return __builtin_amdgcn_rcpf(1.0f + __expf(-z));
  else return 1.0f / (1.0f + expf(-z));
}
// Phi(z) and exp(-z^2 / 2).  By erfc, since 1 + erf(z / sqrt 2) would cancel
// for z far below 0.  For bf16 results erfc(x) = t Q(t) exp(-x^2), t = 1 / (1 +
// 0.4 x), with Q of degree 7 fitted here to exp(x^2) erfc(x) / t over 0 <= x
// <= 10 for the least relative error, 4.5e-7 (reweighted least squares at
// Chebyshev points); the library's erfcf took 58 us of a 4096 x 5632 backward
// pass's act' against 23 us of memory.
template <typename T>
__device__ __forceinline__ float normal_cdf(float z, float& gauss) {
  if constexpr (sizeof(T) == 2) {
    gauss = __expf(-0.5f * z * z);
    const float t = __builtin_amdgcn_rcpf(fmaf(0.4f * 0.70710678118654752f, fabsf(z), 1.0f));
    float q = 0.051215760409832f;
    q = fmaf(q, t, -0.2920388877391815f);
    q = fmaf(q, t, 0.49442407488822937f);
    q = fmaf(q, t, -0.18401390314102173f);
    q = fmaf(q, t, 0.2983193099498749f);
    q = fmaf(q, t, 0.1769629865884781f);
    q = fmaf(q, t, 0.22967028617858887f);
    q = fmaf(q, t, 0.22545994818210602f);
    q *= 0.5f * t * gauss;
    return z > 0.f ? 1.0f - q : q;
  } else {
    gauss = expf(-0.5f * z * z);
    return 0.5f * erfcf(z * -0.70710678118654752f);
  }
}

// act and act' of 8 values; the choice is made once, outside the loops (inside,
// every element takes the branches: 18 us more for each 224 x 256 tile).
template <typename T>
__device__ __forceinline__ void act8(int act, float (&v)[8]) {
  float gauss;
  if (act == ACT_RELU) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = v[i] < 0.f ? 0.f : v[i];
  } else if (act == ACT_GELU) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= normal_cdf<T>(v[i], gauss);
  } else if (act == ACT_SILU) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= logistic<T>(v[i]);
  }
}
template <typename T>
__device__ __forceinline__ void act_slope8(int act, float (&v)[8]) {
  if (act == ACT_RELU) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = v[i] > 0.f ? 1.f : 0.f;
  } else if (act == ACT_GELU) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float gauss;
      const float cdf = normal_cdf<T>(v[i], gauss);
      v[i] = fmaf(v[i] * 0.39894228040143268f, gauss, cdf);
    }
  } else if (act == ACT_SILU) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float g = logistic<T>(v[i]);
      v[i] = g * (1.f + v[i] * (1.f - g));
    }
  }
}

// What the epilogue of 8 columns reads: the bias, and the residual of a row.
// Loaded apart from epilogue8, so that a kernel with many of them can ask for
// all early: a load behind a store waits for the store to finish.
__device__ __forceinline__ Raw8<float> epilogue_bias(const Epilogue& e, int N, int c) {
  Raw8<float> b = {};
  if (e.bias && c < N) b = load8<float>(e.bias + c, min(8, N - c));
  return b;
}
template <typename T>
__device__ __forceinline__ Raw8<T> epilogue_res(const Epilogue& e, int M, int N, int64_t r, int c) {
  Raw8<T> a = {};
  if (e.res && r < M && c < N) a = load8<T>((const T*)e.res + r * e.ldr + c, min(8, N - c));
  return a;
}

// The epilogue of 8 columns, from c (c % 8 == 0), of row r.  Every lane of
// the wave calls it together (the checkpoints' exchange between the lanes of a
// block); rows and columns past the end are not stored.  The blocks' scale
// bytes are returned (z's in bits 0 .. 7, out's in bits 8 .. 15), and written
// unless the caller does.
template <typename T, int LANES, bool SCALE = true>
__device__ __forceinline__ uint32_t epilogue8(const Epilogue& e, int M, int N, int64_t r, int c,
                                              float (&v)[8], const Raw8<float>& bias,
                                              const Raw8<T>& res) {
  const int n = min(8, N - c);
  const bool live = r < M && n > 0;
  uint32_t bytes = 0;
  if (e.bias) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += bias.get(i);
  }
  if (e.z && live) store8<T>((T*)e.z + r * e.ldz + c, v, n);
  if (e.z_codes) {
    float q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = i < n ? rounded<T>(v[i]) : 0.f;
    bytes = ckpt_store8<LANES, SCALE>(e.z_codes, e.z_scales, r, c, N, q, n, live);
  }
  act8<T>(e.act, v);
  if (e.res) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += res.get(i);
  }
  if (live) store8<T>((T*)e.out + r * e.ldo + c, v, n);
  if (e.out_codes) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? rounded<T>(v[i]) : 0.f;
    bytes |= ckpt_store8<LANES, SCALE>(e.out_codes, e.out_scales, r, c, N, v, n, live) << 8;
  }
  return bytes;
}

// One step of K on MF x NF fragments of 16 x 16 outputs: 16 bytes per lane and
// operand, that is 32 of K for bf16, 16 for fp32 (whose four instructions per
// fragment do not follow each other: each would wait for the last).
template <typename T, int MF, int NF>
__device__ __forceinline__ void mma_step(const uint4 (&a)[MF], const uint4 (&b)[NF], floatx4 (&c)[MF][NF]) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
      for (int j = 0; j < NF; ++j)
        c[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, b[j]),
                                                          __builtin_bit_cast(bf16x8, a[i]), c[i][j], 0, 0, 0);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int j = 0; j < NF; ++j)
          c[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float((&b[j].x)[k]),
                                                         __uint_as_float((&a[i].x)[k]), c[i][j], 0, 0, 0);
  }
}

// Two 16 x 16 accumulators of neighbouring column fragments (the weights are
// the MFMA's row operand, so lane l holds row l % 16 and columns 4 (l / 16) ..
// + 3 of each) to 8 consecutive columns per lane: odd 16-lane groups of the
// first change places with even groups of the second.  Lane group g then
// holds columns col8(g) .. + 7 of the 32.
__device__ __forceinline__ void join8(const floatx4& x, const floatx4& y, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x[i]), __float_as_uint(y[i]),
                                                    false, false);
    v[i] = __uint_as_float(p[0]);
    v[4 + i] = __uint_as_float(p[1]);
  }
}
__device__ __forceinline__ int col8(int lane) { return 16 * ((lane >> 4) & 1) + 8 * (lane >> 5); }

}  // namespace
}  // namespace fs
