// Shared by the linear's kernels: the product they compute, and the epilogue
// they all end in.
#pragma once

#include "internal.hpp"
#include "saved.hpp"

namespace fs {

// out[i, j] = sum over k of A(i, k) B(j, k), i < M, j < N.  An operand is
// "along" when k runs along its rows (element (i, k) at i * ld + k), else
// "across" (at k * ld + i).
struct Product {
  const void* A;
  int64_t lda;
  bool a_along;
  const void* B;
  int64_t ldb;
  bool b_along;
  int M, N, K;
};

// z = product + bias;  out = act(z) + residual, rounded once.  z and out may
// also be kept as checkpoints of their rounded values.
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

enum { ACT_NONE = 0, ACT_RELU = 1, ACT_GELU = 2, ACT_SILU = 3 };

namespace {

// Logistic function; for bf16 results the hardware exponential and reciprocal
// (about 1 ulp each in fp32).
template <typename T>
__device__ __forceinline__ float logistic(float z) {
  if constexpr (sizeof(T) == 2) return __builtin_amdgcn_rcpf(1.0f + __expf(-z));
  else return 1.0f / (1.0f + expf(-z));
}
// Phi(z), by erfc: 1 + erf(z / sqrt 2) would cancel for z far below 0
__device__ __forceinline__ float normal_cdf(float z) { return 0.5f * erfcf(z * -0.70710678118654752f); }

template <typename T>
__device__ __forceinline__ float act_value(int act, float z) {
  switch (act) {
    case ACT_RELU: return z < 0.f ? 0.f : z;
    case ACT_GELU: return z * normal_cdf(z);
    case ACT_SILU: return z * logistic<T>(z);
    default: return z;
  }
}
template <typename T>
__device__ __forceinline__ float act_slope(int act, float z) {
  switch (act) {
    case ACT_RELU: return z > 0.f ? 1.f : 0.f;
    case ACT_GELU: return normal_cdf(z) + z * 0.39894228040143268f * __expf(-0.5f * z * z);
    case ACT_SILU: {
      const float g = logistic<T>(z);
      return g * (1.f + z * (1.f - g));
    }
    default: return 1.f;
  }
}

// The epilogue of 8 columns, from c (c % 8 == 0), of row r.  Every lane of
// the wave calls it together (the checkpoints' exchange between the lanes that
// differ in bits X1 and X2); rows and columns past the end are not stored.
template <typename T, int X1, int X2>
__device__ __forceinline__ void epilogue8(const Epilogue& e, int M, int N, int64_t r, int c,
                                          float (&v)[8]) {
  const int n = min(8, N - c);
  const bool live = r < M && n > 0;
  if (e.bias && n > 0) {
    const Raw8<float> b = load8<float>(e.bias + c, n);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += b.get(i);
  }
  if (e.z && live) store8<T>((T*)e.z + r * e.ldz + c, v, n);
  if (e.z_codes) {
    float q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = i < n ? rounded<T>(v[i]) : 0.f;
    ckpt_store8<X1, X2>(e.z_codes, e.z_scales, r, c, N, q, n, live);
  }
  if (e.act != ACT_NONE) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = act_value<T>(e.act, v[i]);
  }
  if (e.res && live) {
    const Raw8<T> a = load8<T>((const T*)e.res + r * e.ldr + c, n);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += a.get(i);
  }
  if (live) store8<T>((T*)e.out + r * e.ldo + c, v, n);
  if (e.out_codes) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? rounded<T>(v[i]) : 0.f;
    ckpt_store8<X1, X2>(e.out_codes, e.out_scales, r, c, N, v, n, live);
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
