// Forward products of few tokens (up to kFewTokens), which are bound by
// reading the weight once, and for one token by latency: no LDS, no K split
// over workgroups, one launch.
//
// A wave holds R weight rows; its lanes lie along K, so that a load is 1 KB of
// one row, and each lane multiplies its 16 bytes with every token's.  Four
// steps' loads are asked for together.  bf16 pairs go through v_dot2_f32_bf16
// (fp32 sum); the lanes' sums are added over the wave at the end.

#include "linear.hpp"

namespace fs {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

template <typename T>
__device__ __forceinline__ float dot16(const uint4& a, const uint4& b, float s) {
  const uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 2)
      s = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, x[i]), __builtin_bit_cast(bf16x2, y[i]),
                                          s, false);
    else
      s = fmaf(__uint_as_float(x[i]), __uint_as_float(y[i]), s);
  }
  return s;
}

template <typename T, int M, int R>
__global__ __launch_bounds__(256) void linear_few_kernel(Product p, Epilogue e) {
  constexpr int V = 16 / sizeof(T), STEP = 64 * V, U = M * R <= 8 ? 4 : 2;
  const int lane = threadIdx.x & 63;
  const int n0 = ((int)blockIdx.x * 4 + (threadIdx.x >> 6)) * R;
  if (n0 >= p.N) return;
  const T *a[M], *w[R];
#pragma unroll
  for (int t = 0; t < M; ++t) a[t] = (const T*)p.A + (int64_t)min(t, p.M - 1) * p.lda + lane * V;
#pragma unroll
  for (int r = 0; r < R; ++r) w[r] = (const T*)p.B + (int64_t)min(n0 + r, p.N - 1) * p.ldb + lane * V;
  float s[M][R] = {};
  int k = 0;
  for (; k + U * STEP <= p.K; k += U * STEP) {
    uint4 wv[U][R], av[U][M];
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int r = 0; r < R; ++r) wv[u][r] = load16<T>(w[r] + k + u * STEP, V);
#pragma unroll
      for (int t = 0; t < M; ++t) av[u][t] = load16<T>(a[t] + k + u * STEP, V);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int t = 0; t < M; ++t)
#pragma unroll
        for (int r = 0; r < R; ++r) s[t][r] = dot16<T>(av[u][t], wv[u][r], s[t][r]);
  }
  // the rest a step at a time, the last one short
  for (; k < p.K; k += STEP) {
    const int n = p.K - k - lane * V;
    uint4 wv[R], av[M];
#pragma unroll
    for (int r = 0; r < R; ++r) wv[r] = n > 0 ? load16<T>(w[r] + k, n) : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int t = 0; t < M; ++t) av[t] = n > 0 ? load16<T>(a[t] + k, n) : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int t = 0; t < M; ++t)
#pragma unroll
      for (int r = 0; r < R; ++r) s[t][r] = dot16<T>(av[t], wv[r], s[t][r]);
  }
  // lane t R + r ends up with token t, row r
  float v = 0.f;
#pragma unroll
  for (int t = 0; t < M; ++t)
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const float x = wave_sum(s[t][r]);
      v = lane == t * R + r ? x : v;
    }
  const int t = lane / R, c = n0 + lane % R;
  if (t >= p.M || lane >= M * R || c >= p.N) return;
  float q[8] = {v};
  if (e.bias) q[0] += e.bias[c];
  if (e.z) ((T*)e.z)[t * e.ldz + c] = from_f32<T>(q[0]);
  act8<T>(e.act, q);
  if (e.res) q[0] += to_f32<T>(((const T*)e.res)[t * e.ldr + c]);
  ((T*)e.out)[t * e.ldo + c] = from_f32<T>(q[0]);
}

// Rows per wave: one while that gives at most eight waves per CU, then two,
// which halves the reads of the tokens.
template <typename T, int M>
void run_few(const Product& p, const Epilogue& e, int cus, hipStream_t s) {
  if (p.N <= 8 * cus) launch_k(linear_few_kernel<T, M, 1>, (unsigned)cdiv64(p.N, 4), 256, 0, s, p, e);
  else launch_k(linear_few_kernel<T, M, 2>, (unsigned)cdiv64(p.N, 8), 256, 0, s, p, e);
}

}  // namespace

void launch_few(int dtype, const Product& p, const Epilogue& e, int cus, hipStream_t s) {
#define FS_FEW(T)                              \
  do {                                         \
    if (p.M == 1) run_few<T, 1>(p, e, cus, s); \
    else if (p.M == 2) run_few<T, 2>(p, e, cus, s); \
    else if (p.M <= 4) run_few<T, 4>(p, e, cus, s); \
    else run_few<T, 8>(p, e, cus, s);          \
  } while (0)
  if (dtype == 0) FS_FEW(float);
  else FS_FEW(bf16_t);
#undef FS_FEW
}

}  // namespace fs
