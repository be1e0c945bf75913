// Layer norm (or, uncentred, root-mean-square norm) of rows, fused with the
// deferred residual add before it, and its backward pass.
//
//   s = round(x + add);  mean = sum(s) / d;  var = sum((s - mean)^2) / d;
//   rstd = 1 / sqrt(var + eps);  y = (s - mean) * rstd * gamma + beta
//   (uncentred: mean = 0)
//   h = (s - mean) * rstd;  u = gamma * dy;
//   dx = dres + rstd * (u - mean(u) - h * mean(u * h))   (uncentred: no mean(u))
//   dgamma = sum over rows of dy * h;  dbeta = sum over rows of dy
//
// Both are bound by memory.  A row stays in the registers of its TPR threads
// (NC chunks of 8 columns each) from the load to the store, so every input is
// read once; the variance is a second sum over the registers, of squares of
// differences, which loses no digits to a large mean.

#include "internal.hpp"
#include "saved.hpp"

namespace fs {
namespace {

// Sum over the TPR threads of a row; `red` holds one float per wave, and two
// calls that follow each other use different ones.
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* red) {
  v = wave_sum(v);
  if constexpr (TPR > 64) {
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < TPR / 64; ++w) v += red[w];
  }
  return v;
}

constexpr int threads_of(int tpr) { return tpr < 256 ? 256 : tpr; }

template <typename T, int TPR, int NC>
__global__ __launch_bounds__(threads_of(TPR)) void norm_kernel(NormArgs a) {
  constexpr int RPB = threads_of(TPR) / TPR;
  __shared__ float red[2][TPR / 64];
  const int tid = threadIdx.x % TPR;
  const int64_t r = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
  if (r >= a.rows) return;   // a whole wave; with more waves per row, none
  const T* x = (const T*)a.x + r * a.ldx;
  const T* add = (const T*)a.add + r * a.ldadd;
  float v[NC][8];
  float s = 0.f;
#pragma unroll
  for (int j = 0; j < NC; ++j) {
    const int c = (j * TPR + tid) * 8, n = min(8, a.cols - c);
    Raw8<T> q = {}, p = {};
    if (n > 0) q = load8<T>(x + c, n);
    if (a.add && n > 0) p = load8<T>(add + c, n);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[j][i] = a.add ? rounded<T>(q.get(i) + p.get(i)) : q.get(i);
#pragma unroll
    for (int i = 0; i < 8; ++i) s += v[j][i];   // 0 past the row's end
  }
  const float inv_d = 1.0f / (float)a.cols;
  const float mean = a.center ? row_sum<TPR>(s, red[0]) * inv_d : 0.f;
  float q = 0.f;
#pragma unroll
  for (int j = 0; j < NC; ++j) {
    const int n = a.cols - (j * TPR + tid) * 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float t = v[j][i] - mean;
      q += i < n ? t * t : 0.f;
    }
  }
  const float rstd = 1.0f / sqrtf(row_sum<TPR>(q, red[1]) * inv_d + a.eps);
  if (tid == 0) {
    if (a.mean) a.mean[r] = mean;
    if (a.rstd) a.rstd[r] = rstd;
  }
#pragma unroll
  for (int j = 0; j < NC; ++j) {
    const int c = (j * TPR + tid) * 8, n = min(8, a.cols - c);
    if (a.sum && n > 0) store8<T>((T*)a.sum + r * a.ldsum + c, v[j], n);
    if (a.in_codes) ckpt_store8<LANES_NEXT>(a.in_codes, a.in_scales, r, c, a.cols, v[j], n, true);
    float y[8] = {};
    if (n > 0) {
      Raw8<float> g = {}, b = {};
      if (a.gamma) g = load8<float>(a.gamma + c, n);
      if (a.beta) b = load8<float>(a.beta + c, n);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float t = (v[j][i] - mean) * rstd;
        if (a.gamma) t *= g.get(i);
        if (a.beta) t += b.get(i);
        y[i] = i < n ? rounded<T>(t) : 0.f;
      }
      store8<T>((T*)a.y + r * a.ldy + c, y, n);
    }
    if (a.y_codes) ckpt_store8<LANES_NEXT>(a.y_codes, a.y_scales, r, c, a.cols, y, n, true);
  }
}

// One group of TPR threads takes rows g, g + groups, ..; each thread keeps its
// columns' part of dgamma and dbeta in registers and writes it once at the
// end, part[0][group][cols] and part[1][group][cols], which colsum_kernel adds
// in group order.
template <typename T, int TPR, int NC, bool CODES>
__global__ __launch_bounds__(threads_of(TPR)) void norm_backward_kernel(NormBackArgs a) {
  constexpr int RPB = threads_of(TPR) / TPR, NW = TPR / 64;
  __shared__ float red[2][2][NW];
  const int tid = threadIdx.x % TPR, wave = (threadIdx.x % TPR) >> 6;
  const int64_t group = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
  const int64_t groups = (int64_t)gridDim.x * RPB;
  const int nb = (a.cols + kCkptBlock - 1) / kCkptBlock;
  const float inv_d = 1.0f / (float)a.cols;
  float dg[NC][8] = {}, db[NC][8] = {};
  Raw8<T> xr[NC], yr[NC], rr[NC];
  uint2 xc[NC];
  int xb[NC];
  float nmean = 0.f, nrstd = 0.f;
  auto load = [&](int64_t r) {
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      const int c = (j * TPR + tid) * 8, n = min(8, a.cols - c);
      xr[j] = {}, yr[j] = {}, rr[j] = {};
      xc[j] = make_uint2(0, 0);
      xb[j] = 127;
      if (n <= 0) continue;
      if constexpr (CODES) {
        xc[j] = load_codes(a.x_codes + r * a.cols + c, n);
        xb[j] = a.x_scales[r * nb + c / kCkptBlock];
      } else {
        xr[j] = load8<T>((const T*)a.x + r * a.ldx + c, n);
      }
      yr[j] = load8<T>((const T*)a.dy + r * a.lddy + c, n);
      if (a.dres) rr[j] = load8<T>((const T*)a.dres + r * a.lddres + c, n);
    }
    nmean = a.mean ? a.mean[r] : 0.f;
    nrstd = a.rstd[r];
  };
  if (group < a.rows) load(group);
  int par = 0;
  for (int64_t r = group; r < a.rows; r += groups, par ^= 1) {
    const float mean = nmean, rstd = nrstd;
    float h[NC][8], u[NC][8];
    Raw8<T> res[NC];
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      const int c = (j * TPR + tid) * 8, n = min(8, a.cols - c);
      float x[8];
      if constexpr (CODES) {
        ckpt_values(xc[j], xb[j], x);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = xr[j].get(i);
      }
      Raw8<float> g = {};
      if (a.gamma && n > 0) g = load8<float>(a.gamma + c, n);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const bool in = i < n;
        const float dy = yr[j].get(i);   // 0 past the row's end
        h[j][i] = in ? (x[i] - mean) * rstd : 0.f;
        u[j][i] = a.gamma ? dy * g.get(i) : dy;
        dg[j][i] = fmaf(dy, h[j][i], dg[j][i]);
        db[j][i] += dy;
        s1 += u[j][i];
        s2 = fmaf(u[j][i], h[j][i], s2);
      }
      res[j] = rr[j];
    }
    if (r + groups < a.rows) load(r + groups);   // in flight during this row's sums
    s1 = wave_sum(s1);
    s2 = wave_sum(s2);
    if constexpr (TPR > 64) {
      if ((threadIdx.x & 63) == 0) red[par][0][wave] = s1, red[par][1][wave] = s2;
      __syncthreads();
      s1 = s2 = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) s1 += red[par][0][w], s2 += red[par][1][w];
    }
    const float m1 = a.center ? s1 * inv_d : 0.f, m2 = s2 * inv_d;
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      const int c = (j * TPR + tid) * 8, n = min(8, a.cols - c);
      if (n <= 0) continue;
      float o[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        o[i] = rstd * (u[j][i] - m1 - h[j][i] * m2);
        if (a.dres) o[i] += res[j].get(i);
      }
      store8<T>((T*)a.dx + r * a.lddx + c, o, n);
    }
  }
  if (a.part) {
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      const int c = (j * TPR + tid) * 8, n = min(8, a.cols - c);
      if (n <= 0) continue;
      float* p = a.part + group * a.cols + c;
      store8<float>(p, dg[j], n);
      store8<float>(p + groups * a.cols, db[j], n);
    }
  }
}

// out[c] = sum over p of part[p][c], in a fixed order: 32 slices of the P
// rows, each added in ascending order, then the slices in ascending order.
__global__ __launch_bounds__(1024) void colsum_kernel(const float* __restrict__ part, int P, int cols,
                                                      float* out0, float* out1) {
  __shared__ float sm[32][33];
  float* out = blockIdx.y ? out1 : out0;
  if (!out) return;
  const float* src = part + (size_t)blockIdx.y * P * cols;
  const int cl = threadIdx.x & 31, sl = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + cl;
  float s = 0.f;
  if (c < cols)
    for (int p = sl; p < P; p += 32) s += src[(size_t)p * cols + c];
  sm[sl][cl] = s;
  __syncthreads();
  if (sl == 0 && c < cols) {
    s = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) s += sm[i][cl];
    out[c] = s;
  }
}

// Threads per row and chunks per thread.  A wave per row up to 2048 columns
// (four rows to a workgroup, sums without a barrier), then the workgroup that
// holds the row in at most 4 chunks per thread.
template <typename F>
void with_shape(int cols, F&& f) {
  using std::integral_constant;
#define FS_NORM_SHAPE(TPR, NC) \
  if (cols <= TPR * NC * 8) return f(integral_constant<int, TPR>{}, integral_constant<int, NC>{})
  FS_NORM_SHAPE(64, 1);
  FS_NORM_SHAPE(64, 2);
  FS_NORM_SHAPE(64, 4);
  FS_NORM_SHAPE(256, 2);
  FS_NORM_SHAPE(256, 3);
  FS_NORM_SHAPE(256, 4);
  FS_NORM_SHAPE(1024, 2);
  FS_NORM_SHAPE(1024, 4);
#undef FS_NORM_SHAPE
}

constexpr int kNormGroups = 512;   // workgroups of the backward pass

// Groups (rows of partial sums) of the backward pass.
int64_t norm_groups(int64_t rows, int cols, int tpr) {
  (void)cols;
  const int rpb = threads_of(tpr) / tpr;
  const int64_t wg = cdiv64(rows, rpb);
  return (wg < kNormGroups ? wg : kNormGroups) * rpb;
}

}  // namespace

size_t norm_ws_bytes(int64_t rows, int cols) {
  int64_t g = 0;
  with_shape(cols, [&](auto tpr, auto) { g = norm_groups(rows, cols, tpr); });
  return (size_t)g * cols * 2 * sizeof(float);
}

hipError_t launch_norm(int dtype, const NormArgs& a, hipStream_t s) {
  with_shape(a.cols, [&](auto tpr, auto nc) {
    constexpr int TPR = decltype(tpr)::value, NC = decltype(nc)::value;
    const unsigned grid = (unsigned)cdiv64(a.rows, threads_of(TPR) / TPR);
    if (dtype == 0) launch_k(norm_kernel<float, TPR, NC>, grid, threads_of(TPR), 0, s, a);
    else launch_k(norm_kernel<bf16_t, TPR, NC>, grid, threads_of(TPR), 0, s, a);
  });
  return hipGetLastError();
}

hipError_t launch_norm_backward(int dtype, const NormBackArgs& a, float* dgamma, float* dbeta,
                                hipStream_t s) {
  int64_t groups = 0;
  with_shape(a.cols, [&](auto tpr, auto nc) {
    constexpr int TPR = decltype(tpr)::value, NC = decltype(nc)::value;
    groups = norm_groups(a.rows, a.cols, TPR);
    const unsigned grid = (unsigned)(groups / (threads_of(TPR) / TPR)), nt = threads_of(TPR);
    if (dtype == 0) {
      if (a.x_codes) launch_k(norm_backward_kernel<float, TPR, NC, true>, grid, nt, 0, s, a);
      else launch_k(norm_backward_kernel<float, TPR, NC, false>, grid, nt, 0, s, a);
    } else {
      if (a.x_codes) launch_k(norm_backward_kernel<bf16_t, TPR, NC, true>, grid, nt, 0, s, a);
      else launch_k(norm_backward_kernel<bf16_t, TPR, NC, false>, grid, nt, 0, s, a);
    }
  });
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.part) return e;
  return launch_colsum(a.part, (int)groups, a.cols, dgamma, dbeta, s);
}

hipError_t launch_colsum(const float* part, int P, int cols, float* out0, float* out1, hipStream_t s) {
  launch_k(colsum_kernel, dim3((unsigned)cdiv64(cols, 32), out1 ? 2 : 1), 1024, 0, s, part, P, cols,
           out0, out1);
  return hipGetLastError();
}

}  // namespace fs
