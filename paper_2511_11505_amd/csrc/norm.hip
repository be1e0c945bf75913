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
// Both are bound by memory.  A row stays in registers from the load to the
// store, so every input is read once; the variance is a second sum over the
// registers, of squares of differences, which loses no digits to a large mean.
// A row of up to 1024 columns belongs to a wave (sums without a barrier, four
// rows to a workgroup), a longer one to a workgroup of as many threads as it
// has 8-column chunks, or half or a quarter of that (NC chunks per thread).
// Measured on bf16 (us; 256 threads with three or four chunks each before):
// forward of 8192 x 5120 with the add and an 8-bit copy, 379 MB, 91 -> 89 (a
// copy's rate, 5.1 TB/s, would take 74), 64 x 7168 7.5 -> 4.9, bound by latency;
// backward of 8192 x 5120 from its 8-bit input, 295 MB, 92 -> 70.

#include <algorithm>
#include <type_traits>

#include "internal.hpp"
#include "saved.hpp"

namespace fs {
namespace {

// Sums of N values over the threads of a row; `red` holds N floats per wave,
// and two calls that follow each other use different ones.
template <bool WAVE, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float (*red)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
  if constexpr (!WAVE) {
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) red[threadIdx.x >> 6][i] = v[i];
    __syncthreads();
    // lane w of 16 takes wave w's; a fixed tree over 16 lanes
    const int w = threadIdx.x & 15, nw = blockDim.x >> 6;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float x = w < nw ? red[w][i] : 0.f;
      x += dpp_f<kDppXor1>(x);
      x += dpp_f<kDppXor2>(x);
      x += dpp_f<kDppHalfMirror>(x);
      x += dpp_f<kDppMirror>(x);
      v[i] = x;
    }
  }
}

template <typename T, bool WAVE, int NC>
__global__ __launch_bounds__(WAVE ? 256 : 1024) void norm_kernel(NormArgs a) {
  __shared__ float red[2][16][1];
  const int tpr = WAVE ? 64 : blockDim.x, tid = WAVE ? threadIdx.x & 63 : threadIdx.x;
  const int64_t r = WAVE ? (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x;
  if (r >= a.rows) return;   // a whole wave of its own row
  const T* x = (const T*)a.x + r * a.ldx;
  const T* add = (const T*)a.add + r * a.ldadd;
  float v[NC][8];
  float s[1] = {0.f};
#pragma unroll
  for (int j = 0; j < NC; ++j) {
    const int c = (j * tpr + tid) * 8, n = min(8, a.cols - c);
    Raw8<T> q = {}, p = {};
    if (n > 0) q = load8<T>(x + c, n);
    if (a.add && n > 0) p = load8<T>(add + c, n);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[j][i] = a.add ? rounded<T>(q.get(i) + p.get(i)) : q.get(i);
#pragma unroll
    for (int i = 0; i < 8; ++i) s[0] += v[j][i];   // 0 past the row's end
  }
  const float inv_d = 1.0f / (float)a.cols;
  float mean = 0.f;
  if (a.center) {
    row_sums<WAVE>(s, red[0]);
    mean = s[0] * inv_d;
  }
  float q[1] = {0.f};
#pragma unroll
  for (int j = 0; j < NC; ++j) {
    const int n = a.cols - (j * tpr + tid) * 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float t = v[j][i] - mean;
      q[0] += i < n ? t * t : 0.f;
    }
  }
  row_sums<WAVE>(q, red[1]);
  const float rstd = 1.0f / sqrtf(q[0] * inv_d + a.eps);
  if (tid == 0) {
    if (a.mean) a.mean[r] = mean;
    if (a.rstd) a.rstd[r] = rstd;
  }
#pragma unroll
  for (int j = 0; j < NC; ++j) {
    const int c = (j * tpr + tid) * 8, n = min(8, a.cols - c);
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

// One group (a wave, or a workgroup) takes rows g, g + groups, ..; each thread
// keeps its columns' part of dgamma and dbeta in registers; at the end a workgroup
// writes them once, part[0][workgroup][cols] and part[1][workgroup][cols], which
// colsum_kernel adds in a fixed order.  The next row is in flight during a row's sums; h and u
// are computed twice rather than kept.
template <typename T, bool WAVE, int NC, bool CODES>
__global__ __launch_bounds__(WAVE ? 256 : 1024) void norm_backward_kernel(NormBackArgs a) {
  __shared__ float red[2][16][2];
  const int tpr = WAVE ? 64 : blockDim.x, tid = WAVE ? threadIdx.x & 63 : threadIdx.x;
  const int64_t group = WAVE ? (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x;
  const int64_t groups = (int64_t)gridDim.x * (WAVE ? 4 : 1);
  const int nb = (a.cols + kCkptBlock - 1) / kCkptBlock;
  const float inv_d = 1.0f / (float)a.cols;
  // More than a chunk per thread of a workgroup's row leaves no registers for a
  // row ahead and gamma, four not even for the row: the second pass loads it
  // again (2048 x 32768 in bf16, from rows: 331 us, where a copy's rate would take 79;
  // 4096 x 12288, two chunks, 82 of 59).
  constexpr bool AHEAD = WAVE || NC == 1, HOLD = WAVE || NC < 4;
  float dg[NC][8] = {}, db[NC][8] = {};
  struct Chunk {
    Raw8<T> x, dy, res;
    uint2 codes;
    int byte;
  };
  auto chunk = [&](int j, int64_t r) __attribute__((always_inline)) {
    const int c = (j * tpr + tid) * 8, n = min(8, a.cols - c);
    Chunk w = {};
    w.byte = 127;
    if (n > 0) {
      if constexpr (CODES) {
        w.codes = load_codes(a.x_codes + r * a.cols + c, n);
        w.byte = a.x_scales[r * nb + c / kCkptBlock];
      } else {
        w.x = load8<T>((const T*)a.x + r * a.ldx + c, n);
      }
      w.dy = load8<T>((const T*)a.dy + r * a.lddy + c, n);
      if (a.dres) w.res = load8<T>((const T*)a.dres + r * a.lddres + c, n);
    }
    return w;
  };
  auto load_gamma = [&](int j) __attribute__((always_inline)) {
    const int c = (j * tpr + tid) * 8, n = min(8, a.cols - c);
    Raw8<float> g;
#pragma unroll
    for (int i = 0; i < 8; ++i) g.w[i] = 0x3F800000u;
    if (a.gamma && n > 0) g = load8<float>(a.gamma + c, n);
    return g;
  };
  // h of a chunk, 0 past the row's end
  auto values = [&](const Chunk& w, int j, float mean, float rstd, float (&h)[8]) __attribute__((always_inline)) {
    const int n = a.cols - (j * tpr + tid) * 8;
    if constexpr (CODES) {
      ckpt_values(w.codes, w.byte, h);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) h[i] = w.x.get(i);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] = i < n ? (h[i] - mean) * rstd : 0.f;
  };
  Raw8<float> gamma[AHEAD ? NC : 1];
  Chunk row[HOLD ? NC : 1], next[AHEAD ? NC : 1];
  float nmean = 0.f, nrstd = 0.f;
  auto load_next = [&](int64_t r) __attribute__((always_inline)) {
    if constexpr (AHEAD) {
#pragma unroll
      for (int j = 0; j < NC; ++j) next[j] = chunk(j, r);
    }
    nmean = a.mean ? a.mean[r] : 0.f;
    nrstd = a.rstd[r];
  };
  if constexpr (AHEAD) {
#pragma unroll
    for (int j = 0; j < NC; ++j) gamma[j] = load_gamma(j);
  }
  if (group < a.rows) load_next(group);
  int par = 0;
  for (int64_t r = group; r < a.rows; r += groups, par ^= 1) {
    const float mean = nmean, rstd = nrstd;
    if constexpr (AHEAD) {
#pragma unroll
      for (int j = 0; j < NC; ++j) row[j] = next[j];
    }
    if (r + groups < a.rows) load_next(r + groups);
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      Chunk& w = row[HOLD ? j : 0];
      if constexpr (!AHEAD) w = chunk(j, r);
      const Raw8<float> g = AHEAD ? gamma[AHEAD ? j : 0] : load_gamma(j);
      float h[8];
      values(w, j, mean, rstd, h);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float dy = w.dy.get(i), u = dy * g.get(i);   // 0 past the row's end
        dg[j][i] = fmaf(dy, h[i], dg[j][i]);
        db[j][i] += dy;
        s[0] += u;
        s[1] = fmaf(u, h[i], s[1]);
      }
    }
    row_sums<WAVE>(s, red[par]);
    const float m1 = a.center ? s[0] * inv_d : 0.f, m2 = s[1] * inv_d;
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      const int c = (j * tpr + tid) * 8, n = min(8, a.cols - c);
      if (n <= 0) continue;
      Chunk& w = row[HOLD ? j : 0];
      if constexpr (!HOLD) w = chunk(j, r);
      const Raw8<float> g = AHEAD ? gamma[AHEAD ? j : 0] : load_gamma(j);
      float h[8], o[8];
      values(w, j, mean, rstd, h);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        o[i] = rstd * (w.dy.get(i) * g.get(i) - m1 - h[i] * m2);
        if (a.dres) o[i] += w.res.get(i);
      }
      store8<T>((T*)a.dx + r * a.lddx + c, o, n);
    }
  }
  if (a.part) {
    float* part = a.part + (int64_t)blockIdx.x * a.cols;
    if constexpr (WAVE) {
      // the four waves' sums, in wave order
      __shared__ float sm[4][NC * 512];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < NC; ++j)
#pragma unroll
          for (int i = 0; i < 8; ++i) sm[threadIdx.x >> 6][j * 512 + i * 64 + tid] = h ? db[j][i] : dg[j][i];
        __syncthreads();
        for (int q = threadIdx.x; q < NC * 512; q += 256) {
          // place q holds column 8 (64 j + lane) + i, q = 512 j + 64 i + lane
          const int c = 512 * (q / 512) + 8 * (q % 64) + q / 64 % 8;
          const float v = ((sm[0][q] + sm[1][q]) + sm[2][q]) + sm[3][q];
          if (c < a.cols) part[(int64_t)h * gridDim.x * a.cols + c] = v;
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < NC; ++j) {
        const int c = (j * tpr + tid) * 8, n = min(8, a.cols - c);
        if (n <= 0) continue;
        store8<float>(part + c, dg[j], n);
        store8<float>(part + (int64_t)gridDim.x * a.cols + c, db[j], n);
      }
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
  if (c < cols) {
    int p = sl;
    for (; p + 7 * 32 < P; p += 8 * 32) {   // eight loads in flight
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = src[(size_t)(p + 32 * i) * cols + c];
#pragma unroll
      for (int i = 0; i < 8; ++i) s += x[i];
    }
    for (; p < P; p += 32) s += src[(size_t)p * cols + c];
  }
  sm[sl][cl] = s;
  __syncthreads();
  if (sl == 0 && c < cols) {
    s = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) s += sm[i][cl];
    out[c] = s;
  }
}

// Calls f(wave per row?, chunks per thread) with the threads of a workgroup.
template <typename F>
void with_shape(int cols, F&& f) {
  using std::integral_constant;
  using Yes = std::true_type;
  using No = std::false_type;
  const int chunks = (cols + 7) / 8;
  auto threads = [&](int nc) { return (chunks + 64 * nc - 1) / (64 * nc) * 64; };
  if (chunks <= 64) f(Yes{}, integral_constant<int, 1>{}, 256);
  else if (chunks <= 128) f(Yes{}, integral_constant<int, 2>{}, 256);
  else if (chunks <= 1024) f(No{}, integral_constant<int, 1>{}, threads(1));
  else if (chunks <= 2048) f(No{}, integral_constant<int, 2>{}, threads(2));
  else f(No{}, integral_constant<int, 4>{}, threads(4));
}

// Workgroups of the backward pass: about 8 waves per CU, one workgroup at
// least.  More of them write more partial sums, 8 bytes per column each (us with
// 1, 2, 4, 8 workgroups per CU: 8192 x 5120, ten waves, 80, 84, 92, 109; 8192 x
// 2048, four waves, 46, 33, 35, 47).
int64_t norm_groups(int64_t rows, bool wave, int threads) {
  const int64_t wgs = wave ? cdiv64(rows, 4) : rows;
  const int64_t most = (int64_t)compute_units() * std::max(1, 8 * 64 / threads);
  return wgs < most ? wgs : most;
}

}  // namespace

size_t norm_ws_bytes(int64_t rows, int cols) {
  int64_t g = 0;
  with_shape(cols, [&](auto wave, auto, int threads) { g = norm_groups(rows, wave, threads); });
  return (size_t)g * cols * 2 * sizeof(float);
}

hipError_t launch_norm(int dtype, const NormArgs& a, hipStream_t s) {
  with_shape(a.cols, [&](auto wave, auto nc, int threads) {
    constexpr bool W = decltype(wave)::value;
    constexpr int NC = decltype(nc)::value;
    const unsigned grid = (unsigned)cdiv64(a.rows, W ? 4 : 1);
    if (dtype == 0) launch_k(norm_kernel<float, W, NC>, grid, threads, 0, s, a);
    else launch_k(norm_kernel<bf16_t, W, NC>, grid, threads, 0, s, a);
  });
  return hipGetLastError();
}

hipError_t launch_norm_backward(int dtype, const NormBackArgs& a, float* dgamma, float* dbeta,
                                hipStream_t s) {
  int64_t groups = 0;
  with_shape(a.cols, [&](auto wave, auto nc, int threads) {
    constexpr bool W = decltype(wave)::value;
    constexpr int NC = decltype(nc)::value;
    groups = norm_groups(a.rows, W, threads);
    const unsigned grid = (unsigned)groups;
    if (dtype == 0) {
      if (a.x_codes) launch_k(norm_backward_kernel<float, W, NC, true>, grid, threads, 0, s, a);
      else launch_k(norm_backward_kernel<float, W, NC, false>, grid, threads, 0, s, a);
    } else {
      if (a.x_codes) launch_k(norm_backward_kernel<bf16_t, W, NC, true>, grid, threads, 0, s, a);
      else launch_k(norm_backward_kernel<bf16_t, W, NC, false>, grid, threads, 0, s, a);
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
