// The linear with its epilogue and its backward pass.
//
//   z = a w^T + bias;  out = act(z) + residual
//   dz = round(dout * act'(z));  da = dz w;  dw = dz^T a
//   dbias = column sums of dout * act'(z), before the rounding
//
// The three products differ in which way their operands lie (linear.hpp):
// forward along/along, da along/across, dw across/across.

#include <algorithm>
#include <type_traits>

#include "linear.hpp"
#include "linear_rules.hpp"

namespace fs {
namespace {

typedef __attribute__((address_space(3))) short lds_i16;
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
  // 16 rows from r0 of the step's K (32 for bf16, 16 for fp32): lane l row
  // l % 16; bf16: k 8 (l / 16) .. + 7; fp32: k 4 (l / 16) .. + 3
  static __device__ __forceinline__ uint4 frag(const unsigned char* lds, int r0, int step) {
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    if constexpr (ALONG) {
      return *reinterpret_cast<const uint4*>(lds + (r0 + r) * STRIDE + step * 64 + g * 16);
    } else if constexpr (sizeof(T) == 4) {
      uint4 f;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        (&f.x)[i] = *reinterpret_cast<const uint32_t*>(lds + (step * 16 + 4 * g + i) * STRIDE + (r0 + r) * 4);
      return f;
    } else {
      // a transposing read: in each 16-lane group lane p gives the address
      // of 4 elements of row p / 4, columns 4 (p % 4) .., and gets the 4 rows
      // of column p
      const unsigned char* p = lds + (step * 32 + 8 * g + (r >> 2)) * STRIDE + (r0 + 4 * (r & 3)) * 2;
      const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)p);
      const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(p + 4 * STRIDE));
      const uint2 a = __builtin_bit_cast(uint2, lo), b = __builtin_bit_cast(uint2, hi);
      return make_uint4(a.x, a.y, b.x, b.y);
    }
  }
};

// 64 x 64 tiles, four waves of 32 x 32, staged through registers: any type,
// alignment, stride and size.  Grid (tiles, K slices); with more than one
// slice the fp32 sums go to part[slice][M][np].
template <typename T, bool LA, bool LB>
__global__ __launch_bounds__(256) void linear_any_kernel(Product p, Epilogue e, int kper,
                                                         float* __restrict__ part, int np) {
  using PA = Panel<T, LA>;
  using PB = Panel<T, LB>;
  constexpr int BK = 128 / sizeof(T);
  __shared__ __align__(16) unsigned char sa[2][PA::BYTES], sb[2][PB::BYTES];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wm = (wave >> 1) * 32, wn = (wave & 1) * 32;
  const int tiles_n = (p.N + 63) / 64;
  const int n0 = (int)(blockIdx.x % tiles_n) * 64, m0 = (int)(blockIdx.x / tiles_n) * 64;
  const int k0 = blockIdx.y * kper, kend = min(p.K, k0 + kper);
  const T *A = (const T*)p.A, *B = (const T*)p.B;
  floatx4 acc[2][2] = {};
  // blocks go through registers two ahead: the loads of block i + 2 are sent
  // out when block i is in LDS (with one ahead, a block of one workgroup per CU
  // took a load's whole latency)
  uint4 ra[2][2], rb[2][2];
  PA pa;
  PB pb;
  pa.init(A, p.lda, m0, p.M, k0);
  pb.init(B, p.ldb, n0, p.N, k0);
  auto fetch = [&](int i, int kb) __attribute__((always_inline)) {
    if (kb < kend) {
      pa.fetch(kend - kb, ra[i]);
      pb.fetch(kend - kb, rb[i]);
    }
  };
  auto block = [&](int i, int kb) __attribute__((always_inline)) {
    PA::put(sa[i], ra[i]);
    PB::put(sb[i], rb[i]);
    __syncthreads();
    fetch(i, kb + 2 * BK);
#pragma unroll
    for (int step = 0; step < 2; ++step) {
      uint4 fa[2], fb[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        fa[j] = PA::frag(sa[i], wm + 16 * j, step);
        fb[j] = PB::frag(sb[i], wn + 16 * j, step);
      }
      mma_step<T>(fa, fb, acc);
    }
  };
  fetch(0, k0);
  fetch(1, k0 + BK);
  for (int kb = k0; kb < kend; kb += 2 * BK) {
    block(0, kb);
    if (kb + BK < kend) block(1, kb + BK);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float v[8];
    join8(acc[i][0], acc[i][1], v);
    const int64_t r = m0 + wm + 16 * i + (lane & 15);
    const int c = n0 + wn + col8(lane);
    if (part) {
      if (r < p.M && c < p.N) store8<float>(part + ((int64_t)blockIdx.y * p.M + r) * np + c, v, 8);
    } else {
      epilogue8<T, LANES_APART>(e, p.M, p.N, r, c, v, epilogue_bias(e, p.N, c), epilogue_res<T>(e, p.M, p.N, r, c));
    }
  }
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

// Copies of up to two bf16 matrices with rows of whole 16-byte chunks, zeros
// behind the last element.  A thread copies a chunk.
struct PackArgs {
  const bf16_t* src[2];
  int64_t ld[2];
  bf16_t* dst[2];
  int rows[2], cols[2];
};
__global__ __launch_bounds__(256) void pack_rows_kernel(PackArgs a) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int ch = (a.cols[i] + 7) / 8;
    const int64_t total = (int64_t)a.rows[i] * ch;
    for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < total; q += (int64_t)gridDim.x * 256) {
      const int64_t r = q / ch;
      const int c = (int)(q - r * ch) * 8;
      st16(a.dst[i] + r * ch * 8 + c, load16<bf16_t>(a.src[i] + r * a.ld[i] + c, a.cols[i] - c));
    }
  }
}

// dz = round(dout * act'(z)) (when dz is given: [m, ldz8], columns past n are
// 0) and the column sums of 8 R rows of it before the rounding (when part is
// given: [m / (8 R) rounded up][n]).  32 threads of 8 columns by 8 rows.
template <typename T, int R>
__global__ __launch_bounds__(256) void act_grad_kernel(const T* __restrict__ dout, int64_t ldo, int m,
                                                       int n, int act, const T* __restrict__ z,
                                                       int64_t ldz, const uint8_t* __restrict__ codes,
                                                       const uint8_t* __restrict__ scales,
                                                       T* __restrict__ dz, int64_t ld8,
                                                       float* __restrict__ part) {
  __shared__ float sm[8][256 + 4];
  const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
  const int panels = (n + 255) / 256, panel = (int)(blockIdx.x % panels);
  const int64_t rb = blockIdx.x / panels;
  const int c = panel * 256 + tx * 8, nv = min(8, n - c);
  float sum[8] = {};
  if (nv > 0) {
#pragma unroll 4
    for (int i = 0; i < R; ++i) {
      const int64_t r = rb * 8 * R + 8 * i + ty;
      if (r >= m) break;
      const Raw8<T> d = load8<T>(dout + r * ldo + c, nv);
      float g[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) g[j] = d.get(j);
      if (act != ACT_NONE) {
        float x[8];
        saved_load8<T>(z, ldz, codes, scales, r, c, n, nv, x);
        act_slope8<T>(act, x);
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] = j < nv ? g[j] * x[j] : 0.f;
      }
      if (dz) store8<T>(dz + r * ld8 + c, g, 8);
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[j] += g[j];
    }
  }
  if (!part) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) sm[ty][tx * 8 + j] = sum[j];
  __syncthreads();
  const int col = panel * 256 + threadIdx.x;
  if (col < n) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += sm[i][threadIdx.x];
    part[(size_t)rb * n + col] = s;
  }
}

// Rows of a workgroup of act_grad_kernel: 64, fewer while that leaves less than
// two workgroups per CU (512 x 1408 fp32: 48 workgroups took 10.8 us, 384
// 6.1 us).
int act_grad_rows(int m, int n) {
  int rows = 64;
  while (rows > 8 && cdiv64(m, rows) * cdiv64(n, 256) < 2 * compute_units()) rows /= 2;
  return rows;
}

int pad8(int n) { return (n + 7) / 8 * 8; }

template <typename T>
void run_any(const Product& p, const Epilogue& e, const ProductPlan& plan, float* part, int np,
             hipStream_t s) {
  const dim3 grid((unsigned)(cdiv64(p.N, 64) * cdiv64(p.M, 64)), (unsigned)plan.slices);
  if (p.a_along && p.b_along)
    launch_k(linear_any_kernel<T, true, true>, grid, 256, 0, s, p, e, plan.per, part, np);
  else if (p.a_along)
    launch_k(linear_any_kernel<T, true, false>, grid, 256, 0, s, p, e, plan.per, part, np);
  else
    launch_k(linear_any_kernel<T, false, false>, grid, 256, 0, s, p, e, plan.per, part, np);
}

size_t product_ws_bytes(int dtype, bool a_along, bool b_along, int M, int N, int K) {
  return product_ws(dtype == 1, a_along, b_along, M, N, K, compute_units());
}

hipError_t run_product(int dtype, Product p, const Epilogue& e, void* ws, hipStream_t s) {
  const int cus = compute_units(), np = pad8(p.N);
  // (the few-token kernel has no checkpoints: a block's columns lie in many waves)
  if (p.a_along && p.b_along && p.M <= kFewTokens && !e.z_codes && !e.out_codes) {
    launch_few(dtype, p, e, cus, s);
    return hipGetLastError();
  }
  const bool ok_a = tile_operand((uintptr_t)p.A, p.lda, p.a_padded ? 0 : p.a_along ? p.K : p.M);
  const bool ok_b = tile_operand((uintptr_t)p.B, p.ldb, p.b_padded ? 0 : p.b_along ? p.K : p.N);
  bool ok = ok_a && ok_b;
  if (!ok && (ok_a || p.a_pack) && (ok_b || p.b_pack)) {
    PackArgs q{};
    if (!ok_a) {
      const int rows = p.a_along ? p.M : p.K, cols = p.a_along ? p.K : p.M;
      q.src[0] = (const bf16_t*)p.A, q.ld[0] = p.lda, q.dst[0] = (bf16_t*)p.a_pack;
      q.rows[0] = rows, q.cols[0] = cols;
      p.A = p.a_pack, p.lda = pad8(cols), p.a_padded = true;
    }
    if (!ok_b) {
      const int rows = p.b_along ? p.N : p.K, cols = p.b_along ? p.K : p.N;
      q.src[1] = (const bf16_t*)p.B, q.ld[1] = p.ldb, q.dst[1] = (bf16_t*)p.b_pack;
      q.rows[1] = rows, q.cols[1] = cols;
      p.B = p.b_pack, p.ldb = pad8(cols), p.b_padded = true;
    }
    const int64_t most = std::max((int64_t)q.rows[0] * pad8(q.cols[0]), (int64_t)q.rows[1] * pad8(q.cols[1])) / 8;
    launch_k(pack_rows_kernel, (unsigned)std::min<int64_t>(cdiv64(most, 256), 16 * cus), 256, 0, s, q);
    ok = p.lda <= (1 << 22) && p.ldb <= (1 << 22);
  }
  const ProductPlan plan = product_plan(dtype == 1, ok, p.a_along, p.b_along, p.M, p.N, p.K, cus);
  if (plan.mid && p.a_along && p.b_along) {
    launch_mid(dtype, p, e, plan.mid, s);
    return hipGetLastError();
  }
  float* part = plan.slices > 1 ? (float*)ws : nullptr;
  if (plan.height) {
    const TileGrid g{(int)cdiv64(p.M, plan.height), (int)cdiv64(p.N, plan.width), plan.slices, plan.per, part, np};
    TileLaunch* run = p.a_along ? p.b_along ? launch_tile_forward : launch_tile_da : launch_tile_dw;
    run(p, e, g, plan.height / 32, cus, s);
  } else if (dtype == 0) {
    run_any<float>(p, e, plan, part, np, s);
  } else {
    run_any<bf16_t>(p, e, plan, part, np, s);
  }
  if (part) {
    const int64_t chunks = (int64_t)p.M * ((p.N + 31) / 32 * 4);
    const unsigned grid = (unsigned)cdiv64(chunks, 256);
    if (dtype == 0)
      launch_k(linear_reduce_kernel<float>, grid, 256, 0, s, (const float*)part, plan.slices, p.M, p.N, np, e);
    else
      launch_k(linear_reduce_kernel<bf16_t>, grid, 256, 0, s, (const float*)part, plan.slices, p.M, p.N, np, e);
  }
  return hipGetLastError();
}

size_t up256(size_t b) { return (b + 255) / 256 * 256; }

size_t rows_bytes(int dtype, int64_t rows, int cols) {
  return up256((size_t)rows * pad8(cols) * (dtype == 0 ? 4 : 2));
}

// Workspace of the forward pass: copies of a and w, the product's K slices.
struct ForwardSpace {
  bool packs;
  size_t w, prod, bytes;
  ForwardSpace(int dtype, int m, int n, int k) {
    packs = m > kFewTokens && product_packs(dtype == 1, true, true, m, n, k, compute_units());
    w = packs ? rows_bytes(dtype, m, k) : 0;
    prod = w + (packs ? rows_bytes(dtype, n, k) : 0);
    bytes = prod + up256(product_ws_bytes(dtype, true, true, m, n, k));
  }
};

// Workspace of the backward pass: dz, or dout with whole chunks; the bias
// gradient's partial sums; a restored from its checkpoint, or with whole
// chunks; w with whole chunks; the products' K slices.
struct BackSpace {
  bool packs_da, packs_dw, keeps_dz;
  size_t dz, part, a, w, prod, bytes;
  BackSpace(int dtype, int act, int m, int n, int k) {
    const int cus = compute_units();
    packs_da = product_packs(dtype == 1, true, false, m, k, n, cus);
    packs_dw = product_packs(dtype == 1, false, false, n, k, m, cus);
    keeps_dz = act != ACT_NONE || (n % 8 != 0 && (packs_da || packs_dw));
    dz = 0;
    part = dz + (keeps_dz ? rows_bytes(dtype, m, n) : 0);
    a = part + up256((size_t)cdiv64(m, act_grad_rows(m, n)) * n * 4);
    w = a + rows_bytes(dtype, m, k);
    prod = w + (packs_da && k % 8 != 0 ? rows_bytes(dtype, n, k) : 0);
    bytes = prod + up256(std::max(product_ws_bytes(dtype, true, false, m, k, n),
                                  product_ws_bytes(dtype, false, false, n, k, m)));
  }
};

}  // namespace

size_t linear_ws_bytes(int dtype, int m, int n, int k) { return ForwardSpace(dtype, m, n, k).bytes; }

size_t linear_backward_ws_bytes(int dtype, int act, int m, int n, int k) {
  return BackSpace(dtype, act, m, n, k).bytes;
}

hipError_t launch_linear(int dtype, int m, int n, int k, const void* a, int64_t lda, const void* w,
                         int64_t ldw, const LinearOut& o, void* ws, hipStream_t s) {
  const ForwardSpace sp(dtype, m, n, k);
  char* base = static_cast<char*>(ws);
  const Product p{a, lda, true, false, w, ldw, true, false, m, n, k,
                  sp.packs ? base : nullptr, sp.packs ? base + sp.w : nullptr};
  const Epilogue e{o.bias, o.res, o.ldr, o.out, o.ldo, o.z, o.ldz, o.z_codes, o.z_scales,
                   o.out_codes, o.out_scales, o.act};
  return run_product(dtype, p, e, base + sp.prod, s);
}

hipError_t launch_linear_backward(int dtype, const LinearBack& b, void* ws, hipStream_t s) {
  const BackSpace sp(dtype, b.act, b.m, b.n, b.k);
  char* base = static_cast<char*>(ws);
  const void* dz = b.dout;
  int64_t lddz = b.ldo;
  bool padded = false;
  float* part = b.dbias ? (float*)(base + sp.part) : nullptr;
  const bool need_dz = sp.keeps_dz && (b.da || b.dw);
  // (with one part it is the gradient itself)
  const int rows = act_grad_rows(b.m, b.n);
  const bool one_part = b.m <= rows;
  if (b.m == 0) {
    // no rows: the weight's gradients are 0
    if (b.dbias) {
      const hipError_t err = launch_colsum(part, 0, b.n, b.dbias, nullptr, s);
      if (err != hipSuccess) return err;
    }
  } else if (need_dz || part) {
    const unsigned grid = (unsigned)(cdiv64(b.n, 256) * cdiv64(b.m, rows));
    void* dst = need_dz ? base + sp.dz : nullptr;
    const int64_t ld8 = pad8(b.n);
    float* sums = one_part ? b.dbias : part;
    auto run = [&](auto r) {
      constexpr int R = decltype(r)::value;
      if (dtype == 0)
        launch_k(act_grad_kernel<float, R>, grid, 256, 0, s, (const float*)b.dout, b.ldo, b.m, b.n, b.act,
                 (const float*)b.z, b.ldz, b.z_codes, b.z_scales, (float*)dst, ld8, sums);
      else
        launch_k(act_grad_kernel<bf16_t, R>, grid, 256, 0, s, (const bf16_t*)b.dout, b.ldo, b.m, b.n, b.act,
                 (const bf16_t*)b.z, b.ldz, b.z_codes, b.z_scales, (bf16_t*)dst, ld8, sums);
    };
    if (rows == 8) run(std::integral_constant<int, 1>{});
    else if (rows == 16) run(std::integral_constant<int, 2>{});
    else if (rows == 32) run(std::integral_constant<int, 4>{});
    else run(std::integral_constant<int, 8>{});
    hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    if (need_dz) dz = dst, lddz = ld8, padded = true;
    if (part && !one_part) {
      err = launch_colsum(part, (int)cdiv64(b.m, rows), b.n, b.dbias, nullptr, s);
      if (err != hipSuccess) return err;
    }
  }
  Epilogue e{};
  if (b.da && b.m > 0) {
    e.out = b.da;
    e.ldo = b.ldda;
    const Product p{dz, lddz, true, padded, b.w, b.ldw, false, false, b.m, b.k, b.n, nullptr,
                    sp.packs_da && b.k % 8 != 0 ? base + sp.w : nullptr};
    const hipError_t err = run_product(dtype, p, e, base + sp.prod, s);
    if (err != hipSuccess) return err;
  }
  if (b.dw) {
    const void* a = b.a;
    int64_t lda = b.lda;
    const bool restored = b.a_codes && b.m > 0;
    if (restored) {
      a = base + sp.a;
      lda = pad8(b.k);
      const hipError_t err =
          launch_restore(dtype, b.a_codes, b.a_scales, b.m, b.k, base + sp.a, lda, s);
      if (err != hipSuccess) return err;
    }
    e.out = b.dw;
    e.ldo = b.lddw;
    // (the columns behind a's last are not zeros here, but only reach columns
    // of dw that are not stored)
    const Product p{dz, lddz, false, padded, a, lda, false, restored, b.n, b.k, b.m, nullptr,
                    sp.packs_dw && b.k % 8 != 0 && !restored ? base + sp.a : nullptr};
    return run_product(dtype, p, e, base + sp.prod, s);
  }
  return hipSuccess;
}

}  // namespace fs
