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

// What the backward pass does before its products, in one launch.
//   the first `blocks` workgroups: dz = round(dout * act'(z)) (when dz is given:
//     [m, ld8], columns past n are 0) and the column sums of 8 R rows of it before
//     the rounding (when part is given: [m / (8 R) rounded up][n]); 32 threads of 8
//     columns by 8 rows
//   the others: 64 rows x 256 columns each of a, restored from its checkpoint
template <typename T>
struct PrepArgs {
  const T* dout;
  int64_t ldo;
  int m, n, act;
  const T* z;
  int64_t ldz;
  const uint8_t *codes, *scales;
  T* dz;
  int64_t ld8;
  float* part;
  unsigned blocks;
  const uint8_t *a_codes, *a_scales;
  T* a;
  int64_t lda;
  int k;
};
template <typename T, int R>
__global__ __launch_bounds__(256) void prepare_kernel(PrepArgs<T> q) {
  __shared__ float sm[8][256 + 4];
  const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
  if (blockIdx.x >= q.blocks) {
    const unsigned id = blockIdx.x - q.blocks;
    const int panels = (q.k + 255) / 256, c = (int)(id % panels) * 256 + tx * 8, nv = min(8, q.k - c);
    const int64_t r0 = (int64_t)(id / panels) * 64 + ty;
    if (nv > 0)
#pragma unroll 4
      for (int i = 0; i < 8; ++i) {
        const int64_t r = r0 + 8 * i;
        if (r >= q.m) break;
        float v[8];
        saved_load8<T>(nullptr, 0, q.a_codes, q.a_scales, r, c, q.k, nv, v);
        store8<T>(q.a + r * q.lda + c, v, nv);
      }
    return;
  }
  const int m = q.m, n = q.n;
  const int panels = (n + 255) / 256, panel = (int)(blockIdx.x % panels);
  const int64_t rb = blockIdx.x / panels;
  const int c = panel * 256 + tx * 8, nv = min(8, n - c);
  float sum[8] = {};
  if (nv > 0) {
#pragma unroll 4
    for (int i = 0; i < R; ++i) {
      const int64_t r = rb * 8 * R + 8 * i + ty;
      if (r >= m) break;
      const Raw8<T> d = load8<T>(q.dout + r * q.ldo + c, nv);
      float g[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) g[j] = d.get(j);
      if (q.act != ACT_NONE) {
        float x[8];
        saved_load8<T>(q.z, q.ldz, q.codes, q.scales, r, c, n, nv, x);
        act_slope8<T>(q.act, x);
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] = j < nv ? g[j] * x[j] : 0.f;
      }
      if (q.dz) store8<T>(q.dz + r * q.ld8 + c, g, 8);
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[j] += g[j];
    }
  }
  if (!q.part) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) sm[ty][tx * 8 + j] = sum[j];
  __syncthreads();
  const int col = panel * 256 + threadIdx.x;
  if (col < n) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += sm[i][threadIdx.x];
    q.part[(size_t)rb * n + col] = s;
  }
}

// Rows of a workgroup of prepare_kernel: 64, fewer while that leaves less than
// two workgroups per CU (512 x 1408 fp32: 48 workgroups took 10.8 us, 384
// 6.1 us).
int act_grad_rows(int m, int n) {
  // (up to 128 rows one part, the gradient itself: no launch to add parts, and a
  // restored in the same launch: 15.0 -> 12.8 us for 9 rows, whole pass)
  if (m <= 128) return m <= 64 ? 64 : 128;
  int rows = 64;
  while (rows > 8 && cdiv64(m, rows) * cdiv64(n, 256) < 2 * compute_units()) rows /= 2;
  return rows;
}

int pad8(int n) { return (n + 7) / 8 * 8; }

size_t product_ws_bytes(int dtype, bool a_along, bool b_along, int M, int N, int K) {
  return product_ws(dtype == 1, a_along, b_along, M, N, K, compute_units());
}

// The product's plan; operands that need it are first copied to whole chunks.
ProductPlan plan_product(int dtype, Product& p, hipStream_t s) {
  const int cus = compute_units();
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
  return product_plan(dtype == 1, ok, p.a_along, p.b_along, p.M, p.N, p.K, cus);
}

bool is_any(const ProductPlan& plan) { return plan.height == 0 && plan.mid == MID_NONE; }

hipError_t run_plan(int dtype, const Product& p, const Epilogue& e, const ProductPlan& plan, void* ws,
                    hipStream_t s) {
  const int np = pad8(p.N);
  float* part = plan.slices > 1 ? (float*)ws : nullptr;
  if (plan.height) {
    const TileGrid g{(int)cdiv64(p.M, plan.height), (int)cdiv64(p.N, plan.width), plan.slices, plan.per, part, np};
    (p.a_along ? p.b_along ? launch_tile_forward : launch_tile_da : launch_tile_dw)(
        p, e, g, plan.height / 32, compute_units(), s);
  } else if (plan.mid) {
    launch_mid(dtype, p, e, plan.mid, s);
  } else {
    launch_any(dtype, p, e, plan.slices, plan.per, part, np, s);
  }
  if (part) launch_reduce(dtype, part, plan.slices, p.M, p.N, np, e, s);
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
  Product p{a, lda, true, false, w, ldw, true, false, m, n, k,
            sp.packs ? base : nullptr, sp.packs ? base + sp.w : nullptr};
  const Epilogue e{o.bias, o.res, o.ldr, o.out, o.ldo, o.z, o.ldz, o.z_codes, o.z_scales,
                   o.out_codes, o.out_scales, o.act};
  // (the few-token kernel has no checkpoints: a block's columns lie in many waves)
  if (m <= kFewTokens && !e.z_codes && !e.out_codes) {
    launch_few(dtype, p, e, compute_units(), s);
    return hipGetLastError();
  }
  const ProductPlan plan = plan_product(dtype, p, s);
  return run_plan(dtype, p, e, plan, base + sp.prod, s);
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
  const bool restored = b.dw && b.a_codes && b.m > 0;
  const void* a = restored ? base + sp.a : b.a;
  const int64_t lda = restored ? pad8(b.k) : b.lda;
  hipError_t err = hipSuccess;
  if (b.m > 0 && (need_dz || part)) {
    void* dst = need_dz ? base + sp.dz : nullptr;
    const int64_t ld8 = pad8(b.n);
    const unsigned blocks = (unsigned)(cdiv64(b.n, 256) * cdiv64(b.m, rows));
    const unsigned more = restored ? (unsigned)(cdiv64(b.k, 256) * cdiv64(b.m, 64)) : 0;
    float* sums = one_part ? b.dbias : part;
    auto run = [&](auto type, auto r) {
      using T = decltype(type);
      const PrepArgs<T> q{(const T*)b.dout, b.ldo, b.m, b.n, b.act, (const T*)b.z, b.ldz, b.z_codes, b.z_scales,
                          (T*)dst, ld8, sums, blocks, b.a_codes, b.a_scales, (T*)(base + sp.a), lda, b.k};
      launch_k(prepare_kernel<T, decltype(r)::value>, blocks + more, 256, 0, s, q);
    };
    auto with_rows = [&](auto type) {
      switch (rows) {
        case 8: run(type, std::integral_constant<int, 1>{}); break;
        case 16: run(type, std::integral_constant<int, 2>{}); break;
        case 32: run(type, std::integral_constant<int, 4>{}); break;
        case 64: run(type, std::integral_constant<int, 8>{}); break;
        default: run(type, std::integral_constant<int, 16>{}); break;
      }
    };
    if (dtype == 0) with_rows(float{});
    else with_rows(bf16_t{});
    err = hipGetLastError();
    if (need_dz) dz = dst, lddz = ld8, padded = true;
  } else if (restored) {
    err = launch_restore(dtype, b.a_codes, b.a_scales, b.m, b.k, base + sp.a, lda, s);
  }
  if (err != hipSuccess) return err;
  // (no rows: the sums of no parts, 0)
  if (part && (b.m == 0 || !one_part)) {
    err = launch_colsum(part, (int)cdiv64(b.m, rows), b.n, b.dbias, nullptr, s);
    if (err != hipSuccess) return err;
  }
  Epilogue eda{}, edw{};
  eda.out = b.da, eda.ldo = b.ldda;
  edw.out = b.dw, edw.ldo = b.lddw;
  const bool odd_k = b.k % 8 != 0;
  Product da{dz, lddz, true, padded, b.w, b.ldw, false, false, b.m, b.k, b.n, nullptr,
             sp.packs_da && odd_k ? base + sp.w : nullptr};
  // (the columns behind a's last are not zeros when restored, but only reach
  // columns of dw that are not stored)
  Product dw{dz, lddz, false, padded, a, lda, false, restored, b.n, b.k, b.m, nullptr,
             sp.packs_dw && odd_k && !restored ? base + sp.a : nullptr};
  ProductPlan pda{}, pdw{};
  const bool run_da = b.da && b.m > 0;
  if (run_da) pda = plan_product(dtype, da, s);
  if (b.dw) pdw = plan_product(dtype, dw, s);
  // (of few tiles one launch for both, 23 -> 15 us with 9 rows; of many tiles each
  // product fills the chip by itself)
  const int64_t tiles = (cdiv64(b.m, 64) + cdiv64(b.n, 64)) * cdiv64(b.k, 64);
  if (run_da && b.dw && is_any(pda) && is_any(pdw) && pda.slices == 1 && pdw.slices == 1 &&
      tiles <= 8 * compute_units()) {
    launch_any_pair(dtype, da, eda, dw, edw, s);
    return hipGetLastError();
  }
  if (run_da) {
    err = run_plan(dtype, da, eda, pda, base + sp.prod, s);
    if (err != hipSuccess) return err;
  }
  return b.dw ? run_plan(dtype, dw, edw, pdw, base + sp.prod, s) : hipSuccess;
}

}  // namespace fs
