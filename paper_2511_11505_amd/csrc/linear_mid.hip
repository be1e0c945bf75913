// Forward products with too few tiles for the large ones: tiles of 16 MF tokens
// x 16 NF outputs, whose waves split K among them.
//
// Such a product is bound by latency, or by one read of the weight from
// memory.  Each wave takes a K range and loads its operands from memory
// straight into the MFMA's registers (a load is 16 rows x 64 bytes), two steps
// ahead, so that nothing waits for a barrier until the waves add their
// accumulators through LDS; then the waves share out the epilogue.  Any
// alignment, stride and size: the loads take any address, and the last step of
// K is masked.

#include "linear.hpp"
#include "linear_rules.hpp"

namespace fs {
namespace {

template <typename T, int MF, int NF, int NW>
__global__ __launch_bounds__(64 * NW) void linear_mid_kernel(Product p, Epilogue e, int kper) {
  constexpr int V = 16 / sizeof(T), STEP = 4 * V, F = MF * NF;
  __shared__ __align__(16) floatx4 sums[NW][F][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
  const int tiles_n = (p.N + 16 * NF - 1) / (16 * NF);
  const int n0 = (int)(blockIdx.x % tiles_n) * 16 * NF, m0 = (int)(blockIdx.x / tiles_n) * 16 * MF;
  const int k0 = wave * kper, k1 = min(p.K, k0 + kper);
  const T *a[MF], *b[NF];
#pragma unroll
  for (int i = 0; i < MF; ++i) a[i] = (const T*)p.A + (int64_t)min(m0 + 16 * i + r, p.M - 1) * p.lda + g * V;
#pragma unroll
  for (int i = 0; i < NF; ++i) b[i] = (const T*)p.B + (int64_t)min(n0 + 16 * i + r, p.N - 1) * p.ldb + g * V;
  floatx4 acc[MF][NF] = {};
  uint4 fa[2][MF], fb[2][NF];
  auto load = [&](int buf, int k) __attribute__((always_inline)) {
    if (k + STEP <= k1) {   // (uniform)
#pragma unroll
      for (int i = 0; i < NF; ++i) fb[buf][i] = load16<T>(b[i] + k, V);
#pragma unroll
      for (int i = 0; i < MF; ++i) fa[buf][i] = load16<T>(a[i] + k, V);
    } else {
      const int n = k1 - k - g * V;
#pragma unroll
      for (int i = 0; i < NF; ++i) fb[buf][i] = n > 0 ? load16<T>(b[i] + k, n) : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < MF; ++i) fa[buf][i] = n > 0 ? load16<T>(a[i] + k, n) : make_uint4(0, 0, 0, 0);
    }
  };
  load(0, k0);
  load(1, k0 + STEP);
  for (int k = k0; k < k1; k += 2 * STEP) {
    mma_step<T>(fa[0], fb[0], acc);
    load(0, k + 2 * STEP);
    mma_step<T>(fa[1], fb[1], acc);
    load(1, k + 3 * STEP);
  }
#pragma unroll
  for (int i = 0; i < F; ++i) sums[wave][i][lane] = acc[i / NF][i % NF];
  __syncthreads();
#pragma unroll
  for (int q = 0; q < F / 2; q += NW) {
    const int pair = q + wave;
    if (pair >= F / 2) break;
    const int i = pair / (NF / 2), j = pair % (NF / 2) * 2;
    floatx4 x = sums[0][i * NF + j][lane], y = sums[0][i * NF + j + 1][lane];
#pragma unroll
    for (int w = 1; w < NW; ++w) {
      x += sums[w][i * NF + j][lane];
      y += sums[w][i * NF + j + 1][lane];
    }
    float v[8];
    join8(x, y, v);
    const int64_t row = m0 + 16 * i + r;
    const int c = n0 + 16 * j + col8(lane);
    epilogue8<T, LANES_APART>(e, p.M, p.N, row, c, v, epilogue_bias(e, p.N, c),
                              epilogue_res<T>(e, p.M, p.N, row, c));
  }
}

template <typename T, int MF, int NF, int NW>
void run_mid(const Product& p, const Epilogue& e, hipStream_t s) {
  const int step = 64 / (int)sizeof(T);
  const int kper = (int)(cdiv64(cdiv64(p.K, NW), step) * step);
  const int64_t tiles = cdiv64(p.M, 16 * MF) * cdiv64(p.N, 16 * NF);
  launch_k(linear_mid_kernel<T, MF, NF, NW>, (unsigned)tiles, 64 * NW, 0, s, p, e, kper);
}

}  // namespace

void launch_mid(int dtype, const Product& p, const Epilogue& e, int shape, hipStream_t s) {
#define FS_MID(T)                                             \
  do {                                                        \
    if (shape == MID_16) run_mid<T, 1, 2, 8>(p, e, s);        \
    else if (shape == MID_32) run_mid<T, 2, 2, 8>(p, e, s);   \
    else run_mid<T, 4, 2, 8>(p, e, s);                        \
  } while (0)
  if (dtype == 0) FS_MID(float);
  else FS_MID(bf16_t);
#undef FS_MID
}

}  // namespace fs
