// 8-bit checkpoints of activations: rows to codes and scale bytes, and back
// (the format is in saved.hpp).  Both are one pass over memory: a thread
// holds 8 columns, the four threads of a 32-column block take its amax with
// two lane exchanges, and every load and store is 16 or 8 bytes.

#include "internal.hpp"
#include "saved.hpp"

namespace fs {
namespace {

// Threads: tx chunks of 8 columns (a power of two, at least 4) by 256 / tx
// rows; chunks past the row's end only take part in the exchange.
template <typename T, bool RESTORE>
__global__ __launch_bounds__(256) void checkpoint_kernel(T* __restrict__ x, int64_t ld, int64_t rows,
                                                         int cols, uint8_t* __restrict__ codes,
                                                         uint8_t* __restrict__ scales, int tx_log2) {
  const int tx = 1 << tx_log2;
  const int c = ((int)blockIdx.x * tx + (threadIdx.x & (tx - 1))) * 8;
  const int n = min(8, cols - c);
  const int ty = threadIdx.x >> tx_log2, rpb = 256 >> tx_log2;
  for (int64_t r0 = (int64_t)blockIdx.y * rpb; r0 < rows; r0 += (int64_t)gridDim.y * rpb) {
    const int64_t r = r0 + ty;
    const bool live = r < rows && n > 0;
    float v[8];
    if constexpr (RESTORE) {
      if (live) {
        saved_load8<T>(nullptr, 0, codes, scales, r, c, cols, n, v);
        store8<T>(x + r * ld + c, v, n);
      }
    } else {
      Raw8<T> a = {};
      if (live) a = load8<T>(x + r * ld + c, n);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = a.get(i);
      ckpt_store8<LANES_NEXT>(codes, scales, r, c, cols, v, n, live);
    }
  }
}

template <typename T, bool RESTORE>
hipError_t run(T* x, int64_t ld, int64_t rows, int cols, uint8_t* codes, uint8_t* scales,
               hipStream_t s) {
  const int chunks = (cols + kCkptBlock - 1) / kCkptBlock * 4;
  int lg = 2;
  while (lg < 8 && (1 << lg) < chunks) ++lg;
  const int64_t by = cdiv64(rows, 256 >> lg);
  const dim3 grid((unsigned)cdiv64(chunks, 1 << lg), (unsigned)(by < 65535 ? by : 65535));
  launch_k(checkpoint_kernel<T, RESTORE>, grid, 256, 0, s, x, ld, rows, cols, codes, scales, lg);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_checkpoint(int dtype, const void* x, int64_t ld, int64_t rows, int cols,
                             uint8_t* codes, uint8_t* scales, hipStream_t s) {
  if (dtype == 0) return run<float, false>((float*)x, ld, rows, cols, codes, scales, s);
  return run<bf16_t, false>((bf16_t*)x, ld, rows, cols, codes, scales, s);
}

hipError_t launch_restore(int dtype, const uint8_t* codes, const uint8_t* scales, int64_t rows,
                          int cols, void* x, int64_t ld, hipStream_t s) {
  if (dtype == 0)
    return run<float, true>((float*)x, ld, rows, cols, (uint8_t*)codes, (uint8_t*)scales, s);
  return run<bf16_t, true>((bf16_t*)x, ld, rows, cols, (uint8_t*)codes, (uint8_t*)scales, s);
}

}  // namespace fs
