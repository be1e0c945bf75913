// Saved activations: rows, or 8-bit checkpoints of rows.
//
// A checkpoint cuts each row into blocks of 32 columns (the last may be
// short).  A block holds E4M3 codes and one scale byte e + 127, where e is
// the least integer in [-117, 119] with amax <= 448 * 2^e (amax = max |x| over
// the block; 119 where there is none); code = E4M3(x * 2^-e), rounded to
// nearest, ties to even.  The scale is a power of two, so x * 2^-e is exact
// and at most 448, except that values above 448 * 2^119 (the last eighth of
// fp32's range) become 448.  code * 2^e has four significant bits, is at least
// 2^-126 in size and finite: the value read back is exact in fp32 and in bf16,
// and a matrix product of it has no rounding that the code did not make.  A block with an infinity or a
// NaN has byte 255 and codes 0x7F (E4M3 NaN) and reads back as NaN.
#pragma once

#include <string.h>

#include "common.hpp"

namespace fs {

constexpr int kCkptBlock = 32;
constexpr int kCkptMinExp = -117, kCkptMaxExp = 119;

namespace {

// ---- 8 consecutive elements of a row at any element alignment.  (The copies
// compile to 16-byte global loads and stores: the target takes them at any
// alignment.)
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(1)));

template <typename T>
struct Raw8 {
  uint32_t w[8 * sizeof(T) / 4];
  __device__ __forceinline__ float get(int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    else return __uint_as_float((i & 1) ? (w[i >> 1] & 0xFFFF0000u) : (w[i >> 1] << 16));
  }
};

template <typename T>
__device__ __forceinline__ Raw8<T> load8(const T* p, int n) {
  Raw8<T> r;
  if (n >= 8) {
#pragma unroll
    for (unsigned i = 0; i < sizeof(r.w) / 16; ++i) {
      const u32x4_any v = reinterpret_cast<const u32x4_any*>(p)[i];
      r.w[4 * i] = v[0], r.w[4 * i + 1] = v[1], r.w[4 * i + 2] = v[2], r.w[4 * i + 3] = v[3];
    }
  } else {
#pragma unroll
    for (unsigned i = 0; i < sizeof(r.w) / 4; ++i) r.w[i] = 0;
    // (an opaque offset: else the element loads of this branch are merged
    // into the vector load of the other, which falls apart)
    int z = 0;
    asm volatile("" : "+v"(z));
    p += z;
#pragma unroll
    for (int i = 0; i < 7; ++i)
      if (i < n) {
        if constexpr (sizeof(T) == 4) r.w[i] = __float_as_uint(p[i]);
        else r.w[i >> 1] |= (uint32_t)p[i] << (16 * (i & 1));
      }
  }
  return r;
}

// 16 bytes of a row at element p, the first n (of 16 / sizeof(T)) elements;
// the rest 0.
template <typename T>
__device__ __forceinline__ uint4 load16(const T* p, int n) {
  constexpr int V = 16 / sizeof(T);
  if (n >= V) {
    const u32x4_any v = *reinterpret_cast<const u32x4_any*>(p);
    return make_uint4(v[0], v[1], v[2], v[3]);
  }
  uint32_t w[4] = {0, 0, 0, 0};
  int z = 0;   // as in load8
  asm volatile("" : "+v"(z));
  p += z;
#pragma unroll
  for (int i = 0; i < V - 1; ++i)
    if (i < n) {
      if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(p[i]);
      else w[i >> 1] |= (uint32_t)p[i] << (16 * (i & 1));
    }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&v)[8], int n) {
  if (n >= 8) {
    T t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = from_f32<T>(v[i]);
    memcpy(p, t, sizeof(t));
  } else {
#pragma unroll
    for (int i = 0; i < 7; ++i)
      if (i < n) p[i] = from_f32<T>(v[i]);
  }
}

// v rounded to T and back
template <typename T>
__device__ __forceinline__ float rounded(float v) { return to_f32<T>(from_f32<T>(v)); }

// ---- checkpoint codes
// Scale byte of a block from the bits of its largest |x| (as integers NaN and
// infinity are the largest, so none is lost in the maximum).
__device__ __forceinline__ int ckpt_byte(uint32_t amax) {
  if (amax >= 0x7F800000u) return 255;
  const int e = (int)(amax >> 23) - 135 + ((amax & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return min(max(e, kCkptMinExp), kCkptMaxExp) + 127;
}
__device__ __forceinline__ uint32_t amax8(const float (&v)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
  return m;
}
// Codes of 8 values under scale byte b.
__device__ __forceinline__ uint2 ckpt_codes(const float (&v)[8], int b) {
  const float inv = __uint_as_float((uint32_t)(254 - min(b, 254)) << 23);
  float q[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) q[i] = v[i] * inv;
  if (b == kCkptMaxExp + 127) {
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = fminf(fmaxf(q[i], -448.f), 448.f);
  }
  int w0 = 0, w1 = 0;
  w0 = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], w0, false);
  w0 = __builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], w0, true);
  w1 = __builtin_amdgcn_cvt_pk_fp8_f32(q[4], q[5], w1, false);
  w1 = __builtin_amdgcn_cvt_pk_fp8_f32(q[6], q[7], w1, true);
  const bool nan = b == 255;
  return make_uint2(nan ? 0x7F7F7F7Fu : (uint32_t)w0, nan ? 0x7F7F7F7Fu : (uint32_t)w1);
}
__device__ __forceinline__ void store_codes(uint8_t* p, uint2 c, int n) {
  if (n >= 8) {
    memcpy(p, &c, 8);
  } else {
#pragma unroll
    for (int i = 0; i < 7; ++i)
      if (i < n) p[i] = (uint8_t)((i < 4 ? c.x : c.y) >> (8 * (i & 3)));
  }
}
__device__ __forceinline__ uint2 load_codes(const uint8_t* p, int n) {
  uint2 c = make_uint2(0, 0);
  if (n >= 8) {
    const u32x2_any v = *reinterpret_cast<const u32x2_any*>(p);
    c = make_uint2(v[0], v[1]);
  } else {
    int z = 0;   // as in load8
    asm volatile("" : "+v"(z));
    p += z;
#pragma unroll
    for (int i = 0; i < 7; ++i)
      if (i < n) (i < 4 ? c.x : c.y) |= (uint32_t)p[i] << (8 * (i & 3));
  }
  return c;
}
__device__ __forceinline__ void ckpt_values(uint2 c, int b, float (&v)[8]) {
  const float s = __uint_as_float((uint32_t)b << 23);
  typedef float f2 __attribute__((ext_vector_type(2)));
  const f2 a0 = __builtin_amdgcn_cvt_pk_f32_fp8(c.x, false), a1 = __builtin_amdgcn_cvt_pk_f32_fp8(c.x, true);
  const f2 a2 = __builtin_amdgcn_cvt_pk_f32_fp8(c.y, false), a3 = __builtin_amdgcn_cvt_pk_f32_fp8(c.y, true);
  v[0] = a0[0] * s, v[1] = a0[1] * s, v[2] = a1[0] * s, v[3] = a1[1] * s;
  v[4] = a2[0] * s, v[5] = a2[1] * s, v[6] = a3[0] * s, v[7] = a3[1] * s;
}

// Largest of m over the four lanes that hold a block: neighbours (lane bits 0
// and 1), or the lanes of the four 16-lane groups (bits 4 and 5; the swap of a
// register with itself leaves both groups' values in its two results).
enum { LANES_NEXT = 0, LANES_APART = 1 };
template <int LANES>
__device__ __forceinline__ uint32_t block_max(uint32_t m) {
  if constexpr (LANES == LANES_NEXT) {
    m = max(m, (uint32_t)dpp_i<kDppXor1>((int)m));
    return max(m, (uint32_t)dpp_i<kDppXor2>((int)m));
  } else {
    const auto a = __builtin_amdgcn_permlane16_swap(m, m, false, false);
    m = max(a[0], a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(m, m, false, false);
    return max(b[0], b[1]);
  }
}

// Write 8 values (already rounded to the stored type; those past n are 0) of
// row r from column c, c % 8 == 0, into a checkpoint of `cols` columns; the
// block's scale byte is returned, and written unless the caller does.  Every
// lane of the wave calls this, `live` where its row exists.
template <int LANES, bool SCALE = true>
__device__ __forceinline__ int ckpt_store8(uint8_t* codes, uint8_t* scales, int64_t r, int c, int cols,
                                           const float (&v)[8], int n, bool live) {
  const int b = ckpt_byte(block_max<LANES>(amax8(v)));
  if (live && n > 0) {
    store_codes(codes + r * cols + c, ckpt_codes(v, b), n);
    if (SCALE && c % kCkptBlock == 0)
      scales[r * ((cols + kCkptBlock - 1) / kCkptBlock) + c / kCkptBlock] = (uint8_t)b;
  }
  return b;
}

// 8 values of a saved activation, row r, columns c .. c + n - 1.
template <typename T>
__device__ __forceinline__ void saved_load8(const T* rows, int64_t ld, const uint8_t* codes,
                                            const uint8_t* scales, int64_t r, int c, int cols, int n,
                                            float (&v)[8]) {
  if (codes) {
    const int b = scales[r * ((cols + kCkptBlock - 1) / kCkptBlock) + c / kCkptBlock];
    ckpt_values(load_codes(codes + r * cols + c, n), b, v);
  } else {
    const Raw8<T> x = load8(rows + r * ld + c, n);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = x.get(i);
  }
}

}  // namespace
}  // namespace fs
