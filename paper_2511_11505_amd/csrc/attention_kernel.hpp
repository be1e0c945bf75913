// Attention of new tokens over a paged key-value cache.
//
// For a query row q and the tokens j that it sees, out = sum_j e^(s_j) v_j /
// sum_j e^(s_j), s_j = scale q . k_j, in one pass over the cache: the running
// maximum m, the sum l and the sum of values are rescaled when m grows (in powers
// of two, s times log2 e).
//
// Reading the cache once bounds it (a step of one token does 2 G operations a
// byte in bf16, G query heads a key head), so all rows that read the same keys,
// the G heads of n new tokens, are one tile's rows, and the cache goes from
// memory to registers to the matrix cores, with no LDS between:
//
//  * S^T = K Q^T: keys are the first operand, a lane holds 8 columns of one
//    token (16 tokens by 4 column groups), as rows lie in memory.  The result
//    has a query row in each lane column: lane (q, g) holds tokens 4 g .. 4 g + 3
//    of each group of 16.
//  * O^T = V^T P^T: as the order of the tokens in a sum is free, the tokens that
//    a lane's probabilities are of are also the ones whose values it loads, so
//    that P goes from one product's result to the next one's operand in place.
//    A lane loads 8 columns of 8 tokens (a wave reads whole rows) and packs
//    them by column; which column is which row of the product is free too.
//  * The result again has a query row in each lane column: the statistics are
//    per lane, and rescaling needs no exchange.
//
// A wave runs one tile ahead (16 KB of a bf16 cache of head_dim 128 in flight
// beside the 16 KB in use).  The tokens of all sequences are divided evenly over
// a fixed number of workgroups whatever the lengths are (the host does not know
// them); a workgroup's part may hold the end of one sequence, whole ones and
// the start of another.  Parts of a sequence are joined by a second kernel in
// the order of the workgroups.
#pragma once

#include <type_traits>

#include "attention.hpp"
#include "saved.hpp"

namespace fs {
namespace {

template <int BYTES> struct RawT;
template <> struct RawT<16> { typedef u32x4_any type; };
template <> struct RawT<8> { typedef u32x2_any type; };
typedef uint32_t u32x1_any __attribute__((ext_vector_type(1), aligned(1)));
template <> struct RawT<4> { typedef u32x1_any type; };

__device__ __forceinline__ int lane_i(int v, int l) { return __builtin_amdgcn_readlane(v, l); }
__device__ __forceinline__ int64_t lane_i64(int64_t v, int l) {
  return (int64_t)(uint32_t)lane_i((int)v, l) | (int64_t)lane_i((int)(v >> 32), l) << 32;
}
__device__ __forceinline__ int64_t shfl_i64(int64_t v, int l) {
  return (int64_t)(uint32_t)__shfl((int)v, l) | (int64_t)__shfl((int)(v >> 32), l) << 32;
}
// Over the four lanes of a query row (lane bits 4 and 5).
__device__ __forceinline__ float row_max(float v) {
  const uint32_t u = __float_as_uint(v);
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const uint32_t w = __float_as_uint(v);
  const auto b = __builtin_amdgcn_permlane32_swap(w, w, false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float row_sum(float v) {
  const uint32_t u = __float_as_uint(v);
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const uint32_t w = __float_as_uint(v);
  const auto b = __builtin_amdgcn_permlane32_swap(w, w, false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
__device__ __forceinline__ float exp2_hw(float v) { return __builtin_amdgcn_exp2f(v); }

// What an item (a sequence, or a part of its rows) reads.
struct Item {
  int seq, row0, nrows, len;
  int lo, hi;              // tokens that any of its rows sees: [lo, hi)
  int lo_all, hi_all;      // tokens that all of them see
  int first, tiles;        // tiles of TILE tokens, at least one
};
template <int TILE, int R>
__device__ __forceinline__ Item item_of(const AttnPlan& p, int item) {
  Item t;
  t.seq = p.row_groups == 1 ? item : item / p.row_groups;
  t.row0 = p.row_groups == 1 ? 0 : (item - t.seq * p.row_groups) * R;
  t.nrows = min(R, p.rows - t.row0);
  t.len = min(max(p.a.lengths[t.seq], 0), p.c.max_pages * p.c.page_size);
  int i0 = 0, i1 = p.a.n_new - 1;
  if (p.row_groups > 1) i0 = t.row0 / p.group, i1 = (t.row0 + t.nrows - 1) / p.group;
  const int at0 = t.len - p.a.n_new + i0, at1 = t.len - p.a.n_new + i1;
  t.hi = at1 + 1, t.hi_all = at0 + 1;
  t.lo = p.a.window ? max(0, at0 + 1 - p.a.window) : 0;
  t.lo_all = p.a.window ? max(0, at1 + 1 - p.a.window) : 0;
  t.first = 0, t.tiles = 1;
  if (t.hi > t.lo) {
    t.first = t.lo / TILE;
    t.tiles = (t.hi + TILE - 1) / TILE - t.first;
  }
  return t;
}

template <int CACHE, int D, int RT, bool P16>
struct Attn {
  static constexpr bool kF32 = CACHE == CACHE_F32 || CACHE == CACHE_CODES_F32;
  static constexpr bool kCodes = CACHE == CACHE_CODES_BF16 || CACHE == CACHE_CODES_F32;
  static constexpr int ES = kCodes ? 1 : kF32 ? 4 : 2;       // bytes of a cache element
  static constexpr int NG = kF32 ? 1 : 2;                    // groups of 16 tokens in a tile
  static constexpr int TILE = 16 * NG;
  static constexpr int R = 16 * RT;                          // rows of an item
  static constexpr int KE = kF32 ? 4 : 8;                    // columns of K a lane holds together
  static constexpr int KC = D / (4 * KE);
  static constexpr int VE = kF32 || D == 64 ? 4 : 8;         // columns of V
  static constexpr int VC = D / (16 * VE);
  static constexpr int VT = 4 * NG;                          // tokens of V a lane holds
  static constexpr int NO = D / 16;                          // result tiles of a row tile
  static constexpr int STRIDE = D + 4;                       // LDS row (floats)
  typedef typename std::conditional<kF32, float, bf16_t>::type T;
  typedef typename RawT<KE * ES>::type KRaw;
  typedef typename RawT<VE * ES>::type VRaw;
  static_assert(TILE * 16 <= 16 * STRIDE, "a wave's probabilities fit its part of the LDS");

  struct Tile {
    KRaw k[NG][KC];
    VRaw v[VC][VT];
    uint8_t ks[kCodes ? NG : 1][KC], vs[VC][kCodes ? VT : 1];
    uint32_t ok;     // bit t: token t has a place
    bool full;       // every row sees every token
  };

  const AttnPlan& p;
  float* lds;        // this wave's 16 rows of STRIDE
  const int lane, q, g, head;
  Item it;
  // pages: lane i has the offset (elements, of the head's part) of the group
  // (P16) or token window + i, or -1, and its index among the scale rows
  int window;
  int64_t base, srow;
  int koff[KC], voff[VC];
  int lim[RT], low[RT];

  typedef uint32_t Frag __attribute__((ext_vector_type(kF32 ? KE : 4)));
  Frag qf[RT][KC];
  floatx4 o[RT][NO];
  float m[RT], l[RT];
  uint32_t seen[RT];

  __device__ __forceinline__ Attn(const AttnPlan& plan, float* shared, int ln, int hd)
      : p(plan), lds(shared), lane(ln), q(ln & 15), g(ln >> 4), head(hd) {}

  __device__ __forceinline__ const uint8_t* kbase() const {
    return (const uint8_t*)p.c.k + (int64_t)head * p.c.head_stride * ES;
  }
  __device__ __forceinline__ const uint8_t* vbase() const {
    return (const uint8_t*)p.c.v + (int64_t)head * p.c.head_stride * ES;
  }

  // ---- one item's start: its rows and what each of them sees
  __device__ __forceinline__ void begin(const Item& item) {
    it = item;
    window = -(1 << 30);
#pragma unroll
    for (int c = 0; c < KC; ++c) koff[c] = min(c * 4 * KE + g * KE, p.c.d - KE) * ES;
#pragma unroll
    for (int c = 0; c < VC; ++c) voff[c] = min(c * 16 * VE + q * VE, p.c.d - VE) * ES;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int r = t * 16 + q;
      const bool in = r < it.nrows;
      const int row = it.row0 + (in ? r : 0), i = row / p.group;
      lim[t] = it.len - p.a.n_new + i;
      low[t] = p.a.window ? lim[t] - p.a.window : -1;
      const T* src = (const T*)p.a.q.p + ((int64_t)it.seq * p.a.n_new + i) * p.a.q.ts +
                     (int64_t)(head * p.group + row - i * p.group) * p.a.q.hs;
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        const int col = c * 4 * KE + g * KE;
        qf[t][c] = {};
        if (in && col < p.c.d) {
          qf[t][c] = *reinterpret_cast<const u32x4_any*>(src + col);
        }
      }
      m[t] = -INFINITY, l[t] = 0.f, seen[t] = 0;
#pragma unroll
      for (int n = 0; n < NO; ++n) o[t][n] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
  }

  // ---- loads
  static constexpr int PER = P16 ? 64 / NG : 64 / TILE;   // tiles of a window of pages
  __device__ __forceinline__ void find_pages(int tile) {
    if (tile < window + PER) return;
    window = tile;
    const int t = tile * TILE + (P16 ? lane * 16 : lane);
    base = -1, srow = 0;
    if (t < it.hi && t >= (P16 ? it.lo - 15 : it.lo)) {
      const int slot = t / p.c.page_size, place = t - slot * p.c.page_size;
      const int page = p.c.table[(int64_t)it.seq * p.c.ldt + slot];
      if (page >= 0 && page < p.c.n_pages) {
        base = (int64_t)page * p.c.page_stride + (int64_t)place * p.c.place_stride;
        srow = ((int64_t)page * p.c.kv_heads + head) * p.c.page_size + place;
      }
    }
  }
  // Place of token `tok` (within the tile; the lane's own) of a tile at window
  // position w: element offset, and scale row.
  __device__ __forceinline__ int64_t place(int w, int u, int r) const {
    if constexpr (P16) return lane_i64(base, w * NG + u) + r * p.c.place_stride;
    else return shfl_i64(base, w * TILE + u * 16 + r);
  }
  __device__ __forceinline__ int64_t scale_row(int w, int u, int r) const {
    if constexpr (P16) return lane_i64(srow, w * NG + u) + r;
    else return shfl_i64(srow, w * TILE + u * 16 + r);
  }

  template <bool FULL>
  __device__ __forceinline__ void load_rows(Tile& x, int tile, int w) {
    const uint8_t *kb = kbase(), *vb = vbase();
    const int nb = (p.c.d + kCkptBlock - 1) / kCkptBlock;
    auto there = [&](int tok) {
      const int t = tile * TILE + tok;
      return FULL || ((x.ok >> tok & 1) && t >= it.lo && t < it.hi);
    };
#pragma unroll
    for (int u = 0; u < NG; ++u) {
      const int64_t at = place(w, u, q) * ES;
      const int64_t sr = kCodes ? scale_row(w, u, q) : 0;
      const bool in = there(u * 16 + q);
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        x.k[u][c] = {};
        if (in) x.k[u][c] = *reinterpret_cast<const KRaw*>(kb + at + koff[c]);
        if constexpr (kCodes) {
          x.ks[u][c] = 0;
          if (in) x.ks[u][c] = p.c.k_scales[sr * nb + koff[c] / kCkptBlock];
        }
      }
    }
#pragma unroll
    for (int i = 0; i < VT; ++i) {
      const int u = i / 4, r = g * 4 + i % 4;
      const int64_t at = place(w, u, r) * ES;
      const int64_t sr = kCodes ? scale_row(w, u, r) : 0;
      const bool in = there(u * 16 + r);
#pragma unroll
      for (int c = 0; c < VC; ++c) {
        x.v[c][i] = {};
        if (in) x.v[c][i] = *reinterpret_cast<const VRaw*>(vb + at + voff[c]);
        if constexpr (kCodes) {
          x.vs[c][i] = 0;
          if (in) x.vs[c][i] = p.c.v_scales[sr * nb + voff[c] / kCkptBlock];
        }
      }
    }
  }

  __device__ __forceinline__ void load(Tile& x, int tile) {
    find_pages(tile);
    const int w = tile - window;
    if constexpr (P16) {
      x.ok = lane_i64(base, w * NG) >= 0 ? 0xFFFFu : 0u;
      if (NG > 1) x.ok |= lane_i64(base, w * NG + 1) >= 0 ? 0xFFFF0000u : 0u;
    } else {
      x.ok = (uint32_t)(__ballot(base >= 0) >> (w * TILE)) & (uint32_t)((1ull << TILE) - 1);
    }
    const int t0 = tile * TILE;
    x.full = x.ok == (uint32_t)((1ull << TILE) - 1) && t0 >= it.lo_all && t0 + TILE <= it.hi_all;
    if (x.full) load_rows<true>(x, tile, w);
    else load_rows<false>(x, tile, w);
  }

  // ---- operands
  // E4M3 codes of one block to pairs of bf16, exactly.
  static __device__ __forceinline__ uint32_t pair_bf16(uint32_t codes, float scale, bool high) {
    typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
    const bf2 v = high ? (bf2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true)
                       : (bf2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false);
    return __builtin_bit_cast(uint32_t, v);
  }
  static __device__ __forceinline__ float scale_of(uint8_t b) { return __uint_as_float((uint32_t)b << 23); }

  __device__ __forceinline__ Frag kfrag(const Tile& x, int u, int c) const {
    Frag f;
    if constexpr (CACHE == CACHE_CODES_BF16) {
      const float s = scale_of(x.ks[u][c]);
      f[0] = pair_bf16(x.k[u][c][0], s, false), f[1] = pair_bf16(x.k[u][c][0], s, true);
      f[2] = pair_bf16(x.k[u][c][1], s, false), f[3] = pair_bf16(x.k[u][c][1], s, true);
    } else if constexpr (CACHE == CACHE_CODES_F32) {
      float v[8];
      ckpt_values(make_uint2(x.k[u][c][0], 0), x.ks[u][c], v);
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = __float_as_uint(v[i]);
    } else {
      f = x.k[u][c];
    }
    // (columns past head_dim were loaded from inside the row; Q is 0 there, but
    // 0 times an infinity is not)
    if ((c + 1) * 4 * KE > p.c.d && c * 4 * KE + g * KE >= p.c.d) f = Frag{};
    return f;
  }
  // Columns of token slot i as loaded from memory, in the product's type.
  typedef uint32_t VWords __attribute__((ext_vector_type(kF32 ? 4 : VE / 2)));
  __device__ __forceinline__ VWords vwords(const VRaw& raw, uint8_t sb) const {
    VWords f;
    if constexpr (CACHE == CACHE_CODES_BF16) {
      const float s = scale_of(sb);
#pragma unroll
      for (int j = 0; j < VE / 4; ++j) {
        f[2 * j] = pair_bf16(raw[j], s, false);
        f[2 * j + 1] = pair_bf16(raw[j], s, true);
      }
    } else if constexpr (CACHE == CACHE_CODES_F32) {
      float v[8];
      ckpt_values(make_uint2(raw[0], 0), sb, v);
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = __float_as_uint(v[i]);
    } else {
      f = raw;
    }
    return f;
  }
  static __device__ __forceinline__ float velem(const VWords& f, int j) {
    if constexpr (kF32) return __uint_as_float(f[j]);
    else return __uint_as_float((j & 1) ? (f[j / 2] & 0xFFFF0000u) : (f[j / 2] << 16));
  }

  // ---- one tile
  __device__ __forceinline__ void compute(const Tile& x, int tile) {
    Frag kf[NG][KC];
#pragma unroll
    for (int u = 0; u < NG; ++u)
#pragma unroll
      for (int c = 0; c < KC; ++c) kf[u][c] = kfrag(x, u, c);
    float pr[RT][VT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      floatx4 s[NG];
#pragma unroll
      for (int u = 0; u < NG; ++u) {
        s[u] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < KC; ++c) {
          if constexpr (kF32) {
#pragma unroll
            for (int i = 0; i < KE; ++i)
              s[u] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kf[u][c][i]), __uint_as_float(qf[t][c][i]),
                                                          s[u], 0, 0, 0);
          } else {
            s[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf[u][c]),
                                                           __builtin_bit_cast(bf16x8, qf[t][c]), s[u], 0, 0, 0);
          }
        }
      }
      float mx = -INFINITY;
#pragma unroll
      for (int i = 0; i < VT; ++i) {
        float v = s[i / 4][i % 4] * p.scale2;
        if (!x.full) {
          const int tok = (i / 4) * 16 + g * 4 + i % 4, at = tile * TILE + tok;
          const bool vis = (x.ok >> tok & 1) && at <= lim[t] && at > low[t];
          v = vis ? v : -INFINITY;
          seen[t] |= (uint32_t)vis;
        }
        pr[t][i] = v;
        mx = fmaxf(mx, v);
      }
      if (x.full) seen[t] = 1;
      mx = fmaxf(m[t], row_max(mx));
      const float mu = mx == -INFINITY ? 0.f : mx;
      if (__any(mx > m[t])) {
        const float scale = exp2_hw(m[t] - mu);
        l[t] *= scale;
#pragma unroll
        for (int n = 0; n < NO; ++n) o[t][n] *= scale;
        m[t] = mx;
      }
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < VT; ++i) {
        pr[t][i] = exp2_hw(pr[t][i] - mu);
        sum += pr[t][i];
      }
      l[t] += sum;
    }

    if (!x.full && p.a.n_new > 1) {
      // Rows that see different tokens: a value that is not finite must not
      // reach, as 0 times itself, a row that does not see it.
      uint32_t bad = 0;
#pragma unroll
      for (int c = 0; c < VC; ++c)
#pragma unroll
        for (int i = 0; i < VT; ++i) {
          const VWords f = vwords(x.v[c][i], x.vs[c][kCodes ? i : 0]);
#pragma unroll
          for (int j = 0; j < VE; ++j) bad |= (__float_as_uint(velem(f, j)) & 0x7F800000u) == 0x7F800000u;
        }
      if (__any(bad)) {
        values_one_by_one(x, tile, pr);
        return;
      }
    }

    if constexpr (kF32) {
#pragma unroll
      for (int i = 0; i < VT; ++i)
#pragma unroll
        for (int c = 0; c < VC; ++c) {
          const VWords f = vwords(x.v[c][i], x.vs[c][kCodes ? i : 0]);
#pragma unroll
          for (int j = 0; j < VE; ++j)
#pragma unroll
            for (int t = 0; t < RT; ++t)
              o[t][c * VE + j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(f[j]), pr[t][i],
                                                                      o[t][c * VE + j], 0, 0, 0);
        }
    } else {
      bf16x8 pf[RT];
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int i = 0; i < 8; ++i) pf[t][i] = (__bf16)pr[t][i];
#pragma unroll
      for (int c = 0; c < VC; ++c) {
        VWords f[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = vwords(x.v[c][i], x.vs[c][kCodes ? i : 0]);
#pragma unroll
        for (int j = 0; j < VE; ++j) {
          Frag a;
#pragma unroll
          for (int i = 0; i < 4; ++i)
            a[i] = __builtin_amdgcn_perm(f[2 * i + 1][j / 2], f[2 * i][j / 2], (j & 1) ? 0x07060302u : 0x05040100u);
#pragma unroll
          for (int t = 0; t < RT; ++t)
            o[t][c * VE + j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), pf[t],
                                                                       o[t][c * VE + j], 0, 0, 0);
        }
      }
    }
  }

  // The values of a tile token by token, each only for the rows that see it
  // (rare: some value is not finite).
  __device__ __forceinline__ void values_one_by_one(const Tile& x, int tile, const float (&pr)[RT][VT]) {
    const uint8_t* vb = vbase();
    [[maybe_unused]] const int nb = (p.c.d + kCkptBlock - 1) / kCkptBlock;
    const int w = tile - window;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
#pragma unroll
      for (int i = 0; i < VT; ++i) lds[((i / 4) * 16 + g * 4 + i % 4) * 16 + q] = pr[t][i];
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll 1
      for (int tok = 0; tok < TILE; ++tok) {
        const int at = tile * TILE + tok;
        if (!(x.ok >> tok & 1) || at < it.lo || at >= it.hi) continue;
        const bool vis = at <= lim[t] && at > low[t];
        const float pv = lds[tok * 16 + q];
        const int64_t off = P16 ? lane_i64(base, w * NG + tok / 16) + (tok % 16) * p.c.place_stride
                                : lane_i64(base, w * TILE + tok);
#pragma unroll
        for (int c = 0; c < VC; ++c)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int col = min(c * 16 * VE + (4 * g + r) * VE, p.c.d - VE);
            const VRaw raw = *reinterpret_cast<const VRaw*>(vb + (off + col) * ES);
            uint8_t sb = 0;
            if constexpr (kCodes) {
              const int64_t sr = P16 ? lane_i64(srow, w * NG + tok / 16) + tok % 16 : lane_i64(srow, w * TILE + tok);
              sb = p.c.v_scales[sr * nb + col / kCkptBlock];
            }
            const VWords f = vwords(raw, sb);
#pragma unroll
            for (int j = 0; j < VE; ++j) o[t][c * VE + j][r] += vis ? pv * velem(f, j) : 0.f;
          }
      }
      __builtin_amdgcn_wave_barrier();
    }
  }

  __device__ __forceinline__ void tiles(int from, int to) {
    Tile a, b;
    if (from >= to) return;
    load(a, from);
    for (int t = from;; t += 2) {
      if (t + 1 < to) load(b, t + 1);
      __builtin_amdgcn_sched_barrier(0);
      compute(a, t);
      if (t + 1 >= to) return;
      if (t + 2 < to) load(a, t + 2);
      __builtin_amdgcn_sched_barrier(0);
      compute(b, t + 1);
      if (t + 2 >= to) return;
    }
  }
};

// The final row: out = o / l, lse; l < 0 where nothing was seen.
template <typename T, int N>
__device__ __forceinline__ void finish_row(const AttnPlan& p, const Item& it, int head, int row, int col, float m,
                                           float l, const float (&o)[N]) {
  const int r = it.row0 + row, i = r / p.group, h = head * p.group + r - i * p.group;
  const int64_t tok = (int64_t)it.seq * p.a.n_new + i;
  const bool none = l < 0.f;
  if (col == 0 && p.a.lse) p.a.lse[tok * p.a.q_heads + h] = none ? -INFINITY : (m + __log2f(l)) * 0.69314718055994531f;
  T* dst = (T*)p.a.out.p + tok * p.a.out.ts + h * p.a.out.hs + col;
#pragma unroll
  for (int c = 0; c < N; c += 4) {
    if (col + c >= p.c.d) break;
    T v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = from_f32<T>(none ? 0.f : o[c + j] / l);
    memcpy(dst + c, v, sizeof(v));
  }
}

template <int CACHE, int D, int RT, bool P16>
__global__ __launch_bounds__(64 * kAttnWaves) void attention_kernel(AttnPlan p) {
  typedef Attn<CACHE, D, RT, P16> A;
  typedef typename A::T T;
  __shared__ __align__(16) float rows[kAttnWaves][16][A::STRIDE];
  __shared__ float2 stats[kAttnWaves][16];
  __shared__ int64_t scan[kAttnWaves];
  __shared__ int64_t found[2];   // first item | its first tile

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int head = (int)(blockIdx.x % p.c.kv_heads), worker = (int)(blockIdx.x / p.c.kv_heads);
  int item = worker;
  int64_t at = 0, total = 0, left;     // tile `at` of the item; tiles left of this part
  int64_t part0 = 0;
  int parts = 0;
  if (p.workers) {
    // tiles before each thread's items
    const int per = (p.items + 255) / 256, i0 = min(tid * per, p.items), i1 = min(i0 + per, p.items);
    int64_t mine = 0;
    for (int i = i0; i < i1; ++i) mine += item_of<A::TILE, A::R>(p, i).tiles;
    int64_t incl = mine;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int64_t v = shfl_i64(incl, lane - d < 0 ? lane : lane - d);
      if (lane >= d) incl += v;
    }
    if (lane == 63) scan[wave] = incl;
    __syncthreads();
    int64_t before = 0;
#pragma unroll
    for (int w = 0; w < kAttnWaves; ++w) {
      if (w < wave) before += scan[w];
      total += scan[w];
    }
    parts = (int)min((int64_t)p.workers, (total + kAttnMinTiles - 1) / kAttnMinTiles);
    if (worker >= parts) return;
    part0 = worker * total / parts;
    left = (worker + 1) * total / parts - part0;
    int64_t excl = before + incl - mine;
    if (part0 >= excl && part0 < excl + mine)
      for (int i = i0; i < i1; ++i) {
        const int n = item_of<A::TILE, A::R>(p, i).tiles;
        if (part0 < excl + n) {
          found[0] = i, found[1] = part0 - excl;
          break;
        }
        excl += n;
      }
    __syncthreads();
    item = __builtin_amdgcn_readfirstlane((int)found[0]);
    at = __builtin_amdgcn_readfirstlane((int)found[1]);
    total = lane_i64(total, 0), part0 = lane_i64(part0, 0), left = lane_i64(left, 0);
  } else {
    left = 1;   // one item
  }

  A s(p, &rows[wave][0][0], lane, head);
  while (left > 0) {
    const Item it = item_of<A::TILE, A::R>(p, item);
    const int from = (int)at;
    const int n = p.workers ? (int)min((int64_t)(it.tiles - from), left) : it.tiles;
    const bool whole = n == it.tiles;
    s.begin(it);
    s.tiles(it.first + from + (int)((int64_t)n * wave / kAttnWaves),
            it.first + from + (int)((int64_t)n * (wave + 1) / kAttnWaves));
    if (p.workers && from == 0 && head == 0 && tid == 0) {
      // the parts that hold this item: the last part that starts at or before a tile
      const int64_t t0 = part0, t1 = part0 + it.tiles - 1;
      p.span[item] = make_int2((int)(((t0 + 1) * parts - 1) / total), (int)(((t1 + 1) * parts - 1) / total));
    }
    // the four waves' sums
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      if (t * 16 >= it.nrows) break;
#pragma unroll
      for (int c = 0; c < A::VC; ++c)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int j = 0; j < A::VE; j += 4) {
            const floatx4 v{s.o[t][c * A::VE + j][r], s.o[t][c * A::VE + j + 1][r], s.o[t][c * A::VE + j + 2][r],
                            s.o[t][c * A::VE + j + 3][r]};
            *reinterpret_cast<floatx4*>(&rows[wave][s.q][c * 16 * A::VE + (4 * s.g + r) * A::VE + j]) = v;
          }
      const float l = row_sum(s.l[t]);
      const bool seen = row_max((float)s.seen[t]) > 0.f;
      if (s.g == 0) stats[wave][s.q] = make_float2(s.m[t], seen ? l : -1.f);
      __syncthreads();
      constexpr int N = D / 16;
      const int row = tid >> 4, col = (tid & 15) * N;
      if (t * 16 + row < it.nrows) {
        float m = -INFINITY, sum = 0.f, o[N];
        bool any = false;
#pragma unroll
        for (int w = 0; w < kAttnWaves; ++w) m = fmaxf(m, stats[w][row].x);
#pragma unroll
        for (int c = 0; c < N; ++c) o[c] = 0.f;
#pragma unroll
        for (int w = 0; w < kAttnWaves; ++w) {
          const float2 st = stats[w][row];
          const float e = st.x == -INFINITY ? 0.f : exp2_hw(st.x - m);
          any |= !(st.y < 0.f);
          sum += st.y < 0.f ? 0.f : e * st.y;
#pragma unroll
          for (int c = 0; c < N; c += 4) {
            const floatx4 v = *reinterpret_cast<const floatx4*>(&rows[w][row][col + c]);
#pragma unroll
            for (int j = 0; j < 4; ++j) o[c + j] += e * v[j];
          }
        }
        if (!any) sum = -1.f;
        if (whole) {
          finish_row<T, N>(p, it, head, t * 16 + row, col, m, sum, o);
        } else {
          const int64_t pr = (((int64_t)worker * p.c.kv_heads + head) * 2 + (from == 0 ? 1 : 0)) * A::R + t * 16 + row;
#pragma unroll
          for (int c = 0; c < N; c += 4)
            *reinterpret_cast<floatx4*>(p.part + pr * D + col + c) = floatx4{o[c], o[c + 1], o[c + 2], o[c + 3]};
          if (col == 0) p.stat[pr] = make_float2(m, sum);
        }
      }
      __syncthreads();
    }
    left -= p.workers ? n : 1;
    part0 += n;
    at = 0;
    ++item;
  }
}

// Rows of items that several parts hold: a wave a row, the parts in their order.
template <typename T, int D, int R, int TILE>
__global__ __launch_bounds__(256) void attention_join_kernel(AttnPlan p, int blocks) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t id = blockIdx.x;
  const int row = (int)(id % blocks) * 4 + wave;
  const int head = (int)(id / blocks % p.c.kv_heads), item = (int)(id / blocks / p.c.kv_heads);
  const int2 span = p.span[item];
  if (span.x == span.y) return;
  const Item it = item_of<TILE, R>(p, item);
  if (row >= it.nrows) return;
  // the statistics, a lane a part
  const int n = span.y - span.x + 1;
  auto index = [&](int i) {
    return (((int64_t)(span.x + i) * p.c.kv_heads + head) * 2 + (i == 0 ? 1 : 0)) * R + row;
  };
  float m = -INFINITY;
  for (int i = lane; i < n; i += 64) m = fmaxf(m, p.stat[index(i)].x);
  m = wave_max(m);
  constexpr int N = D / 64;
  float o[N], sum = 0.f;
  bool any = false;
#pragma unroll
  for (int c = 0; c < N; ++c) o[c] = 0.f;
#pragma unroll 4
  for (int i = 0; i < n; ++i) {
    const int64_t r = index(i);
    const float2 st = p.stat[r];
    const float e = st.x == -INFINITY ? 0.f : exp2_hw(st.x - m);
    any |= !(st.y < 0.f);
    sum += st.y < 0.f ? 0.f : e * st.y;
#pragma unroll
    for (int c = 0; c < N; ++c) o[c] += e * p.part[r * D + lane * N + c];
  }
  if (!any) sum = -1.f;
  const int q = it.row0 + row, i = q / p.group, h = head * p.group + q - i * p.group;
  const int64_t tok = (int64_t)it.seq * p.a.n_new + i;
  if (lane == 0 && p.a.lse)
    p.a.lse[tok * p.a.q_heads + h] = sum < 0.f ? -INFINITY : (m + __log2f(sum)) * 0.69314718055994531f;
#pragma unroll
  for (int c = 0; c < N; ++c)
    if (lane * N + c < p.c.d)
      ((T*)p.a.out.p)[tok * p.a.out.ts + h * p.a.out.hs + lane * N + c] = from_f32<T>(sum < 0.f ? 0.f : o[c] / sum);
}

}  // namespace

template <int CACHE, int D, int RT, bool P16>
hipError_t run_attention(const AttnPlan& p, hipStream_t s) {
  typedef Attn<CACHE, D, RT, P16> A;
  const int64_t groups = (int64_t)(p.workers ? p.workers : p.items) * p.c.kv_heads;
  launch_k(attention_kernel<CACHE, D, RT, P16>, dim3((unsigned)groups), 64 * kAttnWaves, 0, s, p);
  if (p.workers) {
    const int nrows = p.rows < A::R ? p.rows : A::R, blocks = (nrows + 3) / 4;
    launch_k(attention_join_kernel<typename A::T, D, A::R, A::TILE>,
             dim3((unsigned)((int64_t)p.items * p.c.kv_heads * blocks)), 256, 0, s, p, blocks);
  }
  return hipGetLastError();
}

}  // namespace fs
