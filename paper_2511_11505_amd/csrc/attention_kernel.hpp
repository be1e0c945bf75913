// Attention of new tokens over a paged key-value cache.
//
// For a query row q and the tokens j that it sees, out = sum_j e^(s_j) v_j /
// sum_j e^(s_j), s_j = scale q . k_j, in one pass over the cache: the running
// maximum m, the sum l and the sum of values are rescaled when m grows.
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
// A wave holds one tile of keys and one of values: the next keys are on their way
// while the values are multiplied, the next values while the keys are; of small
// tiles (8 KB with their values) it holds two (an 8-bit cache of 8 sequences of up
// to 65536 tokens took 108 us with one where it took 95 with two).  At two waves a SIMD and 16 KB a
// tile some 100 KB a CU are on their way.
//
// The tokens of all sequences are divided evenly over a fixed number of
// workgroups, about as many as the chip runs at once, whatever the lengths are (the host
// does not know them); a workgroup's part may hold the end of one sequence, whole
// ones and the start of another.  Parts of a sequence are joined by a second
// kernel in the order of the workgroups.  (Each part has a workgroup for every key head,
// and their number is rounded up: where the key heads do not divide 512, or 256 with one
// workgroup a CU, a few workgroups start only when others end.)
//
// Measured (MI355X, head_dim 128, 40 query and 8 key heads): 64 sequences of 20 to
// 8192 tokens in bf16 147 us, 6.1 TB/s; 8 of 650 to 65536 in 8 bits 92 us, 5.3
// TB/s (reading alone goes at 6.5); one of 1500 tokens 11 to 13 us, of which the kernel 7
// and the join 4.5, both a chain of dependent loads.
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
typedef uint16_t u16_any __attribute__((aligned(1)));
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
// e^(a - b).  The difference is taken first: a score that fp32 holds may be one that it
// does not hold times log2 e.
__device__ __forceinline__ float exp_diff(float a, float b) {
  return __builtin_amdgcn_exp2f((a - b) * 1.4426950408889634f);
}
// The least factor of a rescaling, and the least weight among values that may be infinite
// (the sum of weights takes it as it is): with 0, where e^x has no normal fp32 number, an
// infinite value would become a NaN.  It adds at most 2^-126 of a value.
constexpr float kLeast = 0x1p-126f;
__device__ __forceinline__ float rescale(float m, float top) {
  return m == -INFINITY ? 0.f : fmaxf(exp_diff(m, top), kLeast);
}
// A row's output of its sums; without a weight (every score minus infinity) it is 0 / 0.
__device__ __forceinline__ float quotient(float o, float l) { return l == 0.f ? NAN : o / l; }
__device__ __forceinline__ float lse_of(float m, float l) { return m + __log2f(l) * 0.69314718055994531f; }

// Memory from a uniform address on; offsets at or above kNone read 0.  Rows are
// loaded as what is read once: in bf16 148.7 us against 166.4 (64 sequences of up
// to 8192 tokens, 6.0 and 5.4 TB/s).
constexpr uint32_t kNone = 0x80000000u;
constexpr int kOnce = 2;   // the non-temporal bit
template <int AUX>
struct BufferT {
  __amdgpu_buffer_rsrc_t r;
  __device__ __forceinline__ explicit BufferT(const void* p)
      : r(__builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)(kNone - 1), 0x20000)) {}
  __device__ __forceinline__ uint32_t load1(uint32_t off) const { return __builtin_amdgcn_raw_buffer_load_b8(r, off, 0, 0); }
  __device__ __forceinline__ uint32_t load2(uint32_t off) const { return __builtin_amdgcn_raw_buffer_load_b16(r, off, 0, 0); }
  __device__ __forceinline__ uint32_t load4(uint32_t off) const { return __builtin_amdgcn_raw_buffer_load_b32(r, off, 0, 0); }
  __device__ __forceinline__ void load(u32x1_any& v, uint32_t off) const { v[0] = load4(off); }
  __device__ __forceinline__ void load(u32x2_any& v, uint32_t off) const {
    const auto x = __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, AUX);
    v[0] = x[0], v[1] = x[1];
  }
  __device__ __forceinline__ void load(u32x4_any& v, uint32_t off) const {
    const auto x = __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, AUX);
    v[0] = x[0], v[1] = x[1], v[2] = x[2], v[3] = x[3];
  }
};

// What an item (a sequence, or a part of its rows) reads.
struct Item {
  int seq, row0, nrows, len;
  int lo, hi;              // tokens that any of its rows sees: [lo, hi)
  int lo_all, hi_all;      // tokens that all of them see (but those that see nothing)
  int first, tiles;        // tiles of TILE tokens, at least one
  int slots;               // what it counts for when work is divided
};
// Place of query i of a sequence; negative: it sees nothing.
__device__ __forceinline__ int query_place(const AttnPlan& p, int seq, int i, int len) {
  if (__builtin_expect(!p.a.positions, 1)) return len - p.a.n_new + i;
  return max(min(p.a.positions[(int64_t)seq * p.a.n_new + i], len - 1), -1);
}
template <int TILE, int R>
__device__ __forceinline__ Item item_of(const AttnPlan& p, int item, int length) {
  Item t;
  t.seq = p.row_groups == 1 ? item : item / p.row_groups;
  t.row0 = p.row_groups == 1 ? 0 : (item - t.seq * p.row_groups) * R;
  t.nrows = min(R, p.rows - t.row0);
  t.len = min(max(length, 0), p.c.max_pages * p.c.page_size);
  int i0 = 0, i1 = p.a.n_new - 1;
  if (p.row_groups > 1) i0 = t.row0 / p.group, i1 = (t.row0 + t.nrows - 1) / p.group;
  int at0 = t.len - p.a.n_new + i0, at1 = t.len - p.a.n_new + i1;
  if (__builtin_expect(p.a.positions != nullptr, 0)) {
    // the first and the last place of its queries (they may be in any order, and none;
    // one by one: unrolled, 4 new tokens of 192 or 256 columns took 656 us for 555)
    at0 = t.len - 1, at1 = -1;
#pragma unroll 1
    for (int i = i0; i <= i1; ++i) {
      const int at = query_place(p, t.seq, i, t.len);
      at1 = max(at1, at);
      if (at >= 0) at0 = min(at0, at);
    }
  }
  t.hi = at1 + 1, t.hi_all = at0 + 1;
  t.lo = p.a.window ? max(0, at0 + 1 - p.a.window) : 0;
  t.lo_all = p.a.window ? max(0, at1 + 1 - p.a.window) : 0;
  t.first = 0, t.tiles = 1;
  if (t.hi > t.lo) {
    t.first = t.lo / TILE;
    t.tiles = (t.hi + TILE - 1) / TILE - t.first;
  }
  // (starting and ending an item takes about as long as that many tiles)
  t.slots = max(t.tiles, kAttnMinTiles);
  return t;
}

template <int TILE, int R>
__device__ __forceinline__ Item item_of(const AttnPlan& p, int item) {
  return item_of<TILE, R>(p, item, p.a.lengths[p.row_groups == 1 ? item : item / p.row_groups]);
}

// The final row: out = o / l, lse; l < 0 where nothing was seen.
template <typename T, int N>
__device__ __forceinline__ void finish_row(const AttnPlan& p, const Item& it, int head, int row, int col, float m,
                                           float l, const float (&o)[N]) {
  const int r = it.row0 + row, i = r / p.group, h = head * p.group + r - i * p.group;
  const int64_t tok = (int64_t)it.seq * p.a.n_new + i;
  const bool none = l < 0.f;
  if (col == 0 && p.a.lse) p.a.lse[tok * p.a.q_heads + h] = none ? -INFINITY : lse_of(m, l);
  T* dst = (T*)p.a.out.p + tok * p.a.out.ts + h * p.a.out.hs + col;
#pragma unroll
  for (int c = 0; c < N; c += 4) {
    if (col + c >= p.c.d) break;
    T v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = from_f32<T>(none ? 0.f : quotient(o[c + j], l));
    memcpy(dst + c, v, sizeof(v));
  }
}

template <int CACHE, int D, int RT, int PAGES, int NEW>
struct Attn {
  static constexpr bool P16 = PAGES != PAGES_ANY;
  static constexpr bool MANY = NEW != NEW_ONE;
  static constexpr int kCached = NEW == NEW_PROMPT ? 0 : kOnce;   // (a prompt's rows read the cache again and again)
  static constexpr bool kF32 = CACHE == CACHE_F32 || CACHE == CACHE_CODES_F32;
  static constexpr bool kCodes = CACHE == CACHE_CODES_BF16 || CACHE == CACHE_CODES_F32;
  static constexpr int ES = kCodes ? 1 : kF32 ? 4 : 2;       // bytes of a cache element
  static constexpr int NG = kF32 ? 1 : 2;                    // groups of 16 tokens in a tile
  static constexpr int TILE = 16 * NG;
  static constexpr int R = 16 * RT;                          // rows of an item
  static constexpr int KE = kF32 ? 4 : 8;                    // columns of K in an operand of a product
  static constexpr int KC = D / (4 * KE);
  static constexpr int KL = kCodes ? 16 : KE;                // columns of K a lane loads together: 16 bytes
  static constexpr int KN = D / (4 * KL);
  static constexpr int VE = CACHE == CACHE_F32 || D == 64 ? 4 : 8;   // columns of V a lane loads together
  static constexpr int VC = D / (16 * VE);
  static constexpr int VT = 4 * NG;                          // tokens of V a lane holds
  static constexpr int NO = D / 16;                          // result tiles of a row tile
  static constexpr int STRIDE = D + 4;                       // LDS row (floats)
  static constexpr int NB = D / kCkptBlock;                  // scale bytes of a full-width row
  static constexpr int KW = (NB + 3) / 4;                    // words of a row's scales
  static constexpr int VW = NB == 2 && P16 ? 2 : 4 * KW;     // words of four rows'
  typedef typename std::conditional<kF32, float, bf16_t>::type T;
  typedef u32x4_any KRaw;
  typedef typename RawT<VE * ES>::type VRaw;

  typedef uint32_t Frag __attribute__((ext_vector_type(4)));
  typedef BufferT<kCached> Buffer;

  const AttnPlan& p;
  const int lane, q, g, head;
  Item it;
  // pages: lane i has the offset (elements, of the head's part) of the group
  // (P16) or token window + i, or -1, and its index among the scale rows
  int window;
  int64_t base, srow;
  bool last;
  uint32_t koff[KN], voff[VC][4];   // bytes in a row; P16: from the group's start
  int lim[RT], low[RT];

  // queries: in registers, or where they are many in LDS (which the four waves share)
  static constexpr bool kQShared = NEW != NEW_PROMPT && RT * KC * 4 > (kF32 ? 32 : 16);
  Frag qf[kQShared ? 1 : RT][kQShared ? 1 : KC];
  Frag* qs;
  floatx4 o[RT][NO];
  float m[RT], l[RT];
  uint32_t seen[RT];

  struct Tile {
    KRaw k[NG][KN];
    VRaw v[VC][VT];
    uint32_t ks[kCodes ? NG : 1][KW], vs[kCodes ? NG : 1][VW];   // scale bytes of a row; of rows 4 g .. 4 g + 3
    int at, w;       // which tile, at which position of the window
    uint32_t ok;     // bit t: token t has a place
    bool full;       // every row sees every token
    bool edge;       // of row_scales
  };

  __device__ __forceinline__ Attn(const AttnPlan& plan, int ln, int hd, Frag* queries)
      : p(plan), lane(ln), q(ln & 15), g(ln >> 4), head(hd), qs(queries) {}

  __device__ __forceinline__ const uint8_t* kbase() const {
    return (const uint8_t*)p.c.k + (int64_t)head * p.c.head_stride * ES;
  }
  __device__ __forceinline__ const uint8_t* vbase() const {
    return (const uint8_t*)p.c.v + (int64_t)head * p.c.head_stride * ES;
  }

  // First of this lane's columns of operand c.
  __device__ __forceinline__ int kcol(int c) const {
    constexpr int S = KL / KE;
    return (c / S * 4 + g) * KL + c % S * KE;
  }

  // ---- one item's start: its rows and what each of them sees.  (Shared queries
  // are written by all waves, a barrier has to follow.)
  __device__ __forceinline__ Frag query(int t, int c) const {
    if constexpr (kQShared) return qs[(t * KC + c) * 64 + lane];
    else return qf[t][c];
  }
  __device__ __forceinline__ void begin(const Item& item, int wave) {
    it = item;
    window = -(1 << 30);
    // (columns past head_dim have offsets past every buffer)
    const uint32_t step = P16 ? (uint32_t)p.c.place_stride : 0;
#pragma unroll
    for (int c = 0; c < KN; ++c) {
      const int col = c * 4 * KL + g * KL;
      koff[c] = col < p.c.d ? (q * step + col) * ES : kNone;   // (of P16)
    }
#pragma unroll
    for (int c = 0; c < VC; ++c)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int col = c * 16 * VE + q * VE;
        voff[c][r] = col < p.c.d ? ((g * 4 + r) * step + col) * ES : kNone;
      }
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int r = t * 16 + q;
      const bool in = r < it.nrows;
      const int row = it.row0 + (in ? r : 0), i = row / p.group;
      lim[t] = query_place(p, it.seq, i, it.len);
      low[t] = p.a.window ? lim[t] - p.a.window : -1;
      const T* src = (const T*)p.a.q.p + ((int64_t)it.seq * p.a.n_new + i) * p.a.q.ts +
                     (int64_t)(head * p.group + row - i * p.group) * p.a.q.hs;
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        const int col = kcol(c);
        if (kQShared && c % kAttnWaves != wave) continue;
        Frag f = {};
        if (in && col < p.c.d) f = *reinterpret_cast<const u32x4_any*>(src + col);
        if constexpr (kQShared) qs[(t * KC + c) * 64 + lane] = f;
        else qf[t][c] = f;
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
    base = -1, srow = 0, last = false;
    if (t < it.hi && t >= (P16 ? it.lo - 15 : it.lo)) {
      const int slot = t / p.c.page_size, place = t - slot * p.c.page_size;
      const int page = p.c.table[(int64_t)it.seq * p.c.ldt + slot];
      if (page >= 0 && page < p.c.n_pages) {
        base = (int64_t)page * p.c.page_stride + (int64_t)place * p.c.place_stride;
        srow = ((int64_t)page * p.c.kv_heads + head) * p.c.page_size + place;
        if constexpr (kCodes) {
          const int64_t rows = (int64_t)p.c.n_pages * p.c.kv_heads * p.c.page_size;
          const int nb = (p.c.d + kCkptBlock - 1) / kCkptBlock;
          last = (rows - srow - (P16 ? 15 : 0)) * nb < kRowBytes;
        }
      }
    }
  }
  // Scale bytes of column blocks: a lane's columns of V in chunk c are of block
  // vblock(c).
  __device__ __forceinline__ int vblock(int c) const { return (c * 16 * VE + q * VE) / kCkptBlock; }
  // Where the byte of row r (of four) and block b is: two rows to a word in groups
  // of 64 columns (they are loaded together), else words of its own (b / 4 is the
  // chunk at the largest width).
  static constexpr int vword(int r, int c) { return VW == 2 ? r / 2 : KW == 2 ? r * 2 + c : r; }
  static __device__ __forceinline__ int vshift(int r, int b) { return 8 * (VW == 2 ? r % 2 * 2 + b : b % 4); }
  __device__ __forceinline__ uint8_t kscale(const Tile& x, int u, int c) const {
    if constexpr (!kCodes) return 0;
    // (64 columns a load of the four lanes, two blocks; bytes past the row's are
    // another row's, and 0 times what they stand for may not be 0)
    constexpr int S = KL / KE;
    const int word = c / S / 2, past = (p.c.d + kCkptBlock - 1) / kCkptBlock - 4 * word;
    const uint32_t mask = PAGES == PAGES_GROUPS || past >= 4 ? ~0u : past <= 0 ? 0u : (1u << (8 * past)) - 1;
    return (uint8_t)((x.ks[u][word] & mask) >> (16 * (c / S % 2) + 8 * (g >> 1)));
  }
  __device__ __forceinline__ uint8_t vscale(const Tile& x, int i, int c) const {
    if constexpr (!kCodes) return 0;
    return (uint8_t)(x.vs[i / 4][vword(i % 4, c)] >> vshift(i % 4, vblock(c)));
  }

  // Finds the tile's tokens; at position w of the window.
  __device__ __forceinline__ void find(Tile& x, int tile) {
    find_pages(tile);
    const int w = tile - window, t0 = tile * TILE;
    x.at = tile, x.w = w;
    if constexpr (P16) {
      x.ok = lane_i64(base, w * NG) >= 0 ? 0xFFFFu : 0u;
      if (NG > 1) x.ok |= lane_i64(base, w * NG + 1) >= 0 ? 0xFFFF0000u : 0u;
    } else {
      x.ok = (uint32_t)(__ballot(base >= 0) >> (w * TILE)) & (uint32_t)((1ull << TILE) - 1);
    }
    x.edge = kCodes && (__ballot(last) >> (P16 ? w * NG : w * TILE)) & ((1ull << (P16 ? NG : TILE)) - 1);
    x.full = x.ok == (uint32_t)((1ull << TILE) - 1) && t0 >= it.lo_all && t0 + TILE <= it.hi_all;
  }
  // 0 where token `tok` of the tile is one that some row sees, else kNone (for an
  // offset past every buffer: such loads give 0).
  __device__ __forceinline__ uint32_t unseen(const Tile& x, int tok) const {
    const int t = x.at * TILE + tok;
    return (x.ok >> tok & 1) && t >= it.lo && t < it.hi ? 0u : kNone;
  }

  // The scale bytes of one row as whole words.  Where a row has fewer bytes, the
  // rest are the next row's; one by one, where it is not sure that there is a next
  // row, or this one.
  static constexpr int kRowBytes = NB == 2 ? 2 : 4 * KW;
  template <bool FAST>
  __device__ __forceinline__ void row_scales(const uint8_t* scales, int64_t row, bool in, uint32_t* out) const {
    const int nb = (p.c.d + kCkptBlock - 1) / kCkptBlock;
    const uint8_t* at = scales + row * nb;
    if constexpr (FAST) {
      if constexpr (NB == 2) {
        out[0] = *reinterpret_cast<const u16_any*>(at);
      } else {
#pragma unroll
        for (int i = 0; i < KW; ++i) out[i] = (*reinterpret_cast<const u32x1_any*>(at + 4 * i))[0];
      }
    } else {
#pragma unroll
      for (int i = 0; i < KW; ++i) out[i] = 0;
#pragma unroll
      for (int i = 0; i < NB; ++i)
        if (in && i < nb) out[i / 4] |= (uint32_t)at[i] << (8 * (i % 4));
    }
  }

  // P16: a buffer starts at the group, and a lane's offsets never change (past
  // head_dim they are kNone, for 0); else a lane's tokens' places come from the
  // lanes that looked them up, and columns past head_dim are loaded from inside the
  // row (kfrag clears them).  FAST: a full tile; its loads have no branches
  // between them, else they would wait for one another.  (PAGES_GROUPS has none in
  // any tile.)
  template <bool FAST>
  __device__ __forceinline__ void k_rows(Tile& x) const {
    const int nb = (p.c.d + kCkptBlock - 1) / kCkptBlock, w = x.w;
#pragma unroll
    for (int u = 0; u < NG; ++u) {
      uint32_t no = 0;
      if (!FAST && !x.full) no = unseen(x, u * 16 + q);
      if constexpr (P16) {
        const Buffer b(kbase() + lane_i64(base, w * NG + u) * ES);
        if (!kCodes || p.c.d % 16 == 0) {
#pragma unroll
          for (int c = 0; c < KN; ++c) b.load(x.k[u][c], koff[c] | no);
        } else {
          // (codes that end inside a load)
#pragma unroll
          for (int c = 0; c < KN; ++c) {
            u32x2_any lo, hi;
            b.load(lo, koff[c] | no);
            b.load(hi, (koff[c] + 8) | no | ((c * 4 + g) * KL + 8 < p.c.d ? 0u : kNone));
            x.k[u][c][0] = lo[0], x.k[u][c][1] = lo[1], x.k[u][c][2] = hi[0], x.k[u][c][3] = hi[1];
          }
        }
        if constexpr (kCodes) {
          const int64_t row = lane_i64(srow, w * NG + u);
          if constexpr (PAGES == PAGES_GROUPS) {
            const Buffer sb(p.c.k_scales + row * nb);
#pragma unroll
            for (int i = 0; i < KW; ++i) x.ks[u][i] = NB == 2 ? sb.load2(q * 2 | no) : sb.load4((q * NB + 4 * i) | no);
          } else {
            row_scales<FAST>(p.c.k_scales, row + q, !no, x.ks[u]);
          }
        }
      } else {
        const uint8_t* kb = kbase() + shfl_i64(base, w * TILE + u * 16 + q) * ES;
        if constexpr (FAST) {
          if (!kCodes || p.c.d % 16 == 0) {
#pragma unroll
            for (int c = 0; c < KN; ++c) x.k[u][c] = *reinterpret_cast<const KRaw*>(kb + kin(c, 0, KL));
          } else {
#pragma unroll
            for (int c = 0; c < KN; ++c) {
              const u32x2_any lo = *reinterpret_cast<const u32x2_any*>(kb + kin(c, 0, 8));
              const u32x2_any hi = *reinterpret_cast<const u32x2_any*>(kb + kin(c, 8, 8));
              x.k[u][c][0] = lo[0], x.k[u][c][1] = lo[1], x.k[u][c][2] = hi[0], x.k[u][c][3] = hi[1];
            }
          }
        } else {
#pragma unroll
          for (int c = 0; c < KN; ++c) {
            x.k[u][c] = {};
            if constexpr (kCodes) {
#pragma unroll
              for (int h = 0; h < KL; h += 8) {
                u32x2_any v = {};
                if (!no && (c * 4 + g) * KL + h < p.c.d) v = *reinterpret_cast<const u32x2_any*>(kb + kin(c, h, 8));
                x.k[u][c][h / 4] = v[0], x.k[u][c][h / 4 + 1] = v[1];
              }
            } else {
              if (!no && (c * 4 + g) * KL < p.c.d) x.k[u][c] = *reinterpret_cast<const KRaw*>(kb + kin(c, 0, KL));
            }
          }
        }
        if constexpr (kCodes) row_scales<FAST>(p.c.k_scales, shfl_i64(srow, w * TILE + u * 16 + q), !no, x.ks[u]);
      }
    }
  }
  // Byte offset in a row of `n` of this lane's columns of load c from its h-th, or
  // of the row's last n.
  __device__ __forceinline__ uint32_t kin(int c, int h, int n) const {
    return (uint32_t)min((c * 4 + g) * KL + h, p.c.d - n) * ES;
  }

  template <bool FAST>
  __device__ __forceinline__ void v_rows(Tile& x) const {
    const int nb = (p.c.d + kCkptBlock - 1) / kCkptBlock, w = x.w;
#pragma unroll
    for (int u = 0; u < NG; ++u) {
      uint32_t no[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) no[r] = 0;
      if (!FAST && !x.full) {
#pragma unroll
        for (int r = 0; r < 4; ++r) no[r] = unseen(x, u * 16 + g * 4 + r);
      }
      if constexpr (P16) {
        const Buffer b(vbase() + lane_i64(base, w * NG + u) * ES);
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int c = 0; c < VC; ++c) b.load(x.v[c][u * 4 + r], voff[c][r] | no[r]);
        if constexpr (kCodes) {
          const int64_t row = lane_i64(srow, w * NG + u);
          const Buffer sb(p.c.v_scales + row * nb);
          if constexpr (PAGES == PAGES_GROUPS) {
            // (also of rows that nobody sees: add_values clears those)
#pragma unroll
            for (int i = 0; i < VW / 2; ++i) {
              u32x2_any two;
              sb.load(two, (g * 4 * NB + 8 * i) | (x.ok >> (16 * u) & 1 ? 0u : kNone));
              x.vs[u][2 * i] = two[0], x.vs[u][2 * i + 1] = two[1];
            }
          } else if constexpr (VW == 2) {
            x.vs[u][0] = x.vs[u][1] = 0;
#pragma unroll
            for (int r = 0; r < 4; ++r)
              x.vs[u][r / 2] |= sb.load1(((g * 4 + r) * nb + vblock(0)) | no[r] | (voff[0][r] & kNone))
                                << vshift(r, vblock(0));
          } else {
#pragma unroll
            for (int r = 0; r < 4; ++r) row_scales<FAST>(p.c.v_scales, row + g * 4 + r, !no[r], &x.vs[u][r * KW]);
          }
        }
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int i = u * 4 + r, from = w * TILE + u * 16 + g * 4 + r;
          const uint8_t* vb = vbase() + shfl_i64(base, from) * ES;
#pragma unroll
          for (int c = 0; c < VC; ++c) {
            const uint8_t* at = vb + (uint32_t)min(c * 16 * VE + q * VE, p.c.d - VE) * ES;
            if constexpr (FAST) {
              x.v[c][i] = *reinterpret_cast<const VRaw*>(at);
            } else {
              x.v[c][i] = {};
              if (!no[r]) x.v[c][i] = *reinterpret_cast<const VRaw*>(at);
            }
          }
          if constexpr (kCodes) row_scales<FAST>(p.c.v_scales, shfl_i64(srow, from), !no[r], &x.vs[u][r * KW]);
        }
      }
    }
  }
  __device__ __forceinline__ void load_k(Tile& x) const {
    if (PAGES != PAGES_GROUPS && x.full && !x.edge) k_rows<true>(x);
    else k_rows<false>(x);
  }
  __device__ __forceinline__ void load_v(Tile& x) const {
    if (PAGES != PAGES_GROUPS && x.full && !x.edge) v_rows<true>(x);
    else v_rows<false>(x);
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
      const float s = scale_of(kscale(x, u, c));
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = pair_bf16(x.k[u][c / 2][c % 2 * 2 + i / 2], s, i % 2);
    } else if constexpr (CACHE == CACHE_CODES_F32) {
      float v4[8];
      ckpt_values(make_uint2(x.k[u][c / 4][c % 4], 0), kscale(x, u, c), v4);
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = __float_as_uint(v4[i]);
    } else {
      f = x.k[u][c];
    }
    // (Q is 0 past head_dim, but 0 times an infinity is not)
    if (!P16 && kcol(c) >= p.c.d) f = Frag{};
    return f;
  }
  // Columns of token slot i as loaded from memory, in the product's type.
  typedef uint32_t VWords __attribute__((ext_vector_type(kF32 ? VE : VE / 2)));
  __device__ __forceinline__ VWords vwords(const Tile& x, int i, int c) const {
    VWords f;
    if constexpr (CACHE == CACHE_CODES_BF16) {
      const float s = scale_of(vscale(x, i, c));
#pragma unroll
      for (int j = 0; j < VE / 4; ++j) {
        f[2 * j] = pair_bf16(x.v[c][i][j], s, false);
        f[2 * j + 1] = pair_bf16(x.v[c][i][j], s, true);
      }
    } else if constexpr (CACHE == CACHE_CODES_F32) {
      float v8[8];
      ckpt_values(make_uint2(x.v[c][i][0], VE == 8 ? x.v[c][i][VE / 4 - 1] : 0), vscale(x, i, c), v8);
#pragma unroll
      for (int j = 0; j < VE; ++j) f[j] = __float_as_uint(v8[j]);
    } else {
      f = x.v[c][i];
    }
    return f;
  }
  static __device__ __forceinline__ float velem(const VWords& f, int j) {
    if constexpr (kF32) return __uint_as_float(f[j]);
    else return __uint_as_float((j & 1) ? (f[j / 2] & 0xFFFF0000u) : (f[j / 2] << 16));
  }

  // ---- one tile: scores, then weights, then the sums of values
  __device__ __forceinline__ void scores(const Tile& x, float (&pr)[RT][VT]) const {
#pragma clang fp contract(off)   // a score is rounded before the maximum is taken from it
#pragma unroll
    for (int u = 0; u < NG; ++u) {
      floatx4 s[RT];
#pragma unroll
      for (int t = 0; t < RT; ++t) s[t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        const Frag f = kfrag(x, u, c);
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          const Frag y = query(t, c);
          if constexpr (kF32) {
#pragma unroll
            for (int i = 0; i < KE; ++i)
              s[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(f[i]), __uint_as_float(y[i]), s[t], 0,
                                                          0, 0);
          } else {
            s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f),
                                                           __builtin_bit_cast(bf16x8, y), s[t], 0, 0, 0);
          }
        }
      }
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) pr[t][u * 4 + r] = s[t][r] * p.a.scale;
    }
  }

  // The least weight: 0 where rows may see different tokens (what is not finite there
  // does not come to the products); where one new token's rows do not see a token, its
  // values are 0.  (Codes have no infinity.)
  static __device__ __forceinline__ float least(bool all) { return all || !MANY ? kLeast : 0.f; }
  __device__ __forceinline__ void weights(float (&pr)[RT][VT], int tile, uint32_t okay, bool all) {
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      if (!all) {
#pragma unroll
        for (int i = 0; i < VT; ++i) {
          const int tok = (i / 4) * 16 + g * 4 + i % 4, at = tile * TILE + tok;
          const bool vis = (okay >> tok & 1) && at <= lim[t] && at > low[t];
          pr[t][i] = vis ? pr[t][i] : -INFINITY;
          seen[t] |= (uint32_t)vis;
        }
      } else {
        seen[t] = 1;
      }
      float mx = pr[t][0];
#pragma unroll
      for (int i = 1; i < VT; ++i) mx = fmaxf(mx, pr[t][i]);
      mx = fmaxf(m[t], row_max(mx));
      const float mu = mx == -INFINITY ? 0.f : mx;
      if (__any(mx > m[t])) {
        const float scale = rescale(m[t], mu);
        l[t] *= scale;
#pragma unroll
        for (int n = 0; n < NO; ++n) o[t][n] *= scale;
        m[t] = mx;
      }
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < VT; ++i) {
        const float w = exp_diff(pr[t][i], mu);
        sum += w;
        pr[t][i] = kCodes ? w : fmaxf(w, least(all));
      }
      l[t] += sum;
    }
  }

  __device__ __forceinline__ void add_values(Tile& x, const float (&pr)[RT][VT], int tile, uint32_t okay, bool all) {
    if (kCodes && PAGES == PAGES_GROUPS && !all) {
      // scales of rows that nobody sees (0 times what they stand for may not be 0)
#pragma unroll
      for (int i = 0; i < VT; ++i) {
        const int tok = (i / 4) * 16 + g * 4 + i % 4, at = tile * TILE + tok;
        const bool some = (okay >> tok & 1) && at >= it.lo && at < it.hi;
        uint32_t* w = &x.vs[i / 4][vword(i % 4, 0)];
        if constexpr (VW == 2) {
          w[0] &= some ? ~0u : i % 2 ? 0xFFFFu : 0xFFFF0000u;
        } else {
#pragma unroll
          for (int j = 0; j < KW; ++j) w[j] = some ? w[j] : 0u;
        }
      }
    }
    if (MANY && !all) {
      // Rows that see different tokens: a value that is not finite must not
      // reach, as 0 times itself, a row that does not see it.
      uint32_t bad = 0;
#pragma unroll
      for (int c = 0; c < VC; ++c)
#pragma unroll
        for (int i = 0; i < VT; ++i) {
          const VWords f = vwords(x, i, c);
#pragma unroll
          for (int j = 0; j < VE; ++j) bad |= (__float_as_uint(velem(f, j)) & 0x7F800000u) == 0x7F800000u;
        }
      if (__any(bad)) {
        infinities(x, tile, okay);
        clear_infinities(x);
      }
    }
    values(x, pr, all);
  }

  // What values that are not finite add to the rows that see them: a weight is
  // above 0, so an infinity gives itself, and a NaN counts as both infinities.
  __device__ __forceinline__ void infinities(const Tile& x, int tile, uint32_t okay) {
    float sees[RT][VT];
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int i = 0; i < VT; ++i) {
        const int tok = (i / 4) * 16 + g * 4 + i % 4, at = tile * TILE + tok;
        sees[t][i] = (okay >> tok & 1) && at <= lim[t] && at > low[t] ? 1.f : 0.f;
      }
#pragma unroll
    for (int c = 0; c < VC; ++c)
#pragma unroll
      for (int j = 0; j < VE; ++j) {
        float up[VT], down[VT];
        __builtin_amdgcn_sched_barrier(0);   // (one column at a time: this path is rare, its registers are not free)
#pragma unroll
        for (int i = 0; i < VT; ++i) {
          const float e = velem(vwords(x, i, c), j);
          up[i] = !(e <= 3.4028235e38f) ? 1.f : 0.f;
          down[i] = !(e >= -3.4028235e38f) ? 1.f : 0.f;
        }
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          const floatx4 zero{0.f, 0.f, 0.f, 0.f};
          const floatx4 a = sum_tokens(up, sees[t], zero), b = sum_tokens(down, sees[t], zero);
#pragma unroll
          for (int r = 0; r < 4; ++r) o[t][c * VE + j][r] += (a[r] > 0.f ? INFINITY : 0.f) - (b[r] > 0.f ? INFINITY : 0.f);
        }
      }
  }
  static __device__ __forceinline__ floatx4 sum_tokens(const float (&a)[VT], const float (&b)[VT], floatx4 acc) {
    if constexpr (kF32) {
#pragma unroll
      for (int i = 0; i < VT; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], acc, 0, 0, 0);
    } else {
      bf16x8 x, y;
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = (__bf16)a[i], y[i] = (__bf16)b[i];
      acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, acc, 0, 0, 0);
    }
    return acc;
  }
  // Sets such values to 0, where they are.
  __device__ __forceinline__ void clear_infinities(Tile& x) {
#pragma unroll
    for (int c = 0; c < VC; ++c)
#pragma unroll
      for (int i = 0; i < VT; ++i) {
        constexpr int W = VE * ES / 4;
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (kCodes) {
          const bool all = vscale(x, i, c) == 255;
#pragma unroll
          for (int j = 0; j < W; ++j) {
            uint32_t w = x.v[c][i][j];
#pragma unroll
            for (int b = 0; b < 32; b += 8)
              if (all || (w >> b & 0x7F) == 0x7F) w &= ~(0xFFu << b);
            x.v[c][i][j] = w;
          }
        } else {
#pragma unroll
          for (int j = 0; j < W; ++j) {
            uint32_t w = x.v[c][i][j];
            if (kF32) {
              if ((w & 0x7F800000u) == 0x7F800000u) w = 0;
            } else {
              if ((w & 0x7F80u) == 0x7F80u) w &= 0xFFFF0000u;
              if ((w & 0x7F800000u) == 0x7F800000u) w &= 0xFFFFu;
            }
            x.v[c][i][j] = w;
          }
        }
      }
    if constexpr (kCodes) {
      // (0 times the scale of byte 255 is not 0)
#pragma unroll
      for (int u = 0; u < NG; ++u)
#pragma unroll
        for (int i = 0; i < VW; ++i)
#pragma unroll
          for (int b = 0; b < 32; b += 8)
            if ((x.vs[u][i] >> b & 0xFF) == 0xFF) x.vs[u][i] &= ~(0x80u << b);
    }
  }

  // O += V^T P^T.  A weight meets bf16 values as two bf16 numbers, the second being
  // what rounding takes from it (then 2^-16 of it).  Where reading the cache bounds the
  // kernel the products are free; where they bound it, fewer bits were faster, us with
  // two numbers | one: prompts of 2048 tokens 181 | 172, 512 of 4096 305 | 294, of an 8-bit
  // cache 196 | 173 and 324 | 278; 8 tokens of 8 heads a key head 251 | 231 (274 with the
  // least weight).  One number
  // leaves 2^-8 of a weight: an error against 64 bits of 2.0e-3 for 1.65e-3, the
  // output's own rounding.  The first number is cut, not rounded, and the second at
  // least the least weight: neither is below 0, nor 0 where a value may be infinite.
  __device__ __forceinline__ void values(const Tile& x, const float (&pr)[RT][VT], bool all) {
    if constexpr (kF32) {
#pragma unroll
      for (int i = 0; i < VT; ++i)
#pragma unroll
        for (int c = 0; c < VC; ++c) {
          const VWords f = vwords(x, i, c);
#pragma unroll
          for (int j = 0; j < VE; ++j)
#pragma unroll
            for (int t = 0; t < RT; ++t)
              o[t][c * VE + j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(f[j]), pr[t][i],
                                                                      o[t][c * VE + j], 0, 0, 0);
        }
    } else {
      bf16x8 pf[RT], rest[RT];
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float cut = __uint_as_float(__float_as_uint(pr[t][i]) & 0xFFFF0000u);
          pf[t][i] = (__bf16)cut;
          rest[t][i] = (__bf16)(kCodes ? pr[t][i] - cut : fmaxf(pr[t][i] - cut, least(all)));
        }
#pragma unroll
      for (int c = 0; c < VC; ++c) {
        VWords f[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = vwords(x, i, c);
#pragma unroll
        for (int j = 0; j < VE; ++j) {
          Frag a;
#pragma unroll
          for (int i = 0; i < 4; ++i)
            a[i] = __builtin_amdgcn_perm(f[2 * i + 1][j / 2], f[2 * i][j / 2], (j & 1) ? 0x07060302u : 0x05040100u);
#pragma unroll
          for (int t = 0; t < RT; ++t) {
            o[t][c * VE + j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), pf[t],
                                                                       o[t][c * VE + j], 0, 0, 0);
            o[t][c * VE + j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), rest[t],
                                                                       o[t][c * VE + j], 0, 0, 0);
          }
        }
      }
    }
  }

  // Two tiles where they are small: a wave should have 8 KB on their way while it
  // computes.
  static constexpr bool kDouble = TILE * D * ES <= 4096 && (D == 64 || !MANY);

  __device__ __forceinline__ void load(Tile& x, int tile) {
    find(x, tile);
    load_k(x);
    load_v(x);
  }
  __device__ __forceinline__ void compute(Tile& x) {
    float pr[RT][VT];
    scores(x, pr);
    weights(pr, x.at, x.ok, x.full);
    add_values(x, pr, x.at, x.ok, x.full);
  }
  // Whether the lane's row saw a token.  (In tiles that all rows see, those that see
  // nothing go along.  Asked here: in the loop 8 new tokens of 64 rows a key head took
  // 587 us for 251.)
  __device__ __forceinline__ bool any_seen(int t) const { return row_max((float)seen[t]) > 0.f && lim[t] >= 0; }
  // The item's sums to LDS: 16 rows of STRIDE.
  __device__ __forceinline__ void put_sums(int t, float* to) const {
#pragma unroll
    for (int c = 0; c < VC; ++c)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int j = 0; j < VE; j += 4)
          *reinterpret_cast<floatx4*>(to + q * STRIDE + c * 16 * VE + (4 * g + r) * VE + j) =
              floatx4{o[t][c * VE + j][r], o[t][c * VE + j + 1][r], o[t][c * VE + j + 2][r], o[t][c * VE + j + 3][r]};
  }
  // Of one wave that had the item to itself: through its own part of LDS, to whole
  // rows.
  __device__ __forceinline__ void finish(const Item& item, float* to) {
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      put_sums(t, to + t * 16 * STRIDE);
      const float sum = row_sum(l[t]);
      l[t] = any_seen(t) ? sum : -1.f;
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int at = i * 4 + g, row = t * 16 + at, col = q * NO;
        const float mr = __shfl(m[t], at), lr = __shfl(l[t], at);
        if (row < item.nrows) {
          float v[NO];
#pragma unroll
          for (int c = 0; c < NO; ++c) v[c] = to[row * STRIDE + col + c];
          finish_row<T, NO>(p, item, head, row, col, mr, lr, v);
        }
      }
  }
  __device__ __forceinline__ void tiles(int from, int to) {
    if (from >= to) return;
    Tile a;
    load(a, from);
    if constexpr (kDouble) {
      Tile b;
      for (int t = from;; t += 2) {
        if (t + 1 < to) load(b, t + 1);
        compute(a);
        if (t + 1 >= to) return;
        if (t + 2 < to) load(a, t + 2);
        compute(b);
        if (t + 2 >= to) return;
      }
    } else {
      for (int t = from; t < to; ++t) {
        const uint32_t okay = a.ok;
        const bool all = a.full;
        float pr[RT][VT];
        scores(a, pr);
        if (t + 1 < to) {
          find(a, t + 1);
          load_k(a);
        }
        weights(pr, t, okay, all);
        add_values(a, pr, t, okay, all);
        if (t + 1 < to) load_v(a);
      }
    }
  }
};

template <int CACHE, int D, int RT, int PAGES, int NEW>
__global__ __launch_bounds__(64 * kAttnWaves, attn_groups_per_cu(D, RT)) void attention_kernel(AttnPlan p) {
  typedef Attn<CACHE, D, RT, PAGES, NEW> A;
  typedef typename A::T T;
  __shared__ __align__(16) float rows[kAttnWaves][A::R][A::STRIDE];
  __shared__ __align__(16) typename A::Frag queries[A::kQShared ? RT * A::KC * 64 : 1];
  __shared__ float2 stats[kAttnWaves][A::R];
  __shared__ int64_t scan[kAttnWaves];
  __shared__ int64_t found[2];   // first item | its first tile

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int head = (int)(blockIdx.x % p.c.kv_heads), worker = (int)(blockIdx.x / p.c.kv_heads);
  int item = worker;
  if constexpr (NEW == NEW_PROMPT) {
    // a wave an item; those that read most first
    item = p.items - 1 - (worker * kAttnWaves + wave);
    if (item < 0) return;
  }
  int64_t at = 0, total = 0, left;     // slot `at` of the item; slots left of this part
  int64_t part0 = 0;
  int parts = 0;
  int length = 0;      // of lane i's sequence, where there are at most 64 items of one row group
  const bool few = p.items <= 64 && p.row_groups == 1;
  if (p.workers && few) {
    if (lane < p.items) length = p.a.lengths[lane];
    const int64_t mine = lane < p.items ? item_of<A::TILE, A::R>(p, lane, length).slots : 0;
    int64_t incl = mine;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int64_t v = shfl_i64(incl, lane - d < 0 ? lane : lane - d);
      if (lane >= d) incl += v;
    }
    total = lane_i64(incl, 63);
    parts = (int)min((int64_t)p.workers, (total + kAttnMinTiles - 1) / kAttnMinTiles);
    if (worker >= parts) return;
    part0 = worker * total / parts;
    left = (worker + 1) * total / parts - part0;
    item = __builtin_ctzll(__ballot(part0 < incl));
    at = part0 - lane_i64(incl - mine, item);
  } else if (p.workers) {
    // slots before each thread's items
    const int per = (p.items + 255) / 256, i0 = min(tid * per, p.items), i1 = min(i0 + per, p.items);
    int64_t mine = 0;
    for (int i = i0; i < i1; ++i) mine += item_of<A::TILE, A::R>(p, i).slots;
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
        const int n = item_of<A::TILE, A::R>(p, i).slots;
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

  A s(p, lane, head, queries);
  while (left > 0) {
    const Item it = p.workers && few ? item_of<A::TILE, A::R>(p, item, lane_i(length, item)) : item_of<A::TILE, A::R>(p, item);
    const int from = (int)at;
    const int take = p.workers ? (int)min((int64_t)(it.slots - from), left) : it.slots;
    const int n = min(from + take, it.tiles) - from;
    const bool whole = n == it.tiles;
    left -= p.workers ? take : 1;
    const int64_t start = part0;
    part0 += take;
    at = 0;
    ++item;
    if (n <= 0) continue;    // (slots behind the last tile)
    s.begin(it, wave);
    if constexpr (NEW == NEW_PROMPT) {
      s.tiles(it.first, it.first + it.tiles);
      s.finish(it, &rows[wave][0][0]);
      return;
    }
    if constexpr (A::kQShared) __syncthreads();
    s.tiles(it.first + from + (int)((int64_t)n * wave / kAttnWaves),
            it.first + from + (int)((int64_t)n * (wave + 1) / kAttnWaves));
    if (p.workers && from == 0 && head == 0 && tid == 0) {
      // the parts that hold this item: the last part that starts at or before a tile
      const int64_t t0 = start, t1 = start + it.tiles - 1;
      p.span[item - 1] = make_int2((int)(((t0 + 1) * parts - 1) / total), (int)(((t1 + 1) * parts - 1) / total));
    }
    // the four waves' sums: all of them to LDS, then a loop over the row tiles (not
    // unrolled: what runs once an item waits for its instructions to be fetched)
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      s.put_sums(t, &rows[wave][t * 16][0]);
      const float l = row_sum(s.l[t]);
      const bool seen = s.any_seen(t);
      if (s.g == 0) stats[wave][t * 16 + s.q] = make_float2(s.m[t], seen ? l : -1.f);
    }
    __syncthreads();
    constexpr int N = D / 16;
    const int col = (tid & 15) * N;
#pragma unroll 1
    for (int row = tid >> 4; row < it.nrows; row += 16) {
      float m = -INFINITY, sum = 0.f, o[N];
      bool any = false;
#pragma unroll
      for (int w = 0; w < kAttnWaves; ++w) m = fmaxf(m, stats[w][row].x);
#pragma unroll
      for (int c = 0; c < N; ++c) o[c] = 0.f;
#pragma unroll
      for (int w = 0; w < kAttnWaves; ++w) {
        const float2 st = stats[w][row];
        const float e = rescale(st.x, m);
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
        finish_row<T, N>(p, it, head, row, col, m, sum, o);
      } else {
        const int64_t pr = (((int64_t)worker * p.c.kv_heads + head) * 2 + (from == 0 ? 1 : 0)) * A::R + row;
#pragma unroll
        for (int c = 0; c < N; c += 4)
          *reinterpret_cast<floatx4*>(p.part + pr * D + col + c) = floatx4{o[c], o[c + 1], o[c + 2], o[c + 3]};
        if (col == 0) p.stat[pr] = make_float2(m, sum);
      }
    }
    __syncthreads();
  }
}

// A sum over parts: m, l (with `any` of them), o.
struct Sum {
  float m, l;
  floatx4 o;
  bool any;
  __device__ __forceinline__ void add(float m2, float l2, floatx4 o2, bool any2) {
    const float top = fmaxf(m, m2);
    const float a = rescale(m, top), b = rescale(m2, top);
    l = a * l + b * l2, o = a * o + b * o2, m = top, any |= any2;
  }
};

// Rows of items that several parts hold, ROWS to a workgroup: four, a wave each,
// or one where there are many parts to an item.  A row's columns are D / 4 lanes;
// so many sets of them take the parts in turn, four at once (the loads do not
// wait for one another); the sets are added in a fixed order.
template <typename T, int D, int R, int ROWS>
__global__ __launch_bounds__(256) void attention_join_kernel(AttnPlan p, int blocks) {
  constexpr int LANES = D / 4, SETS = 256 / ROWS / LANES, BATCH = 4;
  __shared__ float4 sums[ROWS][SETS][LANES];
  __shared__ float3 stats[ROWS][SETS];
  const int64_t id = blockIdx.x;
  const int sub = threadIdx.x / (256 / ROWS), row = (int)(id % blocks) * ROWS + sub;
  const int head = (int)(id / blocks % p.c.kv_heads), item = (int)(id / blocks / p.c.kv_heads);
  const int seq = p.row_groups == 1 ? item : item / p.row_groups, row0 = (item - seq * p.row_groups) * R;
  const int2 span = p.span[item];
  if (span.x == span.y) return;
  const int n = row < min(R, p.rows - row0) ? span.y - span.x + 1 : 0;
  const int set = threadIdx.x % (256 / ROWS) / LANES, lane = threadIdx.x % LANES, col = lane * 4;
  Sum s{-INFINITY, 0.f, floatx4{0.f, 0.f, 0.f, 0.f}, false};
  for (int i0 = 0; i0 < n; i0 += SETS * BATCH) {
    float2 st[BATCH];
    floatx4 v[BATCH];
#pragma unroll
    for (int j = 0; j < BATCH; ++j) {
      const int i = i0 + j * SETS + set;
      st[j] = make_float2(-INFINITY, -1.f), v[j] = floatx4{0.f, 0.f, 0.f, 0.f};
      if (i < n) {
        const int64_t r = (((int64_t)(span.x + i) * p.c.kv_heads + head) * 2 + (i == 0 ? 1 : 0)) * R + row;
        st[j] = p.stat[r];
        v[j] = *reinterpret_cast<const floatx4*>(p.part + r * D + col);
      }
    }
#pragma unroll
    for (int j = 0; j < BATCH; ++j) {
      const bool none = st[j].y < 0.f;
      s.add(st[j].x, none ? 0.f : st[j].y, v[j], !none);
    }
  }
  const int sets = min(SETS, n);
  if (set > 0 && set < sets) {
    sums[sub][set][lane] = make_float4(s.o[0], s.o[1], s.o[2], s.o[3]);
    if (lane == 0) stats[sub][set] = make_float3(s.m, s.l, s.any ? 1.f : 0.f);
  }
  __syncthreads();
  if (set > 0 || col >= p.c.d || n == 0) return;
  for (int i = 1; i < sets; ++i) {
    const float4 o = sums[sub][i][lane];
    s.add(stats[sub][i].x, stats[sub][i].y, floatx4{o.x, o.y, o.z, o.w}, stats[sub][i].z > 0.f);
  }
  const int q = row0 + row, i = q / p.group, h = head * p.group + q - i * p.group;
  const int64_t tok = (int64_t)seq * p.a.n_new + i;
  if (lane == 0 && p.a.lse)
    p.a.lse[tok * p.a.q_heads + h] = s.any ? lse_of(s.m, s.l) : -INFINITY;
  T out[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) out[j] = from_f32<T>(s.any ? quotient(s.o[j], s.l) : 0.f);
  memcpy((T*)p.a.out.p + tok * p.a.out.ts + h * p.a.out.hs + col, out, sizeof(out));
}

}  // namespace

template <int CACHE, int D, int RT, int PAGES, int NEW>
hipError_t run_attention(const AttnPlan& p, hipStream_t s) {
  typedef Attn<CACHE, D, RT, PAGES, NEW> A;
  const int64_t parts = p.workers ? p.workers : NEW == NEW_PROMPT ? (p.items + kAttnWaves - 1) / kAttnWaves : p.items;
  const int64_t groups = parts * p.c.kv_heads;
  launch_k(attention_kernel<CACHE, D, RT, PAGES, NEW>, dim3((unsigned)groups), 64 * kAttnWaves, 0, s, p);
  if (p.workers) {
    const int nrows = p.rows < A::R ? p.rows : A::R;
    auto join = [&](auto kernel, int rows) {
      const int blocks = (nrows + rows - 1) / rows;
      launch_k(kernel, dim3((unsigned)((int64_t)p.items * p.c.kv_heads * blocks)), 256, 0, s, p, blocks);
    };
    // (512 parts of one item, 8 rows: 15 us with a row a workgroup, 45 with four; 32
    // items of two or three parts, 32 rows, 8 heads: 6 us with four, 13 with one)
    if (p.workers > 8 * p.items) join(attention_join_kernel<typename A::T, D, A::R, 1>, 1);
    else join(attention_join_kernel<typename A::T, D, A::R, 4>, 4);
  }
  return hipGetLastError();
}

}  // namespace fs
