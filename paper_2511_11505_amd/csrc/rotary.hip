// Rotary positions, their backward pass, and the append to a paged cache.
//
// Pair (a, b) at angle t = position * f becomes (c a - s b, c b + s a) with c =
// m cos t and s = m sin t; the backward pass is the transposed turn, s with its
// sign changed.  Angles are products in 64 bits (at position 10^6 a 32-bit
// product is off by 0.03 radians), reduced by quarter turns in 64 bits.
//
// Memory bounds it: a row is read once and written once, and the angles of a
// token are shared by all its heads.  A wave has one token: its lanes compute
// one angle each into LDS, then take the token's rows (q, k and v heads alike),
// 8 columns a lane and several rows at once, the cosines and sines of their
// columns in registers; a chunk's partner is exchanged between lanes (loading it
// too: 45 us for 42 at 8192 tokens of 48 heads of 128 in bf16, 52 for 43 at 4096 in
// fp32).  A row's lanes read it whole before they write, and a row is one wave's,
// so a row may be turned in place.  Three rows a lane are on their way at once;
// two or four were 2 to 6% slower.
//
// Measured (MI355X): those 8192 tokens 42 us, 4.8 TB/s, where a copy of as many
// bytes takes 40.6; the gradient of 64 of 192 columns of 4096 tokens of 128 heads 83
// us (a copy 78.8); 64 tokens of 40 + 8 + 8 heads into a cache 6.5 us, one row and the
// angles after each other.

#include "internal.hpp"
#include "saved.hpp"

#pragma clang fp contract(off)   // each product of a turn is rounded

namespace fs {
namespace {

constexpr int kMaxPairs = 256;   // rot <= 512
constexpr int kUnroll = 3;       // rows a lane has in flight

// cos and sin of t (|t| < 2^40): t less n quarter turns, by the sum of two
// 64-bit parts of pi / 2, then the Taylor series to r^15 (|r| <= pi / 4: what
// is left out is below 2^-49).
__device__ __forceinline__ void cos_sin(double t, double& c, double& s) {
  const double n = rint(t * 0.63661977236758134308);
  double r = fma(-n, 1.57079632679489655800, t);
  r = fma(-n, 6.12323399573676603587e-17, r);
  const double x = r * r;
  double a = -1.0 / 1307674368000.0;                    // sin: r^15 / 15!
  a = fma(a, x, 1.0 / 6227020800.0);
  a = fma(a, x, -1.0 / 39916800.0);
  a = fma(a, x, 1.0 / 362880.0);
  a = fma(a, x, -1.0 / 5040.0);
  a = fma(a, x, 1.0 / 120.0);
  a = fma(a, x, -1.0 / 6.0);
  a = fma(a * x, r, r);
  double b = -1.0 / 87178291200.0;                      // cos: r^14 / 14!
  b = fma(b, x, 1.0 / 479001600.0);
  b = fma(b, x, -1.0 / 3628800.0);
  b = fma(b, x, 1.0 / 40320.0);
  b = fma(b, x, -1.0 / 720.0);
  b = fma(b, x, 1.0 / 24.0);
  b = fma(b, x, -0.5);
  b = fma(b, x, 1.0);
  const int quarter = (int)(n - 4.0 * floor(n * 0.25));
  const double cc = (quarter & 1) ? a : b, ss = (quarter & 1) ? b : a;
  c = (quarter == 1 || quarter == 2) ? -cc : cc;
  s = (quarter & 2) ? -ss : ss;
}

// Between a wave's writes to LDS and its reads of them.
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// The rows of a token in batches of kUnroll * (64 / lanes of a row), of q, then of
// k, then of v.
struct Batches {
  int size, q, kv;   // rows of a batch; batches of q, of each of k and v
};

// FAST: chunks of 8 columns turn with a whole chunk or within themselves;
// otherwise columns take their partners one by one, from LDS (from memory: 71 us
// for 33, 8192 tokens of 48 heads of 75 in bf16).  Where 8 does not divide a head, its
// last chunk overlaps the one before it (both lanes have the same values).
template <typename T, bool FAST, bool CACHE>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs g, PagedCache pc, Batches bt, int lanes_log2,
                                                     int splits, int per_split) {
  __shared__ __align__(16) float2 table[4][kMaxPairs];
  __shared__ __align__(16) T stage[FAST ? 1 : 4][FAST ? 1 : kUnroll][FAST ? 1 : 64 * 8];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t id = blockIdx.x * 4 + wave;
  const int token = (int)(id / (uint32_t)splits);
  if (token >= g.tokens) return;
  int batch = (int)(id % (uint32_t)splits) * per_split;
  const int last = min(batch + per_split, bt.q + 2 * bt.kv);

  const int pairs = g.rope.rot / 2;
  const bool halves = g.rope.halves;
  const int per_wave = 64 >> lanes_log2, row0 = lane >> lanes_log2;
  const int chunk = (lane & ((1 << lanes_log2) - 1)) * 8;
  const int c0 = FAST ? chunk : max(min(chunk, g.d - 8), 0), n = chunk < g.d ? min(8, g.d - c0) : 0;
  uint32_t turns = 0, ahead = 0;    // bit i: column c0 + i turns; its partner is ahead
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int at = c0 + i - g.rope.first;
    turns |= (uint32_t)(i < n && at >= 0 && at < g.rope.rot) << i;
    ahead |= (uint32_t)(halves ? at < pairs : !(at & 1)) << i;
  }

  enum { Q, K, V };
  Raw8<T> own[kUnroll], other[kUnroll];
  auto fetch = [&](int part, int first, int heads) {
    const HeadRows& h = part == Q ? g.q : part == K ? g.k : g.v;
    const T* base = (const T*)h.p + (int64_t)token * h.ts + c0;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int r = first + u * per_wave + row0;
      own[u] = other[u] = {};
      if (r < heads && n > 0) own[u] = load8<T>(base + r * h.hs, n);
    }
  };
  int part, first, heads;
  auto find = [&](int b) {
    part = !CACHE || b < bt.q ? Q : b < bt.q + bt.kv ? K : V;
    first = (part == Q ? b : part == K ? b - bt.q : b - bt.q - bt.kv) * bt.size;
    heads = part == Q ? g.q_heads : g.kv_heads;
  };
  // the first rows are on their way while the angles are made
  find(batch);
  fetch(part, first, heads);

  const int pos = g.positions[token];
  bool live = true;
  int64_t page = -1;
  int place = 0;
  if constexpr (CACHE) {
    const int seq = g.seqs ? g.seqs[token] : token;
    live = pos >= 0 && seq >= 0 && seq < pc.sequences;
    if (live) {
      const int slot = pos / pc.page_size;
      place = pos - slot * pc.page_size;
      if (slot < pc.max_pages) page = pc.table[(int64_t)seq * pc.ldt + slot];
      if (page >= pc.n_pages) page = -1;
    }
  }
  for (int p = lane; p < pairs; p += 64) {
    double c, s;
    cos_sin((double)pos * g.rope.freqs[p], c, s);
    table[wave][p] = make_float2((float)(c * g.rope.mscale), (float)(s * (g.back ? -g.rope.mscale : g.rope.mscale)));
  }
  wave_fence();
  float cs[8], sn[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int at = c0 + i - g.rope.first;
    const bool a = ahead >> i & 1;
    const float2 w = (turns >> i & 1) ? table[wave][halves ? (a ? at : at - pairs) : at >> 1] : make_float2(1.f, 0.f);
    cs[i] = w.x;
    sn[i] = a ? -w.y : w.y;
  }

  const int partner = lane + ((ahead & 1) ? pairs / 8 : -(pairs / 8));   // has the chunk that this one turns with
  for (;;) {
    if constexpr (!FAST) {
      // (a wave's own part of LDS: it is served in order)
      const int step = halves ? pairs : 1;
#pragma unroll
      for (int u = 0; u < kUnroll; ++u)
        if (n > 0) memcpy(&stage[wave][u][(row0 << (lanes_log2 + 3)) + c0], own[u].w, sizeof(own[u].w));
      wave_fence();
#pragma unroll
      for (int u = 0; u < kUnroll; ++u)
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (turns >> i & 1) {
            const T v = stage[wave][u][(row0 << (lanes_log2 + 3)) + c0 + i + ((ahead >> i & 1) ? step : -step)];
            if constexpr (sizeof(T) == 4) other[u].w[i] = __float_as_uint(v);
            else other[u].w[i >> 1] |= (uint32_t)v << (16 * (i & 1));
          }
      wave_fence();
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int r = first + u * per_wave + row0;
      const bool in = r < heads && n > 0;
      if (FAST && halves && part != V) {
#pragma unroll
        for (unsigned i = 0; i < 8 * sizeof(T) / 4; ++i) other[u].w[i] = (uint32_t)__shfl((int)own[u].w[i], partner);
      }
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = own[u].get(i);
      if (part != V) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float y = FAST && !halves ? own[u].get(i ^ 1) : other[u].get(i);
          const float t = own[u].get(i) * cs[i] + y * sn[i];
          v[i] = (turns >> i & 1) ? t : v[i];
        }
      }
      if (!CACHE || part == Q) {
        if (CACHE && !live) {
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] = 0.f;
        }
        if (in) store8<T>((T*)g.out.p + (int64_t)token * g.out.ts + r * g.out.hs + c0, v, n);
      } else if (live && page >= 0) {
        uint8_t *base = (uint8_t*)(part == K ? pc.k : pc.v), *scales = part == K ? pc.k_scales : pc.v_scales;
        const int64_t at = page * pc.page_stride + r * pc.head_stride + place * pc.place_stride + c0;
        if (pc.codes) {
          const int b = ckpt_byte(block_max<LANES_NEXT>(amax8(v)));
          if (in) {
            store_codes(base + at, ckpt_codes(v, b), 8);
            if (c0 % kCkptBlock == 0)
              scales[((page * pc.kv_heads + r) * pc.page_size + place) * ((g.d + kCkptBlock - 1) / kCkptBlock) +
                     c0 / kCkptBlock] = (uint8_t)b;
          }
        } else if (in) {
          store8<T>((T*)base + at, v, 8);
        }
      }
    }
    if (++batch >= last) break;
    find(batch);
    fetch(part, first, heads);
  }
}

template <typename T>
hipError_t run(const RotaryArgs& g, const PagedCache& pc, hipStream_t s) {
  int lg = 2;
  while ((8 << lg) < g.d) ++lg;
  Batches bt;
  bt.size = (64 >> lg) * kUnroll;
  bt.q = (g.q_heads + bt.size - 1) / bt.size;
  bt.kv = (g.kv_heads + bt.size - 1) / bt.size;
  // A wave takes all of a token's rows while the tokens alone make 64 waves a
  // CU (an angle is computed once); fewer tokens are split over more waves,
  // down to one batch of rows each.
  const int batches = bt.q + 2 * bt.kv;
  int splits = (int)((16384 + g.tokens - 1) / g.tokens);
  splits = splits < batches ? splits : batches;
  const int per_split = (batches + splits - 1) / splits;
  splits = (batches + per_split - 1) / per_split;
  const bool halves = g.rope.halves;
  const bool fast = g.d % 8 == 0 && (halves ? g.rope.first % 8 == 0 && g.rope.rot % 16 == 0 : g.rope.first % 2 == 0);
  const dim3 grid((unsigned)cdiv64((int64_t)g.tokens * splits, 4));
  auto go = [&](auto kernel) { launch_k(kernel, grid, 256, 0, s, g, pc, bt, lg, splits, per_split); };
  if (g.kv_heads) fast ? go(rotary_kernel<T, true, true>) : go(rotary_kernel<T, false, true>);
  else fast ? go(rotary_kernel<T, true, false>) : go(rotary_kernel<T, false, false>);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotary(int dtype, const RotaryArgs& a, const PagedCache& c, hipStream_t s) {
  return dtype == 0 ? run<float>(a, c, s) : run<bf16_t>(a, c, s);
}

}  // namespace fs
