// The linear's bf16 products on tiles of up to 256 x 256: four waves (2 x 2),
// one per SIMD, each up to 128 x 128 through v_mfma_f32_16x16x32_bf16, 256
// accumulators in the AGPRs.
//
//   Operands  Either may lie along K (rows of K) or across it (rows of the
//             output dimension).  Both ways a 64-wide K block of 64 rows is an
//             8 KB panel of 64 LDS rows of 128 bytes, filled by eight
//             global->LDS copies of 8 rows: rows of K, or rows of 64
//             columns at one k, which the fragment reads transpose
//             (ds_read_b64_tr_b16).  The lane picks the 16-byte chunk it
//             copies so that the reads cover every bank once: along, chunk c of
//             row r sits at c ^ ((r / 2) % 8); across, the 32 bytes of columns
//             16 c .. of row k sit at c ^ s(k), s = bits 1 and 3 of k.
//             Products with few tiles take 64 x 128, two workgroups per CU, and
//             K cut into slices whose sums a second kernel adds.
//   Ring      Two 64-wide LDS slots for A, three for B (160 KB at 256
//             rows); one barrier per block.  The copies run on from tile to tile.
//   Tail      K % 64 != 0: chunks past K are copied from 16 zero bytes.
//   Edges     Rows and columns past the end are copied from the last valid ones
//             and not stored.
//   Output    The weights' side is the MFMA's row operand; neighbouring column
//             fragments exchange lane groups, so a lane holds 8 consecutive
//             output columns and stores them without staging (linear.hpp).
//   Order     Items (tile, K slice) go to the XCDs in eight contiguous ranges;
//             in a range m-tiles in bands of eight, then n-tiles, so that the
//             tiles an XCD runs together share both operands.
#pragma once

#include <type_traits>
#include <utility>

#include "gemm_common.hpp"
#include "linear.hpp"

namespace fs {
namespace {

template <typename F, int... I>
__device__ __forceinline__ void static_for_(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void static_for(F&& f) {
  static_for_(f, std::make_integer_sequence<int, N>{});
}

// global->LDS copies to a wave-uniform LDS base plus a constant, from a
// pointer per lane, or from a wave-uniform base plus an offset per lane.
template <int OFF>
__device__ __forceinline__ void copy16_ptr(const void* g, unsigned lds) {
  asm volatile("s_add_u32 m0, %0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
               :
               : "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(g), "n"(OFF)
               : "memory", "scc");
}
template <int OFF>
__device__ __forceinline__ void copy16_off(const unsigned char* base, unsigned off, unsigned lds) {
  asm volatile("s_add_u32 m0, %0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :
               : "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(off), "s"(uniform_ptr(base)), "n"(OFF)
               : "memory", "scc");
}

typedef __attribute__((address_space(3))) bf16x8 lds_b16x8_t;
typedef short tr_i16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) tr_i16x4 lds_tr_t;

__device__ const uint4 kZeroChunk = {0, 0, 0, 0};

// One operand's copies.  ROWS tile rows (a multiple of 32); copy i of a wave
// fills LDS bytes 1024 (4 i + wave) .. of the slot.
template <bool ALONG, int ROWS, bool TAIL>
struct Source {
  static constexpr int LD = ROWS / 32;   // copies per wave and block
  const unsigned char* base;             // origin of the next block to copy
  unsigned off[LD];                      // this lane's byte offsets from it
  int krem;                              // TAIL: k left from there
  int kq;                                // this lane's k in a block (across: of even copies)

  // the tile rows from r0 (of n; across, rounded up to whole chunks), from K
  // block kb
  __device__ __forceinline__ void set(const bf16_t* p, int64_t ld, int r0, int n, int kb, int K) {
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int lr = (threadIdx.x & 63) >> 3, pos = threadIdx.x & 7;
    const int64_t origin = ALONG ? (int64_t)r0 * ld + (int64_t)kb * 64 : (int64_t)kb * 64 * ld + r0;
    base = reinterpret_cast<const unsigned char*>(uniform_ptr(p + origin));
    krem = K - kb * 64;
    if constexpr (ALONG) {
      kq = (pos ^ (4 * (wave & 1) + (lr >> 1))) * 8;
#pragma unroll
      for (int i = 0; i < LD; ++i)
        off[i] = (unsigned)(min(8 * (4 * i + wave) + lr, n - 1 - r0) * (int)ld + kq) * 2;
    } else {
      kq = 8 * wave + lr;
      const int s = ((lr >> 1) & 1) | ((wave & 1) << 1);
#pragma unroll
      for (int i = 0; i < LD; ++i) {
        const int k = kq + 32 * (i & 1), c = 64 * ((4 * i + wave) >> 3) + (pos ^ (s << 1)) * 8;
        off[i] = (unsigned)(k * (int)ld + min(c, n - 8 - r0)) * 2;
      }
    }
  }
  template <int I>
  __device__ __forceinline__ void copy(unsigned lds) const {
    if constexpr (TAIL) {
      const int k = ALONG ? kq : kq + 32 * (I & 1);
      copy16_ptr<I * 4096>(k < krem ? (const void*)(base + off[I]) : (const void*)&kZeroChunk, lds);
    } else {
      copy16_off<I * 4096>(base, off[I], lds);
    }
  }
  __device__ __forceinline__ void next(int64_t ld) {
    base += ALONG ? 128 : 128 * ld;
    if constexpr (TAIL) krem -= 64;
  }
};

// Fragment reads of one operand's slot.  COL0: first row of the wave's
// fragment 0; fragment f starts STEP rows after fragment f - 1.
template <bool ALONG, int STEP>
struct Reader {
  static constexpr int NB = ALONG ? 2 : 64 / STEP;   // lane addresses: by half block, or by 16 columns of a panel
  unsigned b[NB];
  __device__ __forceinline__ void init(unsigned lds, int row0) {
    const int lane = threadIdx.x & 63, p = lane & 15, g = lane >> 4;
    if constexpr (ALONG) {
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
        b[ks] = lds + (row0 + p) * 128 + (((ks * 4 + g) ^ ((p >> 1) & 7)) << 4);
    } else {
      const int s = (p >> 3) | ((g & 1) << 1);
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        const int c = (row0 & 63) / 16 + j * (STEP / 16);
        b[j] = lds + (row0 >> 6) * 8192 + g * 1024 + (p >> 2) * 128 + ((c ^ s) << 5) + (p & 3) * 8;
      }
    }
  }
  // addresses in a slot, opaque, so that they stay registers plus immediate
  // offsets
  struct At {
    unsigned a[NB];
  };
  template <int KS>
  __device__ __forceinline__ At at(unsigned slot) const {
    At r;
    if constexpr (ALONG) {
      r.a[0] = b[KS] + slot;
      asm volatile("" : "+v"(r.a[0]));
    } else {
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        r.a[j] = b[j] + slot;
        asm volatile("" : "+v"(r.a[j]));
      }
    }
    return r;
  }
  template <int F, int KS>
  static __device__ __forceinline__ bf16x8 read(const At& t) {
    if constexpr (ALONG) {
      return *(const lds_b16x8_t*)(uintptr_t)(t.a[0] + F * STEP * 128);
    } else {
      const unsigned p = t.a[F % NB] + (F * STEP / 64) * 8192 + KS * 4096;
      const tr_i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr_t*)(uintptr_t)p);
      const tr_i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr_t*)(uintptr_t)(p + 512));
      typedef short i16x8 __attribute__((ext_vector_type(8)));
      const i16x8 v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
      return __builtin_bit_cast(bf16x8, v);
    }
  }
};

// out tile = 32 TM rows of A x 32 TN rows of B.  FULL: the forward's epilogue;
// else the sums are stored as they are.
template <bool LA, bool LB, int TM, int TN, bool TAIL, bool FULL>
__global__ __launch_bounds__(256, TN == 8 ? 1 : 2) void linear_tile_kernel(Product p, Epilogue e,
                                                                           TileGrid tg) {
  constexpr int BM = 32 * TM, BN = 32 * TN;
  constexpr int ASLOT = BM * 128, BSLOT = BN * 128;
  constexpr int MPS = TM * TN, NR = TM + TN;
  static_assert(LA || TM % 2 == 0, "whole panels");
  __shared__ __align__(1024) unsigned char ring[2 * ASLOT + 3 * BSLOT];
  using SrcA = Source<LA, BM, TAIL>;
  using SrcB = Source<LB, BN, TAIL>;
  constexpr int A_LD = SrcA::LD, B_LD = SrcB::LD;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  auto uni = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  const bf16_t *A = (const bf16_t*)p.A, *B = (const bf16_t*)p.B;
  const int nblocks = (p.K + 63) / 64;
  const int ma = LA ? p.M : (p.M + 7) & ~7, nb = LB ? p.N : (p.N + 7) & ~7;

  const unsigned ring_lds = lds_addr(ring);
  const unsigned ldsA = ring_lds + wave * 1024, ldsB = ring_lds + 2 * ASLOT + wave * 1024;
  Reader<LA, 32> rdA;
  Reader<LB, 16> rdB;
  rdA.init(ring_lds, wm * 16);
  rdB.init(ring_lds + 2 * ASLOT, wn * 16 * TN);

  // items: XCD x takes the range [x per_xcd, (x + 1) per_xcd)
  const int total = tg.tiles_m * tg.tiles_n * tg.slices;
  const int per_xcd = (total + kXcd - 1) / kXcd;
  const int xcd_base = (int)(blockIdx.x % kXcd) * per_xcd;
  const int stride = gridDim.x / kXcd;
  struct Item {
    int m0, n0, slice, kb, nk;
  };
  auto decode = [&](int L, Item& it) {
    const int per = tg.tiles_m * tg.tiles_n;
    it.slice = uni(L / per);
    const int t = uni(L % per);
    constexpr int kBand = 8;
    const int band = uni(t / (kBand * tg.tiles_n));
    const int h = min(kBand, tg.tiles_m - band * kBand), u = uni(t - band * kBand * tg.tiles_n);
    it.m0 = uni((band * kBand + u % h) * BM);
    it.n0 = uni(u / h * BN);
    it.kb = it.slice * tg.kb_per;
    it.nk = min(nblocks - it.kb, tg.kb_per);
  };
  Item it, nx;
  int j = blockIdx.x / kXcd;
  if (j >= per_xcd || xcd_base + j >= total) return;   // a whole workgroup
  decode(xcd_base + j, it);
  SrcA sa;
  SrcB sb;
  sa.set(A, p.lda, it.m0, ma, it.kb, p.K);
  sb.set(B, p.ldb, it.n0, nb, it.kb, p.K);
  // LDS offsets of the slots of the current block, the next (and, B, the one
  // after)
  unsigned oa0 = 0, oa1 = ASLOT, ob0 = 0, ob1 = BSLOT, ob2 = 2 * BSLOT;
  auto copy_a = [&](unsigned o) __attribute__((always_inline)) {
    static_for<A_LD>([&](auto I) __attribute__((always_inline)) { sa.template copy<decltype(I)::value>(ldsA + o); });
    sa.next(p.lda);
  };
  auto copy_b = [&](unsigned o) __attribute__((always_inline)) {
    static_for<B_LD>([&](auto I) __attribute__((always_inline)) { sb.template copy<decltype(I)::value>(ldsB + o); });
    sb.next(p.ldb);
  };
  copy_a(oa0);
  copy_b(ob0);
  copy_b(ob1);
  copy_a(oa1);
  copy_b(ob2);

  for (;;) {
    const bool has_next = j + stride < per_xcd && xcd_base + j + stride < total;
    // without a next item the copies past this one's end re-read its own
    nx = it;
    if (has_next) decode(xcd_base + j + stride, nx);
    floatx4 acc[TM][TN];
    static_for<TM * TN>([&](auto q) __attribute__((always_inline)) {
      acc[q / TN][q % TN] = floatx4{0.f, 0.f, 0.f, 0.f};
    });
    bf16x8 F[2][NR];
    // fragment R in the order the MFMAs use them: A0, all B, A1 ..
    auto read1 = [&](bf16x8 (&f)[NR], const typename Reader<LA, 32>::At& ta,
                     const typename Reader<LB, 16>::At& tb, auto R, auto KS) __attribute__((always_inline)) {
      constexpr int r = decltype(R)::value, ks = decltype(KS)::value;
      constexpr int x = r == 0 ? 0 : (r <= TN ? TM + r - 1 : r - TN);
      if constexpr (x < TM) f[x] = Reader<LA, 32>::template read<x, ks>(ta);
      else f[x] = Reader<LB, 16>::template read<x - TM, ks>(tb);
    };
    using I0 = std::integral_constant<int, 0>;
    using I1 = std::integral_constant<int, 1>;
    // block 0 has landed in every wave (after it B 1, A 1, B 2 went out)
    wait_vmcnt<A_LD + 2 * B_LD>();
    barrier_nofence();
    {
      const auto ta = rdA.template at<0>(oa0);
      const auto tb = rdB.template at<0>(ob0);
      static_for<NR>([&](auto R) __attribute__((always_inline)) { read1(F[0], ta, tb, R, I0{}); });
    }
    // Half block KS: its MFMAs on fc, the reads of the next half block into
    // fn between them.  In the second half the workgroup meets after the
    // first MFMA: the next block has landed (only the B copies of the block
    // after it may be in flight), and every wave holds this half in
    // registers, so the block's slots are free: the A copies of the block
    // two ahead and the B copies of the block three ahead go out there.
    auto half = [&](bf16x8 (&fc)[NR], bf16x8 (&fn)[NR], auto KS, auto END) __attribute__((always_inline)) {
      constexpr int ks = decltype(KS)::value;
      constexpr bool end = decltype(END)::value && ks == 1;
      using KN = std::integral_constant<int, ks ^ 1>;
      const auto ta = rdA.template at<ks ^ 1>(ks == 0 ? oa0 : oa1);
      const auto tb = rdB.template at<ks ^ 1>(ks == 0 ? ob0 : ob1);
      static_for<MPS>([&](auto Q) __attribute__((always_inline)) {
        constexpr int q = decltype(Q)::value, i = q / TN, n = q % TN;
        acc[i][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fc[TM + n], fc[i], acc[i][n], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (q == 0 && ks == 1) {
          wait_lgkm0();
          if constexpr (!end) wait_vmcnt<B_LD>();
          barrier_nofence();
          __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (!end)
          static_for<NR>([&](auto R) __attribute__((always_inline)) {
            if constexpr (q == 1 + decltype(R)::value * (MPS * 3 / 4) / NR) read1(fn, ta, tb, R, KN{});
          });
        if constexpr (ks == 1)
          static_for<A_LD + B_LD>([&](auto D) __attribute__((always_inline)) {
            constexpr int d = decltype(D)::value;
            if constexpr (q == 1 + d * (MPS - 2) / (A_LD + B_LD)) {
              if constexpr (d < A_LD) {
                sa.template copy<d>(ldsA + oa0);
                if constexpr (d == A_LD - 1) sa.next(p.lda);
              } else {
                sb.template copy<d - A_LD>(ldsB + ob0);
                if constexpr (d == A_LD + B_LD - 1) sb.next(p.ldb);
              }
            }
          });
        __builtin_amdgcn_sched_barrier(0);
      });
      if constexpr (ks == 1) {
        const unsigned o = ob0, a = oa0;
        ob0 = ob1;
        ob1 = ob2;
        ob2 = o;
        oa0 = oa1;
        oa1 = a;
      }
    };
    for (int kt = 0; kt + 3 < it.nk; ++kt) {
      half(F[0], F[1], I0{}, I0{});
      half(F[1], F[0], I1{}, I0{});
    }
    // the last three blocks send out the next item's B copies, the last two
    // its A copies
    sb.set(B, p.ldb, nx.n0, nb, nx.kb, p.K);
    half(F[0], F[1], I0{}, I0{});
    half(F[1], F[0], I1{}, I0{});
    sa.set(A, p.lda, nx.m0, ma, nx.kb, p.K);
    half(F[0], F[1], I0{}, I0{});
    half(F[1], F[0], I1{}, I0{});
    half(F[0], F[1], I0{}, I1{});
    half(F[1], F[0], I1{}, I1{});
    const int c0 = it.n0 + wn * 16 * TN + col8(lane);
    const int r0 = it.m0 + wm * 16 + (lane & 15);
    if constexpr (FULL) {
      // A loop over the fragment rows, each fetched from its accumulators by a
      // jump: unrolled, TM rows of this code are far larger than the
      // instruction cache.  The bias is loaded once, the residual of the next
      // 16 rows before this one's stores.
      Raw8<float> bias[TN / 2];
      Raw8<bf16_t> res[TN / 2], rnext[TN / 2];
      static_for<TN / 2>([&](auto P) __attribute__((always_inline)) {
        bias[P] = epilogue_bias(e, p.N, c0 + 32 * P);
        rnext[P] = epilogue_res<bf16_t>(e, p.M, p.N, r0, c0 + 32 * P);
      });
#pragma unroll 1
      for (int i = 0; i < TM; ++i) {
        const int64_t r = r0 + i * 32;
        static_for<TN / 2>([&](auto P) __attribute__((always_inline)) {
          int c = c0 + 32 * P;   // opaque, as below
          asm volatile("" : "+v"(c));
          res[P] = rnext[P];
          rnext[P] = epilogue_res<bf16_t>(e, i + 1 < TM ? p.M : 0, p.N, r + 32, c);
        });
        floatx4 row[TN];
        static_for<TM>([&](auto I) __attribute__((always_inline)) {
          if (i == I)
            static_for<TN>([&](auto Q) __attribute__((always_inline)) { row[Q] = acc[I][Q]; });
        });
        uint32_t zb = 0, ob = 0;   // scale bytes of the row's four blocks
        static_for<TN / 2>([&](auto P) __attribute__((always_inline)) {
          constexpr int n = decltype(P)::value;
          float v[8];
          join8(row[2 * n], row[2 * n + 1], v);
          // (opaque: else the masks of every column's compare with N are kept
          // through the loop, more than there are scalar registers)
          int c = c0 + 32 * n;
          asm volatile("" : "+v"(c));
          if (tg.part) {
            if (r < p.M && c < p.N) store8<float>(tg.part + ((int64_t)it.slice * p.M + r) * tg.np + c, v, 8);
          } else {
            const uint32_t b =
                epilogue8<bf16_t, LANES_APART, false>(e, p.M, p.N, r, c, v, bias[n], res[n]);
            zb |= (b & 255) << (8 * n);
            ob |= (b >> 8) << (8 * n);
          }
          __builtin_amdgcn_sched_barrier(0);
        });
        // every group of lanes holds all of a row's bytes: the first writes
        // z's, the second out's
        uint8_t* scales = lane < 16 ? e.z_scales : lane < 32 ? e.out_scales : nullptr;
        if (scales && r < p.M) {
          constexpr int NB = TN / 2;
          const uint32_t bytes = lane < 16 ? zb : ob;
          const int blks = (p.N + kCkptBlock - 1) / kCkptBlock, b0 = (it.n0 + wn * 16 * TN) / kCkptBlock;
          uint8_t* q = scales + r * blks + b0;
          if (b0 + NB <= blks) {
            memcpy(q, &bytes, NB);
          } else {
#pragma unroll
            for (int j = 0; j < NB - 1; ++j)
              if (b0 + j < blks) q[j] = (uint8_t)(bytes >> (8 * j));
          }
        }
      }
    } else {
      static_for<TM>([&](auto I) __attribute__((always_inline)) {
        constexpr int i = decltype(I)::value;
        const int64_t r = r0 + i * 32;
        static_for<TN / 2>([&](auto P) __attribute__((always_inline)) {
          constexpr int n = decltype(P)::value;
          float v[8];
          join8(acc[i][2 * n], acc[i][2 * n + 1], v);
          const int c = c0 + 32 * n;
          if (r < p.M && c < p.N) {
            if (tg.part) store8<float>(tg.part + ((int64_t)it.slice * p.M + r) * tg.np + c, v, 8);
            else store8<bf16_t>((bf16_t*)e.out + r * e.ldo + c, v, min(8, p.N - c));
          }
          __builtin_amdgcn_sched_barrier(0);
        });
      });
    }
    if (!has_next) break;
    j += stride;
    it = nx;
  }
  wait_vmcnt<0>();   // no copy outlives the workgroup's LDS
}

template <bool LA, bool LB, int TM, int TN, bool FULL>
void run_tile(const Product& p, const Epilogue& e, const TileGrid& tg, int cus, hipStream_t s) {
  const int64_t items = (int64_t)tg.tiles_m * tg.tiles_n * tg.slices;
  const int64_t want = cdiv64(items, kXcd), have = (TN == 8 ? 1 : 2) * cus / kXcd;
  const unsigned grid = (unsigned)((want < have ? want : have) * kXcd);
  if constexpr (TM < 8) {   // (product_plan: no 256 rows with a tail)
    if (p.K % 64) {
      launch_k(linear_tile_kernel<LA, LB, TM, TN, true, FULL>, grid, 256, 0, s, p, e, tg);
      return;
    }
  }
  launch_k(linear_tile_kernel<LA, LB, TM, TN, false, FULL>, grid, 256, 0, s, p, e, tg);
}

}  // namespace
}  // namespace fs
