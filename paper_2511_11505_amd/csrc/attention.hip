// Attention over a paged cache: which kernel runs, on how many workgroups.
// (The kernels are in attention_kernel.hpp, instantiated in attention_*.hip.)

#include "attention.hpp"

namespace fs {
namespace {

constexpr int kCus = 256;
constexpr int kMaxGroups = 1 << 16;
// A prompt of more rows than that, enough of them for the waves below, is not
// divided: a wave has two row tiles (in fp32 and past 128 columns one) to itself and
// nothing is joined.  64 query and 8 key heads of 128 columns, this way | divided, us:
// a prompt of 2048 tokens 188 | 579, of 8192 with 16 query heads 635 | 1356; 512 new
// tokens of 4096, two sequences, 313 | 577, in fp32 1250 | 1645; 64 of 4096, six, 239 |
// 257 (768 waves), five, 230 | 231 (640).  One row tile a wave took 317, 1192,
// 544, -, 305 and 304, four 349, 1282, 546: the products wait for the cache's tiles and
// for the softmax.
constexpr int kPromptTiles = 16;
int prompt_tiles(int dtype, int width) { return dtype == 0 || width == 256 ? 1 : 2; }
int prompt_waves(int dtype, int width) { return prompt_tiles(dtype, width) == 1 ? 1024 : 640; }

int width_of(int d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }

int cache_of(int dtype, const PagedCache& c) {
  return c.codes ? (dtype == 0 ? CACHE_CODES_F32 : CACHE_CODES_BF16) : dtype == 0 ? CACHE_F32 : CACHE_BF16;
}

// Row tiles of an item: what the rows of a sequence need, up to what the
// registers hold (a row tile takes D / 4 of them for its sums and D / 8, in fp32
// D / 4, for its queries).  Four leave one workgroup to a CU and start later, but
// read a long bf16 cache once where two read it twice: 56 rows a key head, 8 of them,
// four tiles | two, us: 32 sequences of 8192 tokens 273 | 312, of 4096 150 | 167, 1 of 65536
// 89 | 109; 8 of 4096 and 32 of 1024 (2^18 tokens and heads) 58 | 58 and 58 | 57, 8 of 512
// 31 | 17, 256 of 512 249 | 185.  With pages of 20 tokens two are faster (32 of 8192 tokens
// 440 | 257, 1 of 65536 132 | 84), and an 8-bit cache does not gain: 16 of 16384 213 | 200.
bool four_tiles(const PagedCache& c, int64_t tokens) {
  return !c.codes && c.page_size % 16 == 0 && tokens > 512 &&
         (double)c.sequences * tokens * c.kv_heads > (1 << 18);
}
// Past 128 columns two row tiles spill registers.  Where all 256 columns of codes in pages of whole
// groups are read, one is faster: 4 new tokens, 8 heads a key head, 8 of them, two | one, us, 32
// sequences of 8192 tokens 582 | 394, of 512 52 | 41, 8 of 512 49 | 21; with pages of 20 tokens
// 527 | 562, of 192 columns 317 | 405, in bf16 544 | 643.
bool one_tile(int dtype, int width, const PagedCache& c) {
  return width == 256 && (dtype == 0 || (c.codes && c.page_size % 16 == 0 && c.d > 256 - 32));
}
int row_tiles(int dtype, int width, int rows, const PagedCache& c, int64_t tokens) {
  if (rows <= 16 || one_tile(dtype, width, c)) return 1;
  return rows <= 32 || dtype == 0 || width == 256 || !four_tiles(c, tokens) ? 2 : 4;
}

struct Shape {
  int width, rt, group, rows, row_groups;
  bool prompt;
  int64_t items;
  int workers;
};
Shape shape_of(int dtype, int q_heads, int n_new, const PagedCache& c, int most_row_tiles = 4) {
  Shape h;
  h.width = width_of(c.d);
  h.group = q_heads / c.kv_heads;
  h.rows = n_new * h.group;
  const int64_t tokens = (int64_t)c.max_pages * c.page_size;
  h.rt = row_tiles(dtype, h.width, h.rows, c, tokens);
  if (h.rt > most_row_tiles) h.rt = most_row_tiles;
  const int tiles = (h.rows + 15) / 16;
  h.workers = 0;
  const int alone = prompt_tiles(dtype, h.width), groups = (tiles + alone - 1) / alone;
  h.prompt = n_new > 1 && tiles > kPromptTiles &&
             (int64_t)c.sequences * groups * c.kv_heads >= prompt_waves(dtype, h.width);
  if (h.prompt) {
    h.rt = alone, h.row_groups = groups, h.items = (int64_t)c.sequences * groups;
    return h;
  }
  h.row_groups = (h.rows + 16 * h.rt - 1) / (16 * h.rt);
  h.items = (int64_t)c.sequences * h.row_groups;
  // A sequence of at most four tiles a wave is not worth a second launch;
  // beyond kAttnMaxItems, or that many workgroups, there is enough to fill the chip.
  const int tile = dtype == 0 ? 16 : 32;
  const int64_t most = (tokens + tile - 1) / tile;
  if (h.items <= kAttnMaxItems && h.items * c.kv_heads <= kMaxGroups && most > 4 * kAttnWaves) {
    const int64_t parts = (h.items * most + kAttnMinTiles - 1) / kAttnMinTiles;
    h.workers = (kCus * attn_groups_per_cu(h.width, h.rt) + c.kv_heads - 1) / c.kv_heads;
    if (parts < h.workers) h.workers = (int)parts;
    if (h.workers < 2) h.workers = 0;   // (one part has nothing to divide)
  }
  return h;
}

size_t up(size_t n) { return (n + 255) / 256 * 256; }
int64_t part_rows(const Shape& h, const PagedCache& c) { return (int64_t)h.workers * c.kv_heads * 2 * 16 * h.rt; }

template <int CACHE, int D, int RT, int PAGES>
hipError_t run_new(const AttnPlan& p, hipStream_t s) {
  if constexpr (RT == 1) {
    if (p.a.n_new == 1) return run_attention<CACHE, D, RT, PAGES, NEW_ONE>(p, s);
  }
  if constexpr (RT == (CACHE == CACHE_F32 || CACHE == CACHE_CODES_F32 || D == 256 ? 1 : 2))
    if (p.prompt) return run_attention<CACHE, D, RT, PAGES, NEW_PROMPT>(p, s);
  return run_attention<CACHE, D, RT, PAGES, NEW_SOME>(p, s);
}
template <int CACHE, int D, int RT>
hipError_t run_pages(const AttnPlan& p, hipStream_t s) {
  constexpr bool codes = CACHE == CACHE_CODES_BF16 || CACHE == CACHE_CODES_F32;
  // (what row_tiles does not choose is not built)
  if constexpr (RT != 4)
    if (p.c.page_size % 16) return run_new<CACHE, D, RT, PAGES_ANY>(p, s);
  if constexpr (codes && D == 256 && RT == 2) {
    return run_new<CACHE, D, RT, PAGES_GROUPS_SHORT>(p, s);
  } else {
    if constexpr (codes)
      if (p.c.d <= D - 32) return run_new<CACHE, D, RT, PAGES_GROUPS_SHORT>(p, s);
    return run_new<CACHE, D, RT, PAGES_GROUPS>(p, s);
  }
}
template <int CACHE>
hipError_t run_cache(int width, int rt, const AttnPlan& p, hipStream_t s) {
  constexpr bool f32 = CACHE == CACHE_F32 || CACHE == CACHE_CODES_F32;
  if (width == 256) {
    if constexpr (!f32)
      if (rt == 2) return run_pages<CACHE, 256, 2>(p, s);
    return run_pages<CACHE, 256, 1>(p, s);
  }
  if (rt == 4) {
    if constexpr (CACHE == CACHE_BF16) return width == 64 ? run_pages<CACHE, 64, 4>(p, s) : run_pages<CACHE, 128, 4>(p, s);
  }
  if (rt == 2) return width == 64 ? run_pages<CACHE, 64, 2>(p, s) : run_pages<CACHE, 128, 2>(p, s);
  return width == 64 ? run_pages<CACHE, 64, 1>(p, s) : run_pages<CACHE, 128, 1>(p, s);
}

}  // namespace

// Enough for narrower page tables too (a program may cut its table to the longest
// sequence that it has now): with the same row tiles these need no more, but they may have
// two where this one has four.
size_t attention_ws_bytes(int dtype, int q_heads, int n_new, const PagedCache& c) {
  size_t most = 0;
  for (int rt : {2, 4}) {
    const Shape h = shape_of(dtype, q_heads, n_new, c, rt);
    if (!h.workers) continue;
    const int64_t rows = part_rows(h, c);
    const size_t bytes = up(rows * h.width * 4) + up(rows * 8) + up(h.items * 8);
    if (bytes > most) most = bytes;
  }
  return most;
}

hipError_t launch_attention(int dtype, const AttnArgs& a, const PagedCache& c, void* ws, hipStream_t s) {
  const Shape h = shape_of(dtype, a.q_heads, a.n_new, c);
  AttnPlan p{};
  p.a = a, p.c = c;
  // (a window as long as the longest sequence hides nothing)
  if (a.window >= (int64_t)c.max_pages * c.page_size) p.a.window = 0;
  p.group = h.group, p.rows = h.rows, p.row_groups = h.row_groups, p.items = (int)h.items, p.workers = h.workers;
  p.prompt = h.prompt;
  if (h.workers) {
    const int64_t rows = part_rows(h, c);
    char* w = (char*)ws;
    p.part = (float*)w;
    p.stat = (float2*)(w + up(rows * h.width * 4));
    p.span = (int2*)(w + up(rows * h.width * 4) + up(rows * 8));
  }
  switch (cache_of(dtype, c)) {
    case CACHE_BF16: return run_cache<CACHE_BF16>(h.width, h.rt, p, s);
    case CACHE_F32: return run_cache<CACHE_F32>(h.width, h.rt, p, s);
    case CACHE_CODES_BF16: return run_cache<CACHE_CODES_BF16>(h.width, h.rt, p, s);
    default: return run_cache<CACHE_CODES_F32>(h.width, h.rt, p, s);
  }
}

}  // namespace fs
