// What the attention's kernels are given (attention_kernel.hpp), and their
// launch (instantiated in attention_*.hip).
#pragma once

#include "internal.hpp"

namespace fs {

enum { CACHE_BF16 = 0, CACHE_F32 = 1, CACHE_CODES_BF16 = 2, CACHE_CODES_F32 = 3 };

// Pages: of any size; of whole groups of 16 tokens; of whole groups, with codes of
// fewer blocks in a row than the kernel's width has.
enum { PAGES_ANY = 0, PAGES_GROUPS = 1, PAGES_GROUPS_SHORT = 2 };

// New tokens: one, with rows for one row tile; several; so many (a prompt's) that
// the rows fill the chip, a wave one or two row tiles to itself.
enum { NEW_ONE = 0, NEW_SOME = 1, NEW_PROMPT = 2 };

constexpr int kAttnWaves = 4;
constexpr int kAttnMaxItems = 4096;    // of a divided call: 16 for each thread
constexpr int kAttnMinTiles = 4;       // of a workgroup's part: one for each wave

// Workgroups a CU runs at once (four waves of 256 registers on each SIMD, or of 512).
// (In fp32 two row tiles of 128 columns take 320 registers and 85 KB of LDS: one of the
// two that are counted here.)
constexpr int attn_groups_per_cu(int width, int row_tiles) { return width < 256 && row_tiles <= 2 ? 2 : 1; }

struct AttnPlan {
  AttnArgs a;
  PagedCache c;
  int group, rows;         // query heads a key head; rows = n_new * group
  int row_groups, items;   // items = sequences * row_groups
  bool prompt;             // a wave for each item
  int workers;             // parts, each of kv_heads workgroups; 0: one for each item
  float* part;             // [workers * kv_heads * 2][rows of an item][D]
  float2* stat;            // [workers * kv_heads * 2][rows of an item]: largest score, sum of weights
  int2* span;              // [items]: first and last part
};

template <int CACHE, int D, int RT, int PAGES, int NEW>
hipError_t run_attention(const AttnPlan& p, hipStream_t s);

}  // namespace fs
