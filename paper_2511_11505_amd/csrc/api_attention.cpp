// C entry points of the attention sublayer: rotary positions and their backward
// pass, the append to a paged cache, and the attention of new tokens over it.
// Every check runs on the host before anything is enqueued; no exception
// leaves an entry.

#include <algorithm>
#include <cmath>
#include <utility>

#include "api_common.hpp"
#include "internal.hpp"

namespace {

constexpr int64_t kMaxStride = (int64_t)1 << 40, kMaxExtent = (int64_t)1 << 48;
constexpr int64_t kMaxTokens = 1 << 24, kMaxHeads = 1 << 16;
constexpr int kMaxRotaryDim = 512, kMaxCacheDim = 256;

// An array argument of `cols` columns that lie together, and up to three outer
// dimensions with strides (elements).
struct Arr {
  const char* name;
  const void* p;
  size_t es;
  int64_t cols;
  int64_t n[3], st[3];
};

Arr heads_of(const char* name, const void* p, size_t es, int64_t tokens, int64_t heads, int64_t d, int64_t ts,
             int64_t hs) {
  return {name, p, es, d, {tokens, heads, 1}, {ts, hs, 0}};
}
Arr flat_of(const char* name, const void* p, size_t es, int64_t n) {
  return {name, n > 0 ? p : nullptr, es, n, {1, 1, 1}, {0, 0, 0}};
}

// Elements from the first to behind the last, and whether no two elements share
// an address: from the inside out, each dimension steps over what is in it.
bool extent(const Arr& a, int64_t* len) {
  int order[3] = {0, 1, 2};
  for (int i = 0; i < 2; ++i)
    for (int j = 0; j < 2 - i; ++j)
      if (a.st[order[j]] > a.st[order[j + 1]]) std::swap(order[j], order[j + 1]);
  *len = a.cols;
  bool apart = true;
  for (int i : order) {
    if (a.n[i] <= 1) continue;
    apart = apart && a.st[i] >= *len;
    *len += (a.n[i] - 1) * a.st[i];
  }
  return apart;
}

fs_status check_arr(const Arr& a) {
  if (!a.p) return fail(FS_ERR_INVALID, std::string(a.name) + " must not be NULL");
  if (!aligned_to(a.p, a.es)) return fail(FS_ERR_INVALID, std::string(a.name) + " must be aligned to its elements");
  for (int i = 0; i < 3; ++i)
    if (a.n[i] > 1 && (a.st[i] < 0 || a.st[i] > kMaxStride || (a.n[i] - 1) > kMaxExtent / (a.st[i] + 1)))
      return fail(FS_ERR_UNSUPPORTED, std::string(a.name) + ": strides must be in [0, 2^40], its extent below 2^48 elements");
  int64_t len;
  if (!extent(a, &len))
    return fail(FS_ERR_INVALID, std::string(a.name) + ": its elements overlap (strides too small)");
  return FS_OK;
}

// Whether two arrays share bytes: the same base, or overlapping ranges without
// gaps, or with gaps where both repeat at the same stride and their parts
// between two repeats meet.  (Of other views with gaps the bytes between may be
// another's.)
bool overlap(const Arr& a, const Arr& b) {
  if (!a.p || !b.p) return false;
  if (a.p == b.p) return true;
  int64_t la, lb;
  if (!extent(a, &la) || !extent(b, &lb)) return true;
  const char *x = (const char*)a.p, *y = (const char*)b.p;
  const int64_t ba = la * (int64_t)a.es, bb = lb * (int64_t)b.es;
  if (x >= y + bb || y >= x + ba) return false;
  auto count = [](const Arr& v) { return v.cols * v.n[0] * v.n[1] * v.n[2]; };
  if (count(a) == la && count(b) == lb) return true;
  // the outermost dimension of each: its stride, and what lies inside of it
  auto outer = [](const Arr& v, int64_t len, int64_t* st, int64_t* in) {
    int k = -1;
    for (int i = 0; i < 3; ++i)
      if (v.n[i] > 1 && (k < 0 || v.st[i] > v.st[k])) k = i;
    *st = k < 0 ? 0 : v.st[k] * (int64_t)v.es;
    *in = (k < 0 ? len : len - (v.n[k] - 1) * v.st[k]) * (int64_t)v.es;
    int64_t inside = v.cols;
    for (int i = 0; i < 3; ++i)
      if (i != k) inside *= v.n[i];
    return inside * (int64_t)v.es == *in;   // no gaps inside
  };
  int64_t sa, ia, sb, ib;
  const bool ga = outer(a, la, &sa, &ia), gb = outer(b, lb, &sb, &ib);
  if (!ga || !gb || sa != sb || sa == 0) return false;
  const int64_t off = ((y - x) % sa + sa) % sa;
  return off < ia || off > sa - ib;
}
fs_status no_overlap(const Arr& out, const Arr& in) {
  if (overlap(out, in)) return fail(FS_ERR_INVALID, std::string(out.name) + " and " + in.name + " overlap");
  return FS_OK;
}

fs_status check_rope(const fs_rope* r, int32_t d, fs::Rope* out) {
  *out = {true, 0, 0, 1.0, nullptr};
  if (!r) return FS_OK;
  if (r->layout != FS_ROPE_HALVES && r->layout != FS_ROPE_PAIRS)
    return fail(FS_ERR_INVALID, "rope: layout must be an fs_rope_layout");
  if (r->rot_dim < 0 || r->rot_dim % 2 || r->first < 0 || r->first > d || r->rot_dim > d - r->first)
    return fail(FS_ERR_INVALID, "rope: rot_dim must be even and first + rot_dim <= head_dim");
  if (r->rot_dim == 0) return FS_OK;
  if (!std::isfinite(r->mscale)) return fail(FS_ERR_INVALID, "rope: mscale must be finite");
  if (!r->freqs || !aligned_to(r->freqs, 8))
    return fail(FS_ERR_INVALID, "rope: freqs must be given and 8-byte aligned");
  *out = {r->layout == FS_ROPE_HALVES, r->first, r->rot_dim, r->mscale, r->freqs};
  return FS_OK;
}
Arr freqs_of(const fs::Rope& r) { return flat_of("rope's freqs", r.freqs, 8, r.rot / 2); }

fs_status check_rotary(const fs_rotary_desc* d) {
  if (!d) return fail(FS_ERR_INVALID, "desc must not be NULL");
  if (d->abi_version != FS_ABI_VERSION) return fail(FS_ERR_INVALID, "desc->abi_version mismatch");
  TRY(check_dtype(d->dtype));
  if (d->tokens < 0 || d->heads <= 0 || d->head_dim <= 0)
    return fail(FS_ERR_INVALID, "tokens >= 0, heads > 0 and head_dim > 0 required");
  if (d->tokens > kMaxTokens || d->heads > kMaxHeads || d->head_dim > kMaxRotaryDim)
    return fail(FS_ERR_UNSUPPORTED, "tokens <= 2^24, heads <= 2^16 and head_dim <= 512 required");
  return FS_OK;
}

// Waves of a rotation: one of a token's rows at least, so a grid of fewer than
// 2^32 threads.
fs_status rotary(const fs_rotary_desc* d, const fs_rope* rope, const char* in_name, const void* x, int64_t tsx,
                 int64_t hsx, const int32_t* positions, const char* out_name, void* out, int64_t tso, int64_t hso,
                 bool back, fs_stream stream) {
  TRY(check_rotary(d));
  fs::RotaryArgs g{};
  TRY(check_rope(rope, d->head_dim, &g.rope));
  if (d->tokens == 0) return FS_OK;
  const size_t es = elem(d->dtype);
  const Arr X = heads_of(in_name, x, es, d->tokens, d->heads, d->head_dim, tsx, hsx);
  const Arr O = heads_of(out_name, out, es, d->tokens, d->heads, d->head_dim, tso, hso);
  TRY(check_arr(X));
  TRY(check_arr(O));
  NEED4(positions, "positions");
  const bool in_place = x == out && (tsx == tso || d->tokens == 1) && (hsx == hso || d->heads == 1);
  if (!in_place) TRY(no_overlap(O, X));
  TRY(no_overlap(O, flat_of("positions", positions, 4, d->tokens)));
  TRY(no_overlap(O, freqs_of(g.rope)));
  TRY(check_stream(stream));
  g.tokens = d->tokens, g.q_heads = d->heads, g.d = d->head_dim, g.back = back, g.positions = positions;
  g.q = {x, tsx, hsx}, g.out = {out, tso, hso};
  FS_HIP(fs::launch_rotary(dt(d->dtype), g, fs::PagedCache{}, S(stream)), "rotary");
  return FS_OK;
}

fs_status check_cache(const fs_kv_cache* c) {
  if (!c) return fail(FS_ERR_INVALID, "cache must not be NULL");
  if (c->abi_version != FS_ABI_VERSION) return fail(FS_ERR_INVALID, "cache->abi_version mismatch");
  TRY(check_dtype(c->dtype));
  if (c->codes != 0 && c->codes != 1) return fail(FS_ERR_INVALID, "cache: codes must be 0/1");
  if (c->n_pages < 0 || c->kv_heads <= 0 || c->page_size <= 0 || c->head_dim <= 0)
    return fail(FS_ERR_INVALID, "cache: n_pages >= 0, kv_heads > 0, page_size > 0 and head_dim > 0 required");
  if ((int64_t)c->n_pages * c->page_size > ((int64_t)1 << 34))
    return fail(FS_ERR_UNSUPPORTED, "cache: n_pages * page_size must be <= 2^34");
  if (c->kv_heads > 4096) return fail(FS_ERR_UNSUPPORTED, "cache: kv_heads must be <= 4096");
  if (c->head_dim % 8 || c->head_dim > kMaxCacheDim)
    return fail(FS_ERR_UNSUPPORTED, "cache: head_dim must be a multiple of 8 and <= 256");
  return FS_OK;
}

// The cache's arrays: k, v and, with codes, their scales.
struct CacheArrs {
  Arr a[4];
};
CacheArrs arrs_of(const fs_kv_cache* c) {
  const size_t es = c->codes ? 1 : elem(c->dtype);
  const int64_t p = c->n_pages, h = c->kv_heads, s = c->page_size, d = c->head_dim;
  const int64_t scales = c->codes ? p * h * s * ((d + 31) / 32) : 0;
  auto rows = [&](const char* name, void* q) {
    return Arr{name, p ? q : nullptr, es, d, {p, h, s}, {c->page_stride, c->head_stride, c->place_stride}};
  };
  return {rows("cache's k", c->k), rows("cache's v", c->v), flat_of("cache's k_scales", c->k_scales, 1, scales),
          flat_of("cache's v_scales", c->v_scales, 1, scales)};
}

fs_status check_cache_memory(const fs_kv_cache* c, const CacheArrs& m) {
  if (c->n_pages == 0) return FS_OK;
  for (int i = 0; i < 2; ++i) {
    TRY(check_arr(m.a[i]));
    if (!aligned_to(m.a[i].p, c->codes ? 8 : 16))
      return fail(FS_ERR_INVALID, std::string(m.a[i].name) + (c->codes ? " must be 8-byte aligned" : " must be 16-byte aligned"));
  }
  const int64_t counts[] = {c->n_pages, c->kv_heads, c->page_size};
  const int64_t strides[] = {c->page_stride, c->head_stride, c->place_stride};
  for (int i = 0; i < 3; ++i)
    if (counts[i] > 1 && strides[i] % 8) return fail(FS_ERR_INVALID, "cache: strides must be multiples of 8");
  if (c->page_size > 1 && c->place_stride > (1 << 20)) return fail(FS_ERR_UNSUPPORTED, "cache: place_stride must be <= 2^20");
  if (c->codes && (!c->k_scales || !c->v_scales)) return fail(FS_ERR_INVALID, "cache: codes without scales");
  if (c->codes && (!aligned_to(c->k_scales, 8) || !aligned_to(c->v_scales, 8)))
    return fail(FS_ERR_INVALID, "cache: scales must be 8-byte aligned");
  for (int i = 0; i < 4; ++i)
    for (int j = i + 1; j < 4; ++j) TRY(no_overlap(m.a[i], m.a[j]));
  return FS_OK;
}

fs_status check_pages(const fs_page_table* t, const fs_kv_cache* c) {
  if (!t) return fail(FS_ERR_INVALID, "pages must not be NULL");
  if (t->sequences < 0 || t->max_pages < 0) return fail(FS_ERR_INVALID, "pages: sequences >= 0 and max_pages >= 0 required");
  if (t->sequences > (1 << 20)) return fail(FS_ERR_UNSUPPORTED, "pages: sequences must be <= 2^20");
  if ((int64_t)t->max_pages * c->page_size > (1 << 30))
    return fail(FS_ERR_UNSUPPORTED, "pages: max_pages * page_size must be <= 2^30");
  return FS_OK;
}
Arr table_of(const fs_page_table* t) {
  return {"pages' table", t->max_pages ? t->table : nullptr, 4, t->max_pages, {t->sequences, 1, 1}, {t->ldt, 0, 0}};
}
fs_status check_table(const fs_page_table* t) {
  if (t->sequences == 0 || t->max_pages == 0) return FS_OK;
  return check_arr(table_of(t));
}

fs::PagedCache cache_of(const fs_kv_cache* c, const fs_page_table* t) {
  return {c->codes, c->n_pages, c->kv_heads, c->page_size, c->head_dim, c->k, c->v, c->page_stride, c->head_stride,
          c->place_stride, c->k_scales, c->v_scales, t->table, t->ldt, t->sequences, t->max_pages};
}

fs_status check_attention(const fs_attention_desc* d, const fs_kv_cache* c, const fs_page_table* t) {
  if (!d) return fail(FS_ERR_INVALID, "desc must not be NULL");
  if (d->abi_version != FS_ABI_VERSION) return fail(FS_ERR_INVALID, "desc->abi_version mismatch");
  TRY(check_cache(c));
  TRY(check_pages(t, c));
  if (d->q_heads <= 0 || d->q_heads % c->kv_heads)
    return fail(FS_ERR_INVALID, "q_heads must be a positive multiple of kv_heads");
  if (d->new_tokens < 1 || d->window < 0) return fail(FS_ERR_INVALID, "new_tokens >= 1 and window >= 0 required");
  if (d->q_heads > kMaxHeads) return fail(FS_ERR_UNSUPPORTED, "q_heads must be <= 2^16");
  if ((int64_t)t->sequences * d->new_tokens > kMaxTokens || d->new_tokens > kMaxTokens)
    return fail(FS_ERR_UNSUPPORTED, "sequences * new_tokens must be <= 2^24");
  // (rows of 16 queries of one key head, and a workgroup for each)
  const int64_t items = (int64_t)std::max(t->sequences, 1) * (((int64_t)d->new_tokens * (d->q_heads / c->kv_heads) + 15) / 16);
  if (items * c->kv_heads >= ((int64_t)1 << 23))
    return fail(FS_ERR_UNSUPPORTED, "sequences * new_tokens * q_heads: more than 2^23 groups of 16 rows");
  if (!(std::fabs(d->scale) <= 1e38f)) return fail(FS_ERR_INVALID, "scale must be within +-1e38");
  return FS_OK;
}

// at: queries are at `positions`, else at their sequences' ends.
fs_status paged_attention(const fs_attention_desc* d, const fs_kv_cache* cache, const void* q, int64_t tsq,
                          int64_t hsq, bool at, const int32_t* positions, const int32_t* lengths, const fs_page_table* pages,
                          void* out, int64_t tso, int64_t hso, float* lse, void* ws, size_t ws_bytes,
                          fs_stream stream) {
  TRY(check_attention(d, cache, pages));
  if (pages->sequences == 0) return FS_OK;
  const size_t es = elem(cache->dtype);
  const int64_t t = (int64_t)pages->sequences * d->new_tokens;
  const Arr Q = heads_of("q", q, es, t, d->q_heads, cache->head_dim, tsq, hsq);
  const Arr O = heads_of("out", out, es, t, d->q_heads, cache->head_dim, tso, hso);
  TRY(check_arr(Q));
  TRY(check_arr(O));
  if (at) NEED4(positions, "positions");
  NEED4(lengths, "lengths");
  OPT4(lse, "lse");
  TRY(check_table(pages));
  const CacheArrs m = arrs_of(cache);
  TRY(check_cache_memory(cache, m));
  const fs::PagedCache pc = cache_of(cache, pages);
  const size_t need = fs::attention_ws_bytes(dt(cache->dtype), d->q_heads, d->new_tokens, pc);
  if (ws_bytes < need) return fail(FS_ERR_WORKSPACE, "workspace smaller than fs_paged_attention_workspace");
  if (need) NEED(ws, "ws");
  const Arr outs[] = {O, flat_of("lse", lse, 4, lse ? t * d->q_heads : 0),
                      flat_of("ws", ws, 1, (int64_t)need)};
  const Arr ins[] = {Q, flat_of("positions", positions, 4, at ? t : 0),
                     flat_of("lengths", lengths, 4, pages->sequences), table_of(pages), m.a[0], m.a[1],
                     m.a[2], m.a[3]};
  for (int i = 0; i < 3; ++i) {
    for (const Arr& x : ins) TRY(no_overlap(outs[i], x));
    for (int j = i + 1; j < 3; ++j) TRY(no_overlap(outs[i], outs[j]));
  }
  TRY(check_stream(stream));
  fs::AttnArgs g{};
  g.q_heads = d->q_heads, g.n_new = d->new_tokens, g.window = d->window, g.scale = d->scale;
  g.q = {q, tsq, hsq}, g.out = {out, tso, hso}, g.lengths = lengths, g.positions = positions, g.lse = lse;
  FS_HIP(fs::launch_attention(dt(cache->dtype), g, pc, ws, S(stream)), "paged_attention");
  return FS_OK;
}

}  // namespace

extern "C" {

fs_status fs_rope_frequencies(int32_t rot_dim, double base, int32_t scaling, double factor, double trained_len,
                              double low, double high, double* freqs) {
  return entry([&]() -> fs_status {
    if (rot_dim < 0 || rot_dim % 2) return fail(FS_ERR_INVALID, "rot_dim must be even and >= 0");
    if (rot_dim > kMaxRotaryDim) return fail(FS_ERR_UNSUPPORTED, "rot_dim must be <= 512");
    if (scaling < FS_ROPE_PLAIN || scaling > FS_ROPE_PARTS)
      return fail(FS_ERR_INVALID, "scaling must be an fs_rope_scaling");
    if (!(base > 0) || !std::isfinite(base)) return fail(FS_ERR_INVALID, "base must be > 0 and finite");
    if (scaling != FS_ROPE_PLAIN && (!(factor > 0) || !std::isfinite(factor)))
      return fail(FS_ERR_INVALID, "factor must be > 0 and finite");
    if (scaling == FS_ROPE_BASE && rot_dim == 2) return fail(FS_ERR_INVALID, "FS_ROPE_BASE needs rot_dim > 2");
    if (scaling == FS_ROPE_PARTS && (!(trained_len > 0) || !std::isfinite(trained_len) || !(low < high) ||
                                     !std::isfinite(low) || !std::isfinite(high)))
      return fail(FS_ERR_INVALID, "FS_ROPE_PARTS needs trained_len > 0 and low < high, all finite");
    if (rot_dim == 0) return FS_OK;
    if (!freqs) return fail(FS_ERR_INVALID, "freqs must not be NULL");
    const double r = rot_dim;
    if (scaling == FS_ROPE_BASE) base *= std::pow(factor, r / (r - 2));
    for (int i = 0; i < rot_dim / 2; ++i) {
      double f = std::pow(base, -2.0 * i / r);
      if (scaling == FS_ROPE_LINEAR) {
        f /= factor;
      } else if (scaling == FS_ROPE_PARTS) {
        const double t = trained_len * f / 6.283185307179586476925;
        const double keep = std::fmin(1.0, std::fmax(0.0, (t - low) / (high - low)));
        f *= keep + (1.0 - keep) / factor;
      }
      freqs[i] = f;
    }
    return FS_OK;
  });
}

fs_status fs_rotary(const fs_rotary_desc* d, const fs_rope* rope, const void* x, int64_t tsx, int64_t hsx,
                    const int32_t* positions, void* out, int64_t tso, int64_t hso, fs_stream stream) {
  return entry([&] { return rotary(d, rope, "x", x, tsx, hsx, positions, "out", out, tso, hso, false, stream); });
}

fs_status fs_rotary_backward(const fs_rotary_desc* d, const fs_rope* rope, const void* dout, int64_t tso,
                             int64_t hso, const int32_t* positions, void* dx, int64_t tsx, int64_t hsx,
                             fs_stream stream) {
  return entry([&] { return rotary(d, rope, "dout", dout, tso, hso, positions, "dx", dx, tsx, hsx, true, stream); });
}

fs_status fs_cache_append(const fs_kv_cache* cache, const fs_rope* rope, int32_t tokens, int32_t q_heads,
                          const void* q, int64_t tsq, int64_t hsq, const void* k, int64_t tsk, int64_t hsk,
                          const void* v, int64_t tsv, int64_t hsv, const int32_t* seqs, const int32_t* positions,
                          const fs_page_table* pages, void* q_out, int64_t tso, int64_t hso, fs_stream stream) {
  return entry([&]() -> fs_status {
    TRY(check_cache(cache));
    TRY(check_pages(pages, cache));
    fs::RotaryArgs g{};
    TRY(check_rope(rope, cache->head_dim, &g.rope));
    if (tokens < 0) return fail(FS_ERR_INVALID, "tokens must be >= 0");
    if (tokens > kMaxTokens) return fail(FS_ERR_UNSUPPORTED, "tokens must be <= 2^24");
    if (q && (q_heads <= 0 || q_heads > kMaxHeads))
      return fail(FS_ERR_INVALID, "q_heads must be in [1, 2^16] where q is given");
    if (!q != !q_out) return fail(FS_ERR_INVALID, "q and q_out are given together");
    if (tokens == 0) return FS_OK;
    const size_t es = elem(cache->dtype);
    const int64_t t = tokens, d = cache->head_dim;
    const Arr Q = heads_of("q", q, es, t, q ? q_heads : 1, d, tsq, hsq);
    const Arr QO = heads_of("q_out", q_out, es, t, q ? q_heads : 1, d, tso, hso);
    const Arr K = heads_of("k", k, es, t, cache->kv_heads, d, tsk, hsk);
    const Arr V = heads_of("v", v, es, t, cache->kv_heads, d, tsv, hsv);
    if (q) {
      TRY(check_arr(Q));
      TRY(check_arr(QO));
    }
    TRY(check_arr(K));
    TRY(check_arr(V));
    OPT4(seqs, "seqs");
    NEED4(positions, "positions");
    TRY(check_table(pages));
    const CacheArrs m = arrs_of(cache);
    TRY(check_cache_memory(cache, m));
    const Arr outs[] = {QO, m.a[0], m.a[1], m.a[2], m.a[3]};
    const Arr ins[] = {Q, K, V, flat_of("seqs", seqs, 4, t), flat_of("positions", positions, 4, t), table_of(pages),
                       freqs_of(g.rope)};
    for (const Arr& o : outs)
      for (const Arr& i : ins) TRY(no_overlap(o, i));
    for (int i = 1; i < 5; ++i) TRY(no_overlap(outs[0], outs[i]));
    TRY(check_stream(stream));
    g.tokens = tokens, g.q_heads = q ? q_heads : 0, g.kv_heads = cache->kv_heads, g.d = cache->head_dim;
    g.positions = positions, g.seqs = seqs;
    g.q = {q, tsq, hsq}, g.out = {q_out, tso, hso}, g.k = {k, tsk, hsk}, g.v = {v, tsv, hsv};
    FS_HIP(fs::launch_rotary(dt(cache->dtype), g, cache_of(cache, pages), S(stream)), "cache_append");
    return FS_OK;
  });
}

fs_status fs_paged_attention_workspace(const fs_attention_desc* d, const fs_kv_cache* cache,
                                       const fs_page_table* pages, size_t* bytes) {
  return entry([&]() -> fs_status {
    TRY(check_attention(d, cache, pages));
    if (!bytes) return fail(FS_ERR_INVALID, "bytes must not be NULL");
    *bytes = fs::attention_ws_bytes(dt(cache->dtype), d->q_heads, d->new_tokens, cache_of(cache, pages));
    return FS_OK;
  });
}

fs_status fs_paged_attention(const fs_attention_desc* d, const fs_kv_cache* cache, const void* q, int64_t tsq,
                             int64_t hsq, const int32_t* lengths, const fs_page_table* pages, void* out,
                             int64_t tso, int64_t hso, float* lse, void* ws, size_t ws_bytes, fs_stream stream) {
  return entry([&] {
    return paged_attention(d, cache, q, tsq, hsq, false, nullptr, lengths, pages, out, tso, hso, lse, ws, ws_bytes,
                           stream);
  });
}

fs_status fs_paged_attention_at(const fs_attention_desc* d, const fs_kv_cache* cache, const void* q, int64_t tsq,
                                int64_t hsq, const int32_t* positions, const int32_t* lengths,
                                const fs_page_table* pages, void* out, int64_t tso, int64_t hso, float* lse, void* ws,
                                size_t ws_bytes, fs_stream stream) {
  return entry([&] {
    return paged_attention(d, cache, q, tsq, hsq, true, positions, lengths, pages, out, tso, hso, lse, ws, ws_bytes,
                           stream);
  });
}

}  // extern "C"
