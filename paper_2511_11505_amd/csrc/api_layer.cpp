// C entry points of the dense sublayer: the linear with its epilogue, layer
// norm, their backward passes, and 8-bit activation checkpoints.  Every check
// runs on the host before anything is enqueued; no exception leaves an entry.

#include "api_common.hpp"
#include "internal.hpp"

namespace {

// A matrix argument: base, rows, columns, row stride (elements), element
// bytes.
struct Mat {
  const char* name;
  const void* p;
  int64_t rows, cols, ld;
  size_t es;
};

fs_status check_mat(const Mat& m) {
  if (!m.p) return fail(FS_ERR_INVALID, std::string(m.name) + " must not be NULL");
  if (!aligned_to(m.p, m.es))
    return fail(FS_ERR_INVALID, std::string(m.name) + " must be aligned to its elements");
  if (m.ld < m.cols)
    return fail(FS_ERR_INVALID, std::string(m.name) + ": the row stride must be >= the columns");
  if (m.ld > ((int64_t)1 << 40)) return fail(FS_ERR_UNSUPPORTED, std::string(m.name) + ": row stride too large");
  return FS_OK;
}

// Whether an output shares bytes with an input: the same base, or where both
// are gapless (of views with gaps the bytes between rows may be another's).
bool overlap(const Mat& a, const Mat& b) {
  if (!a.p || !b.p) return false;
  if (a.p == b.p) return true;
  if ((a.rows > 1 && a.ld != a.cols) || (b.rows > 1 && b.ld != b.cols)) return false;
  const char *x = (const char*)a.p, *y = (const char*)b.p;
  return x < y + b.rows * b.cols * b.es && y < x + a.rows * a.cols * a.es;
}
fs_status no_overlap(const Mat& out, const Mat& in) {
  if (overlap(out, in)) return fail(FS_ERR_INVALID, std::string(out.name) + " and " + in.name + " overlap");
  return FS_OK;
}

// Outputs share bytes with no input and not with each other.
template <size_t NO, size_t NI>
fs_status check_apart(const Mat (&outs)[NO], const Mat (&ins)[NI]) {
  for (size_t i = 0; i < NO; ++i) {
    for (const Mat& in : ins)
      if (overlap(outs[i], in)) return no_overlap(outs[i], in);
    for (size_t j = i + 1; j < NO; ++j)
      if (overlap(outs[i], outs[j])) return no_overlap(outs[i], outs[j]);
  }
  return FS_OK;
}
Mat vec_of(const float* p, const char* name, int64_t n) { return {name, p, 1, n, n, 4}; }
// (bytes of a workspace that are not used: not there)
Mat ws_of(const void* ws, size_t need) { return {"ws", need ? ws : nullptr, 1, (int64_t)need, (int64_t)need, 1}; }

int64_t blocks_of(int64_t cols) { return (cols + 31) / 32; }

// A saved activation [rows, cols].  As an input it has rows or codes, as an
// output either or both.
fs_status check_saved(const fs_saved* s, const char* name, int64_t rows, int64_t cols, size_t es,
                      bool input, bool codes_only) {
  if (!s) return FS_OK;
  if (!s->rows && !s->codes) return fail(FS_ERR_INVALID, std::string(name) + " has neither rows nor codes");
  if (s->rows && codes_only) return fail(FS_ERR_INVALID, std::string(name) + " is kept as codes only");
  if (input && s->rows && s->codes)
    return fail(FS_ERR_INVALID, std::string(name) + " has both rows and codes");
  if (s->codes && !s->scales) return fail(FS_ERR_INVALID, std::string(name) + " has codes without scales");
  if (s->rows) return check_mat({name, s->rows, rows, cols, s->ld, es});
  return FS_OK;
}
Mat rows_of(const fs_saved* s, const char* name, int64_t rows, int64_t cols, size_t es) {
  return {name, s ? s->rows : nullptr, rows, cols, s ? s->ld : cols, es};
}
Mat codes_of(const fs_saved* s, const char* name, int64_t rows, int64_t cols) {
  return {name, s ? s->codes : nullptr, rows, cols, cols, 1};
}
Mat scales_of(const fs_saved* s, const char* name, int64_t rows, int64_t cols) {
  return {name, s && s->codes ? s->scales : nullptr, rows, blocks_of(cols), blocks_of(cols), 1};
}

// Workgroups of a grid over r x c tiles of 64 (256 threads each; a grid holds
// fewer than 2^32 threads).
bool grid_ok(int64_t r, int64_t c) { return (r + 63) / 64 * ((c + 63) / 64) < ((int64_t)1 << 24); }

fs_status check_linear(const fs_linear_desc* d) {
  if (!d) return fail(FS_ERR_INVALID, "desc must not be NULL");
  if (d->abi_version != FS_ABI_VERSION) return fail(FS_ERR_INVALID, "desc->abi_version mismatch");
  TRY(check_dtype(d->dtype));
  if (d->act < FS_ACT_NONE || d->act > FS_ACT_SILU) return fail(FS_ERR_INVALID, "act must be an fs_act");
  if (d->m < 0 || d->n <= 0 || d->k <= 0) return fail(FS_ERR_INVALID, "m >= 0, n > 0, k > 0 required");
  if (d->m > (1 << 24) || d->n > (1 << 24) || d->k > (1 << 24))
    return fail(FS_ERR_UNSUPPORTED, "m, n and k must be <= 2^24");
  if (!grid_ok(d->m, d->n) || !grid_ok(d->m, d->k) || !grid_ok(d->n, d->k))
    return fail(FS_ERR_UNSUPPORTED, "m, n, k: a product of more than 2^24 tiles of 64 x 64");
  return FS_OK;
}

fs_status check_norm(const fs_norm_desc* d) {
  if (!d) return fail(FS_ERR_INVALID, "desc must not be NULL");
  if (d->abi_version != FS_ABI_VERSION) return fail(FS_ERR_INVALID, "desc->abi_version mismatch");
  TRY(check_dtype(d->dtype));
  if (d->rows < 0 || d->cols <= 0) return fail(FS_ERR_INVALID, "rows >= 0, cols > 0 required");
  if (d->cols > fs::kNormMaxCols) return fail(FS_ERR_UNSUPPORTED, "cols must be <= 32768");
  if (d->rows > (1 << 21)) return fail(FS_ERR_UNSUPPORTED, "rows must be <= 2^21");
  if (d->center != 0 && d->center != 1) return fail(FS_ERR_INVALID, "center must be 0/1");
  if (!(d->eps > 0.f) || !(d->eps < 1e30f)) return fail(FS_ERR_INVALID, "eps must be > 0 and finite");
  return FS_OK;
}

}  // namespace

extern "C" {

fs_status fs_linear_workspace(const fs_linear_desc* d, int32_t op, size_t* bytes) {
  return entry([&]() -> fs_status {
    TRY(check_linear(d));
    if (!bytes) return fail(FS_ERR_INVALID, "bytes must not be NULL");
    if (op == FS_OP_LINEAR)
      *bytes = fs::linear_ws_bytes(dt(d->dtype), d->m, d->n, d->k);
    else if (op == FS_OP_LINEAR_BACKWARD)
      *bytes = fs::linear_backward_ws_bytes(dt(d->dtype), d->act, d->m, d->n, d->k);
    else
      return fail(FS_ERR_INVALID, "op must be FS_OP_LINEAR or FS_OP_LINEAR_BACKWARD");
    return FS_OK;
  });
}

fs_status fs_linear(const fs_linear_desc* d, const void* a, int64_t lda, const void* w, int64_t ldw,
                    const float* bias, const void* residual, int64_t ldr, void* out, int64_t ldo,
                    const fs_saved* save_z, const fs_saved* save_out, void* ws, size_t ws_bytes,
                    fs_stream stream) {
  return entry([&]() -> fs_status {
    TRY(check_linear(d));
    if (d->m == 0) return FS_OK;
    const size_t es = elem(d->dtype);
    const int64_t m = d->m, n = d->n, k = d->k;
    const Mat A{"a", a, m, k, lda, es}, W{"w", w, n, k, ldw, es}, R{"residual", residual, m, n, ldr, es},
        O{"out", out, m, n, ldo, es};
    TRY(check_mat(A));
    TRY(check_mat(W));
    TRY(check_mat(O));
    if (residual) TRY(check_mat(R));
    OPT4(bias, "bias");
    TRY(check_saved(save_z, "save_z", m, n, es, false, false));
    TRY(check_saved(save_out, "save_out", m, n, es, false, true));
    const size_t need = fs::linear_ws_bytes(dt(d->dtype), d->m, d->n, d->k);
    if (ws_bytes < need)
      return fail(FS_ERR_WORKSPACE, "workspace smaller than fs_linear_workspace(FS_OP_LINEAR)");
    if (need) NEED(ws, "ws");
    const Mat Z = rows_of(save_z, "save_z", m, n, es);
    const Mat outs[] = {O, Z, codes_of(save_z, "save_z", m, n), scales_of(save_z, "save_z", m, n),
                        codes_of(save_out, "save_out", m, n), scales_of(save_out, "save_out", m, n),
                        ws_of(ws, need)};
    const Mat ins[] = {A, W, vec_of(bias, "bias", n)};
    TRY(check_apart(outs, ins));
    // (out may be residual itself: each element is read before it is written)
    for (const Mat& x : outs)
      if (!(x.p == O.p && out == residual && ldo == ldr)) TRY(no_overlap(x, R));
    TRY(check_stream(stream));
    fs::LinearOut o{bias, d->act, residual, ldr, out, ldo, nullptr, 0, nullptr, nullptr, nullptr, nullptr};
    if (save_z) o.z = save_z->rows, o.ldz = save_z->ld, o.z_codes = save_z->codes;
    // (scales without codes are not part of the call: the checks above left them out)
    if (o.z_codes) o.z_scales = save_z->scales;
    if (save_out) o.out_codes = save_out->codes, o.out_scales = save_out->scales;
    fs::prof_begin(FS_K_DENSE, S(stream));
    const hipError_t e =
        fs::launch_linear(dt(d->dtype), d->m, d->n, d->k, a, lda, w, ldw, o, ws, S(stream));
    fs::prof_end(FS_K_DENSE, S(stream));
    FS_HIP(e, "linear");
    return FS_OK;
  });
}

fs_status fs_linear_backward(const fs_linear_desc* d, const void* dout, int64_t ldo, const fs_saved* a,
                             const void* w, int64_t ldw, const fs_saved* z, void* da, int64_t ldda,
                             void* dw, int64_t lddw, float* dbias, void* ws, size_t ws_bytes,
                             fs_stream stream) {
  return entry([&]() -> fs_status {
    TRY(check_linear(d));
    const size_t es = elem(d->dtype);
    const int64_t m = d->m, n = d->n, k = d->k;
    const bool act = d->act != FS_ACT_NONE;
    if (!da && !dw && !dbias) return fail(FS_ERR_INVALID, "da, dw and dbias are all NULL");
    const Mat G{"dout", dout, m, n, ldo, es}, W{"w", w, n, k, ldw, es}, DA{"da", da, m, k, ldda, es},
        DW{"dw", dw, n, k, lddw, es};
    if (m > 0) {
      TRY(check_mat(G));
      if (da) TRY(check_mat(W));
      if (dw && !a) return fail(FS_ERR_INVALID, "dw needs a");
      if (act && !z) return fail(FS_ERR_INVALID, "z must not be NULL (act is not FS_ACT_NONE)");
      TRY(check_saved(a, "a", m, k, es, true, false));
      if (act) TRY(check_saved(z, "z", m, n, es, true, false));
      if (da) TRY(check_mat(DA));
    }
    if (dw) TRY(check_mat(DW));
    OPT4(dbias, "dbias");
    const size_t need = fs::linear_backward_ws_bytes(dt(d->dtype), d->act, d->m, d->n, d->k);
    if (ws_bytes < need)
      return fail(FS_ERR_WORKSPACE, "workspace smaller than fs_linear_workspace(FS_OP_LINEAR_BACKWARD)");
    if (need) NEED(ws, "ws");
    const Mat outs[] = {DA, DW, vec_of(dbias, "dbias", n), ws_of(ws, need)};
    const Mat ins[] = {G, W, rows_of(a, "a", m, k, es), codes_of(a, "a", m, k), scales_of(a, "a", m, k),
                       rows_of(z, "z", m, n, es), codes_of(z, "z", m, n), scales_of(z, "z", m, n)};
    if (m > 0) TRY(check_apart(outs, ins));
    TRY(check_stream(stream));
    fs::LinearBack b{};
    b.act = d->act, b.m = d->m, b.n = d->n, b.k = d->k;
    b.dout = dout, b.ldo = ldo, b.w = w, b.ldw = ldw;
    if (a) b.a = a->rows, b.lda = a->ld, b.a_codes = a->codes, b.a_scales = a->scales;
    if (act && z) b.z = z->rows, b.ldz = z->ld, b.z_codes = z->codes, b.z_scales = z->scales;
    b.da = da, b.ldda = ldda, b.dw = dw, b.lddw = lddw, b.dbias = dbias;
    FS_HIP(fs::launch_linear_backward(dt(d->dtype), b, ws, S(stream)), "linear_backward");
    return FS_OK;
  });
}

fs_status fs_layer_norm_workspace(const fs_norm_desc* d, size_t* bytes) {
  return entry([&]() -> fs_status {
    TRY(check_norm(d));
    if (!bytes) return fail(FS_ERR_INVALID, "bytes must not be NULL");
    *bytes = fs::norm_ws_bytes(d->rows, d->cols);
    return FS_OK;
  });
}

fs_status fs_layer_norm(const fs_norm_desc* d, const void* x, int64_t ldx, const void* add,
                        int64_t ldadd, const float* gamma, const float* beta, void* sum_out,
                        int64_t ldsum, void* y, int64_t ldy, float* mean, float* rstd,
                        const fs_saved* save_in, const fs_saved* save_y, fs_stream stream) {
  return entry([&]() -> fs_status {
    TRY(check_norm(d));
    if (d->rows == 0) return FS_OK;
    const size_t es = elem(d->dtype);
    const int64_t r = d->rows, c = d->cols;
    const Mat X{"x", x, r, c, ldx, es}, ADD{"add", add, r, c, ldadd, es}, SUM{"sum_out", sum_out, r, c, ldsum, es},
        Y{"y", y, r, c, ldy, es};
    TRY(check_mat(X));
    TRY(check_mat(Y));
    if (add) TRY(check_mat(ADD));
    if (sum_out) TRY(check_mat(SUM));
    for (const void* p : {(const void*)gamma, (const void*)beta, (const void*)mean, (const void*)rstd})
      OPT4(p, "gamma, beta, mean and rstd");
    TRY(check_saved(save_in, "save_in", r, c, es, false, true));
    TRY(check_saved(save_y, "save_y", r, c, es, false, true));
    const Mat outs[] = {SUM, Y, vec_of(mean, "mean", r), vec_of(rstd, "rstd", r),
                        codes_of(save_in, "save_in", r, c), scales_of(save_in, "save_in", r, c),
                        codes_of(save_y, "save_y", r, c), scales_of(save_y, "save_y", r, c)};
    const Mat ins[] = {vec_of(gamma, "gamma", c), vec_of(beta, "beta", c)};
    TRY(check_apart(outs, ins));
    // (sum_out and y may be an input itself: a row is read before it is written)
    for (const Mat& o : outs)
      for (const Mat& i : {X, ADD})
        if (!((o.p == sum_out || o.p == y) && o.p == i.p && o.ld == i.ld)) TRY(no_overlap(o, i));
    TRY(check_stream(stream));
    fs::NormArgs g{};
    g.rows = r, g.cols = d->cols, g.center = d->center, g.eps = d->eps;
    g.x = x, g.ldx = ldx, g.add = add, g.ldadd = ldadd, g.gamma = gamma, g.beta = beta;
    g.sum = sum_out, g.ldsum = ldsum, g.y = y, g.ldy = ldy, g.mean = mean, g.rstd = rstd;
    if (save_in) g.in_codes = save_in->codes, g.in_scales = save_in->scales;
    if (save_y) g.y_codes = save_y->codes, g.y_scales = save_y->scales;
    FS_HIP(fs::launch_norm(dt(d->dtype), g, S(stream)), "layer_norm");
    return FS_OK;
  });
}

fs_status fs_layer_norm_backward(const fs_norm_desc* d, const void* dy, int64_t lddy, const fs_saved* x,
                                 const float* mean, const float* rstd, const float* gamma,
                                 const void* dres, int64_t lddres, void* dx, int64_t lddx,
                                 float* dgamma, float* dbeta, void* ws, size_t ws_bytes,
                                 fs_stream stream) {
  return entry([&]() -> fs_status {
    TRY(check_norm(d));
    const size_t es = elem(d->dtype);
    const int64_t r = d->rows, c = d->cols;
    const Mat DY{"dy", dy, r, c, lddy, es}, DR{"dres", dres, r, c, lddres, es}, DX{"dx", dx, r, c, lddx, es};
    OPT4(dgamma, "dgamma");
    OPT4(dbeta, "dbeta");
    if (r > 0) {
      TRY(check_mat(DY));
      if (!x) return fail(FS_ERR_INVALID, "x must not be NULL");
      TRY(check_saved(x, "x", r, c, es, true, false));
      TRY(check_mat(DX));
      if (dres) TRY(check_mat(DR));
      NEED4(rstd, "rstd");
      if (d->center) NEED4(mean, "mean");
      OPT4(gamma, "gamma");
    }
    const bool grads = dgamma || dbeta;
    const size_t need = grads ? fs::norm_ws_bytes(r, d->cols) : 0;
    if (ws_bytes < need) return fail(FS_ERR_WORKSPACE, "workspace smaller than fs_layer_norm_workspace");
    if (need) NEED(ws, "ws");
    if (r > 0) {
      const Mat outs[] = {DX, vec_of(dgamma, "dgamma", c), vec_of(dbeta, "dbeta", c), ws_of(ws, need)};
      const Mat ins[] = {rows_of(x, "x", r, c, es), codes_of(x, "x", r, c), scales_of(x, "x", r, c),
                         vec_of(mean, "mean", r), vec_of(rstd, "rstd", r), vec_of(gamma, "gamma", c)};
      TRY(check_apart(outs, ins));
      // (dx may be dy or dres itself: a row is read before it is written)
      for (const Mat& o : outs)
        for (const Mat& i : {DY, DR})
          if (!(o.p == dx && i.p == dx && i.ld == lddx)) TRY(no_overlap(o, i));
    }
    if (r == 0 && !grads) return FS_OK;
    TRY(check_stream(stream));
    if (r == 0) {
      // no rows: the gradients are 0
      FS_HIP(fs::launch_colsum(nullptr, 0, d->cols, dgamma, dbeta, S(stream)), "layer_norm_backward");
      return FS_OK;
    }
    fs::NormBackArgs g{};
    g.rows = r, g.cols = d->cols, g.center = d->center;
    g.dy = dy, g.lddy = lddy, g.x = x->rows, g.ldx = x->ld, g.x_codes = x->codes, g.x_scales = x->scales;
    g.mean = d->center ? mean : nullptr, g.rstd = rstd, g.gamma = gamma;
    g.dres = dres, g.lddres = lddres, g.dx = dx, g.lddx = lddx;
    g.part = grads ? (float*)ws : nullptr;
    FS_HIP(fs::launch_norm_backward(dt(d->dtype), g, dgamma, dbeta, S(stream)), "layer_norm_backward");
    return FS_OK;
  });
}

static fs_status ckpt_checks(int32_t dtype, int64_t rows, int32_t cols, const Mat& m, const void* codes,
                             const void* scales) {
  TRY(check_dtype(dtype));
  if (rows < 0 || cols <= 0) return fail(FS_ERR_INVALID, "rows >= 0 and cols > 0 required");
  if (cols > (1 << 28)) return fail(FS_ERR_UNSUPPORTED, "cols must be <= 2^28");
  if (rows == 0) return FS_OK;
  TRY(check_mat(m));
  if (!codes || !scales) return fail(FS_ERR_INVALID, "codes and scales must not be NULL");
  const Mat c{"codes", codes, rows, cols, cols, 1};
  const Mat s{"scales", scales, rows, blocks_of(cols), blocks_of(cols), 1};
  TRY(no_overlap(m, c));
  TRY(no_overlap(m, s));
  return no_overlap(c, s);
}

fs_status fs_checkpoint_fp8(int32_t dtype, int64_t rows, int32_t cols, const void* src, int64_t lds,
                            uint8_t* codes, uint8_t* scales, fs_stream stream) {
  return entry([&]() -> fs_status {
    TRY(ckpt_checks(dtype, rows, cols, {"src", src, rows, cols, lds, elem(dtype)}, codes, scales));
    if (rows == 0) return FS_OK;
    TRY(check_stream(stream));
    FS_HIP(fs::launch_checkpoint(dt(dtype), src, lds, rows, cols, codes, scales, S(stream)),
           "checkpoint_fp8");
    return FS_OK;
  });
}

fs_status fs_checkpoint_restore(int32_t dtype, int64_t rows, int32_t cols, const uint8_t* codes,
                                const uint8_t* scales, void* dst, int64_t ldd, fs_stream stream) {
  return entry([&]() -> fs_status {
    TRY(ckpt_checks(dtype, rows, cols, {"dst", dst, rows, cols, ldd, elem(dtype)}, codes, scales));
    if (rows == 0) return FS_OK;
    TRY(check_stream(stream));
    FS_HIP(fs::launch_restore(dt(dtype), codes, scales, rows, cols, dst, ldd, S(stream)),
           "checkpoint_restore");
    return FS_OK;
  });
}

}  // extern "C"
