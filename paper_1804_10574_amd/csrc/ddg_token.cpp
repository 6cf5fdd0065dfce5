// C boundary of the operators of token models (include/ddg.h): what they refuse, and the plans of their launches.
#include "ddg_token.h"

#include <math.h>
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include "ddg_internal.h"

using namespace ddg;

namespace {

ddg_status fail(ddg_status st, const char* fmt, ...) {
  char msg[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(msg, sizeof(msg), fmt, ap);
  va_end(ap);
  ddg_internal_set_error(msg);
  return st;
}

ddg_status done(hipError_t e, const char* what) {
  return e == hipSuccess ? DDG_OK : fail(DDG_ERR_DEVICE, "%s: %s", what, hipGetErrorString(e));
}

// A tensor argument: [rows][cols] elements of `size` bytes, `ld` elements from row to row
struct Arg {
  const char* name;
  const void* p;
  long rows, cols, ld;
  size_t size;
  bool out;
  uintptr_t lo() const { return (uintptr_t)p; }
  uintptr_t hi() const { return (uintptr_t)p + ((size_t)(rows - 1) * ld + cols) * size; }
  bool empty() const { return !p || rows < 1 || cols < 1; }
};

// Columns of one wider tensor, none of them in both
bool side_by_side(const Arg& a, const Arg& b) {
  const uintptr_t row = a.ld * a.size, wa = a.cols * a.size, wb = b.cols * b.size;
  if (row != b.ld * b.size) return false;
  const uintptr_t apart = a.lo() <= b.lo() ? (b.lo() - a.lo()) % row : (row - (a.lo() - b.lo()) % row) % row;
  return apart >= wa && apart + wb <= row;
}

// Pointers lie on their elements, and no output overlaps another argument; `same` names pairs that may be one tensor.
struct Pair { const char* a; const char* b; };
template <int N, int S> ddg_status check_args(const Arg (&args)[N], const Pair (&same)[S]) {
  for (const Arg& a : args)
    if (a.lo() % a.size) return fail(DDG_ERR_INVALID_ARG, "%s must be aligned to its elements of %zu bytes", a.name, a.size);
  for (int i = 0; i < N; ++i)
    for (int j = 0; j < N; ++j) {
      const Arg& a = args[i]; const Arg& b = args[j];
      if (i == j || !a.out || (b.out && j < i) || a.empty() || b.empty()) continue;
      if (a.hi() <= b.lo() || b.hi() <= a.lo() || side_by_side(a, b)) continue;
      bool allowed = false;
      for (const Pair& s : same)
        if (s.a && !strcmp(s.a, a.name) && !strcmp(s.b, b.name)) allowed = a.p == b.p && a.ld == b.ld;
      if (!allowed) return fail(DDG_ERR_INVALID_ARG, "%s overlaps %s", a.name, b.name);
    }
  return DDG_OK;
}
constexpr Pair NONE[] = {{nullptr, nullptr}};

// Row numbers plus the rows of a round of workgroups stay inside an int, and a tensor's extent in bytes inside 63 bits
constexpr int ROWS_MAX = 1 << 30;
constexpr long LD_MAX = 1l << 30;

ddg_status check_rows(const char* what, int rows, int cols, int dtype) {
  if (dtype != DDG_F32 && dtype != DDG_BF16) return fail(DDG_ERR_INVALID_ARG, "%s: dtype must be DDG_F32 or DDG_BF16", what);
  if (rows < 0 || cols < 1) return fail(DDG_ERR_SHAPE, "%s: need rows >= 0 and columns >= 1 (%d, %d)", what, rows, cols);
  if (rows > ROWS_MAX) return fail(DDG_ERR_SHAPE, "%s: at most %d rows (%d)", what, ROWS_MAX, rows);
  return DDG_OK;
}
ddg_status check_ld(const char* name, long* ld, int cols) {
  if (*ld == 0) *ld = cols;
  if (*ld < cols) return fail(DDG_ERR_SHAPE, "%s = %ld is less than a row of %d", name, *ld, cols);
  if (*ld > LD_MAX) return fail(DDG_ERR_SHAPE, "%s = %ld is more than %ld", name, *ld, LD_MAX);
  return DDG_OK;
}
ddg_status check_drop(float p, uint64_t seed, uint64_t step, DropArgs* d) {
  if (!(p >= 0.f && p < 1.f)) return fail(DDG_ERR_INVALID_ARG, "p must be in [0,1)");
  const long t = lrint(65536.0 * (double)p);
  d->limit = (uint32_t)(t > 65535 ? 65535 : t);
  d->scale = (float)(65536.0 / (65536.0 - d->limit));
  d->key0 = (uint32_t)seed; d->key1 = (uint32_t)(seed >> 32);
  d->step0 = (uint32_t)step; d->step1 = (uint32_t)(step >> 32);
  return DDG_OK;
}
#define CHECK(expr)                          \
  do {                                       \
    const ddg_status st_ = (expr);           \
    if (st_ != DDG_OK) return st_;           \
  } while (0)

ddg_status join_desc(const ddg_join_desc* in, ddg_join_desc* d, uint64_t step, JoinArgs* a) {
  if (!in) return fail(DDG_ERR_INVALID_ARG, "desc is null");
  *d = *in;
  CHECK(check_rows("join", d->rows, d->cols, d->dtype));
  if (d->cols > JOIN_COLS_MAX) return fail(DDG_ERR_SHAPE, "join: at most %d columns (%d)", JOIN_COLS_MAX, d->cols);
  if (!(d->eps > 0.f)) return fail(DDG_ERR_INVALID_ARG, "eps must be > 0");
  CHECK(check_ld("ld_y", &d->ld_y, d->cols));
  CHECK(check_ld("ld_residual", &d->ld_residual, d->cols));
  CHECK(check_ld("ld_x", &d->ld_x, d->cols));
  CHECK(check_ld("ld_out", &d->ld_out, d->cols));
  if (d->group != 0 && d->group != 128) return fail(DDG_ERR_INVALID_ARG, "group must be 0 or 128");
  *a = JoinArgs{};
  CHECK(check_drop(d->p, d->seed, step, &a->drop));
  a->ld_y = d->ld_y; a->ld_residual = d->ld_residual; a->ld_x = d->ld_x; a->ld_out = d->ld_out;
  a->rows = d->rows; a->cols = d->cols; a->dtype = d->dtype; a->group = d->group; a->eps = d->eps;
  return DDG_OK;
}

ddg_status join_forward(const ddg_join_desc* desc, uint64_t step, const void* y, const void* residual, const float* gain, void* x_out, void* out, uint8_t* q,
                        float* scale, float* rstd) {
  ddg_join_desc d;
  JoinArgs a;
  CHECK(join_desc(desc, &d, step, &a));
  const size_t size = dtype_size(d.dtype);
  const int groups = d.group ? (d.cols + d.group - 1) / d.group : 1;
  const Arg args[] = {{"x_out", x_out, d.rows, d.cols, d.ld_x, size, true},
                      {q ? "q" : "out", q ? q : out, d.rows, d.cols, d.ld_out, q ? 1 : size, true},
                      {"scale", scale, d.rows, groups, groups, 4, true},
                      {"rstd", rstd, d.rows, 1, 1, 4, true},
                      {"y", y, d.rows, d.cols, d.ld_y, size, false},
                      {"residual", residual, d.rows, d.cols, d.ld_residual, size, false},
                      {"gain", gain, 1, d.cols, d.cols, 4, false}};
  const Pair same[] = {{"x_out", "y"}, {"x_out", "residual"}};
  CHECK(check_args(args, same));
  if (d.rows == 0 || d.dry_run) return DDG_OK;
  a.y = y; a.residual = residual; a.gain = gain; a.x = x_out; a.out = out; a.q = q; a.scale = scale; a.rstd = rstd;
  return done(join_forward_launch(a, (hipStream_t)d.stream), "join");
}

// Longest row of a tensor that the products read, in bytes: offsets inside a tile of 256 rows have 31 bits
constexpr long ROW_BYTES_MAX = (1l << 23) - 1;
// One workgroup of 256 threads a token: a launch holds fewer than 2^32 threads
constexpr int TOKENS_MAX = 1 << 23;

ddg_status vocab_desc(const ddg_vocab_desc* in, ddg_vocab_desc* d) {
  if (!in) return fail(DDG_ERR_INVALID_ARG, "desc is null");
  *d = *in;
  CHECK(check_rows("vocab loss", d->tokens, d->dim, d->dtype));
  if (d->tokens > TOKENS_MAX) return fail(DDG_ERR_SHAPE, "vocab loss: at most %d tokens (%d)", TOKENS_MAX, d->tokens);
  if (d->vocab < 1) return fail(DDG_ERR_SHAPE, "vocab loss: need vocab >= 1 (%d)", d->vocab);
  CHECK(check_ld("ld_h", &d->ld_h, d->dim));
  CHECK(check_ld("ld_w", &d->ld_w, d->dim));
  CHECK(check_ld("ld_dh", &d->ld_dh, d->dim));
  CHECK(check_ld("ld_dw", &d->ld_dw, d->dim));
  const long size = (long)dtype_size(d->dtype), most = ROW_BYTES_MAX / size;
  if (d->vocab > most - 256 || d->dim > most - 256 || d->ld_h > most || d->ld_w > most)
    return fail(DDG_ERR_SHAPE, "vocab loss: vocabulary, width and row strides of h and w are at most %ld elements", most - 256);
  return DDG_OK;
}
bool in_pieces(const void* p, long ld, int dim, size_t size) { return (uintptr_t)p % 16 == 0 && (size_t)ld * size % 16 == 0 && (size_t)dim * size % 16 == 0; }

}  // namespace

extern "C" {

ddg_status ddg_dropout(const ddg_dropout_desc* desc, uint64_t step, const void* x, void* y) {
  if (!desc) return fail(DDG_ERR_INVALID_ARG, "desc is null");
  ddg_dropout_desc d = *desc;
  CHECK(check_rows("dropout", d.rows, d.cols, d.dtype));
  CHECK(check_ld("ld_x", &d.ld_x, d.cols));
  CHECK(check_ld("ld_y", &d.ld_y, d.cols));
  DropoutArgs a{};
  CHECK(check_drop(d.p, d.seed, step, &a.drop));
  if (d.rows && (!x || !y)) return fail(DDG_ERR_INVALID_ARG, "x and y must not be null");
  const size_t size = dtype_size(d.dtype);
  const Arg args[] = {{"y", y, d.rows, d.cols, d.ld_y, size, true}, {"x", x, d.rows, d.cols, d.ld_x, size, false}};
  const Pair same[] = {{"y", "x"}};
  CHECK(check_args(args, same));
  if (d.rows == 0 || d.dry_run) return DDG_OK;
  a.x = x; a.y = y; a.ld_x = d.ld_x; a.ld_y = d.ld_y; a.rows = d.rows; a.cols = d.cols; a.dtype = d.dtype;
  return done(dropout_launch(a, (hipStream_t)d.stream), "dropout");
}

ddg_status ddg_join_norm(const ddg_join_desc* desc, uint64_t step, const void* y, const void* residual, const float* gain, void* x_out, void* out,
                         float* rstd) {
  if (desc && desc->rows && (!y || !out)) return fail(DDG_ERR_INVALID_ARG, "y and out must not be null");
  return join_forward(desc, step, y, residual, gain, x_out, out, nullptr, nullptr, rstd);
}

ddg_status ddg_join_norm_q8(const ddg_join_desc* desc, uint64_t step, const void* y, const void* residual, const float* gain, void* x_out, uint8_t* q,
                            float* scale, float* rstd) {
  if (desc && desc->rows && (!y || !q || !scale)) return fail(DDG_ERR_INVALID_ARG, "y, q and scale must not be null");
  return join_forward(desc, step, y, residual, gain, x_out, nullptr, q, scale, rstd);
}

size_t ddg_join_norm_workspace(const ddg_join_desc* desc) {
  ddg_join_desc d;
  JoinArgs a;
  return join_desc(desc, &d, 0, &a) == DDG_OK ? (size_t)join_groups(d.rows, d.cols) * d.cols * 4 : 0;
}

ddg_status ddg_join_norm_backward(const ddg_join_desc* desc, uint64_t step, const void* x, const float* rstd, const float* gain, const void* d_out,
                                  const void* d_x, void* d_residual, void* d_y, float* d_gain, void* workspace, size_t workspace_bytes) {
  ddg_join_desc d;
  JoinArgs a;
  CHECK(join_desc(desc, &d, step, &a));
  if (d.rows && (!x || !rstd || !d_out)) return fail(DDG_ERR_INVALID_ARG, "x, rstd and d_out must not be null");
  if (!d_residual && !d_y && !d_gain) return fail(DDG_ERR_INVALID_ARG, "nothing to compute: d_residual, d_y and d_gain are null");
  const size_t size = dtype_size(d.dtype), need = d_gain ? ddg_join_norm_workspace(desc) : 0;
  if (need && (!workspace || workspace_bytes < need)) return fail(DDG_ERR_INVALID_ARG, "d_gain needs a workspace of %zu bytes (%zu)", need, workspace_bytes);
  if (need && (uintptr_t)workspace % 16) return fail(DDG_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
  const Arg args[] = {{"d_residual", d_residual, d.rows, d.cols, d.ld_residual, size, true},
                      {"d_y", d_y, d.rows, d.cols, d.ld_y, size, true},
                      {"d_gain", d_gain, 1, d.cols, d.cols, 4, true},
                      {"workspace", need ? workspace : nullptr, 1, (long)need, (long)need, 1, true},
                      {"x", x, d.rows, d.cols, d.ld_x, size, false},
                      {"rstd", rstd, d.rows, 1, 1, 4, false},
                      {"gain", gain, 1, d.cols, d.cols, 4, false},
                      {"d_out", d_out, d.rows, d.cols, d.ld_out, size, false},
                      {"d_x", d_x, d.rows, d.cols, d.ld_x, size, false}};
  const Pair same[] = {{"d_residual", "d_x"}};
  CHECK(check_args(args, same));
  if (d.dry_run || (d.rows == 0 && !d_gain)) return DDG_OK;
  a.x = const_cast<void*>(x); a.rstd = const_cast<float*>(rstd); a.gain = gain; a.d_out = d_out; a.d_x = d_x;
  a.d_residual = d_residual; a.d_y = d_y; a.d_gain = d_gain; a.partial = (float*)workspace;
  return done(join_backward_launch(a, (hipStream_t)d.stream), "join backward");
}

size_t ddg_vocab_loss_workspace(const ddg_vocab_desc* desc, int gradients) {
  ddg_vocab_desc d;
  if (vocab_desc(desc, &d) != DDG_OK) return 0;
  // (pointers are not known yet: room for the copies that unaligned ones take is part of it where strides, width or the caller say so)
  VocabPlan p{};
  p.tokens = d.tokens; p.dim = d.dim; p.vocab = d.vocab; p.dtype = d.dtype; p.grads = gradients != 0; p.dw_f32 = d.dw_f32 != 0;
  const size_t size = dtype_size(d.dtype);
  p.pack_h = d.unaligned || !in_pieces(nullptr, d.ld_h, d.dim, size);
  p.pack_w = d.unaligned || !in_pieces(nullptr, d.ld_w, d.dim, size);
  vocab_plan(&p);
  return p.bytes;
}

ddg_status ddg_vocab_loss(const ddg_vocab_desc* desc, const void* h, const void* w, const int32_t* targets, const float* weights, float* loss,
                          float* row_loss, float* lse, void* dh, void* dw, void* workspace, size_t workspace_bytes) {
  ddg_vocab_desc d;
  CHECK(vocab_desc(desc, &d));
  if (!w || (d.tokens && (!h || !targets))) return fail(DDG_ERR_INVALID_ARG, "h, w and targets must not be null");
  if (!loss && !row_loss && !lse && !dh && !dw) return fail(DDG_ERR_INVALID_ARG, "nothing to compute: every result is null");
  const size_t size = dtype_size(d.dtype), size_dw = d.dw_f32 ? 4 : size;
  VocabPlan p{};
  p.tokens = d.tokens; p.dim = d.dim; p.vocab = d.vocab; p.dtype = d.dtype; p.grads = dh || dw; p.dw_f32 = d.dw_f32 != 0;
  p.pack_h = !in_pieces(h, d.ld_h, d.dim, size);
  p.pack_w = !in_pieces(w, d.ld_w, d.dim, size);
  vocab_plan(&p);
  if (!workspace || workspace_bytes < p.bytes)
    return fail(DDG_ERR_INVALID_ARG, "needs a workspace of %zu bytes (%zu)", p.bytes, workspace ? workspace_bytes : (size_t)0);
  if ((uintptr_t)workspace % 256) return fail(DDG_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
  const Arg args[] = {{"loss", loss, 1, 1, 1, 4, true},
                      {"row_loss", row_loss, d.tokens, 1, 1, 4, true},
                      {"lse", lse, d.tokens, 1, 1, 4, true},
                      {"dh", dh, d.tokens, d.dim, d.ld_dh, size, true},
                      {"dw", dw, d.vocab, d.dim, d.ld_dw, size_dw, true},
                      {"workspace", workspace, 1, (long)p.bytes, (long)p.bytes, 1, true},
                      {"h", h, d.tokens, d.dim, d.ld_h, size, false},
                      {"w", w, d.vocab, d.dim, d.ld_w, size, false},
                      {"targets", targets, d.tokens, 1, 1, 4, false},
                      {"weights", weights, d.tokens, 1, 1, 4, false}};
  CHECK(check_args(args, NONE));
  if (d.dry_run) return DDG_OK;
  VocabArgs a{h, w, targets, weights, loss, row_loss, lse, dh, dw, (unsigned char*)workspace, d.ld_h, d.ld_w, d.ld_dh, d.ld_dw};
  return done(vocab_launch(p, a, (hipStream_t)d.stream), "vocab loss");
}

}  // extern "C"
