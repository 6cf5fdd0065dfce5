// C boundary of the operators between the joins of a token model (include/ddg.h): what they refuse, and the plans of their launches.
#include "ddg_mixing.h"

#include <math.h>

#include "ddg_check.h"

using namespace ddg;

namespace {

ddg_status rotary_desc(const ddg_rotary_desc* in, ddg_rotary_desc* d) {
  if (!in) return fail(DDG_ERR_INVALID_ARG, "desc is null");
  *d = *in;
  CHECK(check_rows("rotary", d->rows, d->heads, d->dtype));
  if (d->dim < 1 || d->dim > ROTARY_DIM_MAX) return fail(DDG_ERR_SHAPE, "rotary: a head has 1 to %d columns (%d)", ROTARY_DIM_MAX, d->dim);
  if (d->rot == 0) d->rot = d->dim;
  if (d->rot < 2 || d->rot % 2 || d->rot > d->dim) return fail(DDG_ERR_SHAPE, "rotary: rot = %d must be even and within a head of %d", d->rot, d->dim);
  if ((long)d->heads * d->dim > LD_MAX) return fail(DDG_ERR_SHAPE, "rotary: rows of %d heads of %d are too long", d->heads, d->dim);
  CHECK(check_ld("ld_x", &d->ld_x, d->heads * d->dim));
  CHECK(check_ld("ld_y", &d->ld_y, d->heads * d->dim));
  if (!(d->base > 1.0) || !isfinite(d->base)) return fail(DDG_ERR_INVALID_ARG, "base must be > 1");
  if (!(d->factor >= 1.0) || !isfinite(d->factor)) return fail(DDG_ERR_INVALID_ARG, "factor must be 1 or more");
  if (!(d->context >= 0.0) || !isfinite(d->context)) return fail(DDG_ERR_INVALID_ARG, "context must be 0 or more");
  if (d->context > 0.0 && !(d->low >= 0.0 && d->high > d->low && isfinite(d->high))) return fail(DDG_ERR_INVALID_ARG, "need 0 <= low < high");
  if (!(d->magnitude > 0.f) || !isfinite(d->magnitude)) return fail(DDG_ERR_INVALID_ARG, "magnitude must be > 0");
  return DDG_OK;
}

ddg_status gated_desc(const ddg_gated_join_desc* in, ddg_gated_join_desc* d, GatedArgs* a) {
  if (!in) return fail(DDG_ERR_INVALID_ARG, "desc is null");
  *d = *in;
  CHECK(check_rows("gated join", d->rows, d->cols, d->dtype));
  if (d->cols > GATED_COLS_MAX) return fail(DDG_ERR_SHAPE, "gated join: at most %d columns (%d)", GATED_COLS_MAX, d->cols);
  if (!(d->eps > 0.f)) return fail(DDG_ERR_INVALID_ARG, "eps must be > 0");
  if (!isfinite(d->scale) || !isfinite(d->residual_scale)) return fail(DDG_ERR_INVALID_ARG, "scale and residual_scale must be finite");
  if (d->group != 0 && (d->group < 8 || d->group > 512 || (d->group & (d->group - 1)) || d->cols % d->group))
    return fail(DDG_ERR_SHAPE, "gated join: group = %d must be 0, or a power of two from 8 to 512 that divides %d columns", d->group, d->cols);
  if (d->gate < GATE_NONE || d->gate > GATE_SILU) return fail(DDG_ERR_INVALID_ARG, "gate must be one of DDG_GATE_*");
  CHECK(check_ld("ld_y", &d->ld_y, d->cols));
  CHECK(check_ld("ld_gate", &d->ld_gate, d->cols));
  CHECK(check_ld("ld_residual", &d->ld_residual, d->cols));
  CHECK(check_ld("ld_x", &d->ld_x, d->cols));
  CHECK(check_ld("ld_out", &d->ld_out, d->cols));
  *a = GatedArgs{};
  a->ld_y = d->ld_y; a->ld_gate = d->ld_gate; a->ld_residual = d->ld_residual; a->ld_x = d->ld_x; a->ld_out = d->ld_out;
  a->rows = d->rows; a->cols = d->cols; a->dtype = d->dtype; a->group = d->group; a->mode = d->gate;
  a->eps = d->eps; a->scale = d->scale; a->residual_scale = d->residual_scale;
  return DDG_OK;
}
// The gate as an argument: a row of fp32, a tensor, or nothing
Arg gate_arg(const char* name, const ddg_gated_join_desc& d, const void* p, bool out) {
  if (d.gate == GATE_COLUMN) return Arg{name, p, 1, d.cols, d.cols, 4, out};
  return Arg{name, d.gate == GATE_NONE ? nullptr : p, d.rows, d.cols, d.ld_gate, dtype_size(d.dtype), out};
}

// Rows of a launch of one workgroup of 256 threads each, and workgroups of any: fewer than 2^32 threads
constexpr int LINEAR_ROWS_MAX = 1 << 23;
constexpr long GROUPS_MAX = (1l << 24) - 16;

ddg_status linear_desc(const ddg_linear_desc* in, ddg_linear_desc* d) {
  if (!in) return fail(DDG_ERR_INVALID_ARG, "desc is null");
  *d = *in;
  CHECK(check_rows("linear attention", d->rows, d->heads, d->dtype));
  if (d->rows > LINEAR_ROWS_MAX) return fail(DDG_ERR_SHAPE, "linear attention: at most %d rows (%d)", LINEAR_ROWS_MAX, d->rows);
  if (d->kv_heads == 0) d->kv_heads = d->heads;
  if (d->kv_heads < 1 || d->heads % d->kv_heads) return fail(DDG_ERR_SHAPE, "linear attention: %d heads cannot share the keys of %d", d->heads, d->kv_heads);
  if (d->dim_k < 1 || d->dim_v < 1 || d->dim_k > LINEAR_DIM_MAX || d->dim_v > LINEAR_DIM_MAX)
    return fail(DDG_ERR_SHAPE, "linear attention: keys and values have 1 to %d columns (%d, %d)", LINEAR_DIM_MAX, d->dim_k, d->dim_v);
  if ((long)d->heads * LINEAR_DIM_MAX > LD_MAX) return fail(DDG_ERR_SHAPE, "linear attention: too many heads (%d)", d->heads);
  if (d->sequences < 1) return fail(DDG_ERR_SHAPE, "linear attention: need sequences >= 1 (%d)", d->sequences);
  if (d->slots == 0) d->slots = d->sequences;
  if (d->slots < 1) return fail(DDG_ERR_SHAPE, "linear attention: need slots >= 0 (%d)", d->slots);
  CHECK(check_ld("ld_q", &d->ld_q, d->heads * d->dim_k));
  CHECK(check_ld("ld_k", &d->ld_k, d->kv_heads * d->dim_k));
  CHECK(check_ld("ld_v", &d->ld_v, d->kv_heads * d->dim_v));
  CHECK(check_ld("ld_o", &d->ld_o, d->heads * d->dim_v));
  if (!isfinite(d->scale)) return fail(DDG_ERR_INVALID_ARG, "scale must be finite");
  return DDG_OK;
}

long slices_of(int cols) { return (cols + 63) / 64; }

// The cut into segments of a call, and the bytes of the states between them. Sequence n of a ragged call begins with piece start / segment + n; where that may lead past twice the rows, with
// piece 2 start / segment instead: a sequence of several segments has more than one segment's rows, so at least as many numbers as segments, and the others need none.
struct Cut { int segment; long segments; size_t pieces; bool by_rows; };
Cut cut_of(const ddg_linear_desc& d, bool backward, bool ragged) {
  const long k = slices_of(d.dim_k), v = slices_of(d.dim_v), walks = d.heads * (backward ? 2 * k + v : v);
  Cut c;
  c.segment = linear_segment(d.rows, d.sequences, (int)(walks < (1 << 30) ? walks : 1 << 30), ragged, d.dtype);
  c.segments = !c.segment ? d.sequences : ragged ? d.rows / c.segment + (long)d.sequences : (long)d.sequences * ((d.rows / d.sequences + c.segment - 1) / c.segment);
  const long most = c.segment && ragged ? 2l * d.rows / c.segment : c.segments;
  c.by_rows = most < c.segments;
  c.pieces = c.segment ? (size_t)(c.by_rows ? most : c.segments) * d.heads * d.dim_k * d.dim_v * 4 : 0;
  c.pieces = (c.pieces + 255) / 256 * 256;
  return c;
}
size_t shared_bytes(const ddg_linear_desc& d, int dim) { return d.heads == d.kv_heads ? 0 : ((size_t)d.rows * d.heads * dim * 4 + 255) / 256 * 256; }
size_t linear_bytes(const ddg_linear_desc& d, bool backward, bool ragged) {
  const Cut c = cut_of(d, backward, ragged);
  return backward ? 3 * c.pieces + shared_bytes(d, d.dim_k) + shared_bytes(d, d.dim_v) : c.pieces;
}

ddg_status check_grid(const ddg_linear_desc& d, const Cut& c) {
  const long wide = slices_of(d.dim_k > d.dim_v ? d.dim_k : d.dim_v), blocks = ((long)d.dim_k * d.dim_v + 255) / 256;
  if ((double)c.segments * d.heads * wide > (double)GROUPS_MAX || (c.segment && (double)blocks * d.sequences * d.heads > (double)GROUPS_MAX))
    return fail(DDG_ERR_SHAPE, "linear attention: %d sequences of %d heads are more than a launch holds", d.sequences, d.heads);
  return DDG_OK;
}

LinearArgs linear_args(const ddg_linear_desc& d, const Cut& c, const float* log_decay, const int32_t* starts, const int32_t* slots) {
  LinearArgs a{};
  a.log_decay = log_decay; a.starts = starts; a.slots = slots;
  a.rows = d.rows; a.sequences = d.sequences; a.heads = d.heads; a.pool = d.slots; a.dtype = d.dtype;
  a.segment = c.segment ? c.segment : 1; a.segments = (int)c.segments; a.split = c.segment != 0; a.by_rows = c.by_rows;
  return a;
}

ddg_status check_sequences(const ddg_linear_desc& d, const int32_t* starts, const int32_t* slots, bool states) {
  if (!starts && d.rows % d.sequences) return fail(DDG_ERR_SHAPE, "linear attention: %d rows are not %d equal sequences, and starts is null", d.rows, d.sequences);
  if (states && !slots && d.slots < d.sequences) return fail(DDG_ERR_SHAPE, "linear attention: %d states for %d sequences, and slots is null", d.slots, d.sequences);
  return DDG_OK;
}

}  // namespace

extern "C" {

ddg_status ddg_rotary_table(const ddg_rotary_desc* desc, uint64_t* host_table) {
  ddg_rotary_desc d;
  CHECK(rotary_desc(desc, &d));
  if (!host_table) return fail(DDG_ERR_INVALID_ARG, "host_table must not be null");
  const long double turn = 2.0L * 3.14159265358979323846264338L;        // 64 bits of fraction throughout: a step of the table is what is lost
  for (int i = 0; i < d.rot / 2; ++i) {
    const long double theta = powl((long double)d.base, -2.0L * i / d.rot);
    long double keep = 0.0L;
    if (d.context > 0.0) {
      keep = (d.context * theta / turn - d.low) / ((long double)d.high - d.low);
      keep = keep < 0.0L ? 0.0L : keep > 1.0L ? 1.0L : keep;
    }
    host_table[i] = (uint64_t)rintl(theta * (keep + (1.0L - keep) / d.factor) / turn * 0x1p64L);     // (less than 0.16 turns)
  }
  return DDG_OK;
}

ddg_status ddg_rotary(const ddg_rotary_desc* desc, const void* x, const int32_t* positions, long first, const uint64_t* table, int inverse, void* y) {
  ddg_rotary_desc d;
  CHECK(rotary_desc(desc, &d));
  if (d.rows && (!x || !y || !table)) return fail(DDG_ERR_INVALID_ARG, "x, y and table must not be null");
  if (first > ROTARY_FIRST_MAX || first < -ROTARY_FIRST_MAX) return fail(DDG_ERR_INVALID_ARG, "first = %ld must be within %ld of 0", first, ROTARY_FIRST_MAX);
  const size_t size = dtype_size(d.dtype);
  const Arg args[] = {{"y", y, d.rows, d.heads * d.dim, d.ld_y, size, true},
                      {"x", x, d.rows, d.heads * d.dim, d.ld_x, size, false},
                      {"positions", positions, d.rows, 1, 1, 4, false},
                      {"table", table, 1, d.rot / 2, d.rot / 2, 8, false}};
  const Pair same[] = {{"y", "x"}};
  CHECK(check_args(args, same));
  if (d.rows == 0 || d.dry_run) return DDG_OK;
  RotaryArgs a{};
  a.x = x; a.y = y; a.positions = positions; a.table = table; a.ld_x = d.ld_x; a.ld_y = d.ld_y; a.first = first;
  a.rows = d.rows; a.heads = d.heads; a.dim = d.dim; a.rot = d.rot; a.dtype = d.dtype;
  a.interleaved = d.interleaved != 0; a.inverse = inverse != 0; a.magnitude = d.magnitude;
  return done(rotary_launch(a, (hipStream_t)d.stream), "rotary");
}

ddg_status ddg_gated_join(const ddg_gated_join_desc* desc, const void* y, const void* gate, const void* residual, const float* gain_y, const float* gain_x,
                          void* x_out, void* out, float* rstd_y, float* rstd_x) {
  ddg_gated_join_desc d;
  GatedArgs a;
  CHECK(gated_desc(desc, &d, &a));
  if (d.rows && (!y || (d.gate != GATE_NONE && !gate))) return fail(DDG_ERR_INVALID_ARG, "y and gate must not be null");
  if (!x_out && !out && !rstd_y && !rstd_x) return fail(DDG_ERR_INVALID_ARG, "nothing to compute: every result is null");
  const size_t size = dtype_size(d.dtype);
  const int parts = d.group ? d.cols / d.group : 1;
  const Arg args[] = {{"x_out", x_out, d.rows, d.cols, d.ld_x, size, true},
                      {"out", out, d.rows, d.cols, d.ld_out, size, true},
                      {"rstd_y", rstd_y, d.rows, parts, parts, 4, true},
                      {"rstd_x", rstd_x, d.rows, 1, 1, 4, true},
                      {"y", y, d.rows, d.cols, d.ld_y, size, false},
                      gate_arg("gate", d, gate, false),
                      {"residual", residual, d.rows, d.cols, d.ld_residual, size, false},
                      {"gain_y", gain_y, 1, d.cols, d.cols, 4, false},
                      {"gain_x", gain_x, 1, d.cols, d.cols, 4, false}};
  const Pair same[] = {{"x_out", "y"}, {"x_out", "residual"}};
  CHECK(check_args(args, same));
  if (d.rows == 0 || d.dry_run) return DDG_OK;
  a.y = y; a.gate = gate; a.residual = residual; a.gain_y = gain_y; a.gain_x = gain_x; a.x = x_out; a.out = out; a.rstd_y = rstd_y; a.rstd_x = rstd_x;
  return done(gated_forward_launch(a, (hipStream_t)d.stream), "gated join");
}

size_t ddg_gated_join_workspace(const ddg_gated_join_desc* desc) {
  ddg_gated_join_desc d;
  GatedArgs a;
  return gated_desc(desc, &d, &a) == DDG_OK ? (size_t)gated_groups(d.rows, d.cols) * ((d.cols + 7) / 8 * 8) * 4 * (d.gate == GATE_COLUMN ? 3 : 2) : 0;
}

ddg_status ddg_gated_join_backward(const ddg_gated_join_desc* desc, const void* y, const float* rstd_y, const void* gate, const void* x, const float* rstd_x,
                                   const float* gain_y, const float* gain_x, const void* d_out, const void* d_x, void* d_residual, void* d_y, void* d_gate,
                                   float* d_gain_y, float* d_gain_x, void* workspace, size_t workspace_bytes) {
  ddg_gated_join_desc d;
  GatedArgs a;
  CHECK(gated_desc(desc, &d, &a));
  if (d.rows && (!y || !rstd_y || (d.gate != GATE_NONE && !gate))) return fail(DDG_ERR_INVALID_ARG, "y, rstd_y and gate must not be null");
  if (d.rows && d_out && (!x || !rstd_x)) return fail(DDG_ERR_INVALID_ARG, "x and rstd_x must not be null where d_out is not");
  if (d.rows && !d_out && !d_x) return fail(DDG_ERR_INVALID_ARG, "d_out and d_x are both null");
  if (d.gate == GATE_NONE && d_gate) return fail(DDG_ERR_INVALID_ARG, "d_gate: there is no gate");
  if (!d_residual && !d_y && !d_gate && !d_gain_y && !d_gain_x) return fail(DDG_ERR_INVALID_ARG, "nothing to compute: every gradient is null");
  const size_t size = dtype_size(d.dtype);
  const bool sums = d_gain_y || d_gain_x || (d_gate && d.gate == GATE_COLUMN);
  const size_t need = sums ? ddg_gated_join_workspace(desc) : 0;
  if (need && (!workspace || workspace_bytes < need))
    return fail(DDG_ERR_INVALID_ARG, "sums over rows need a workspace of %zu bytes (%zu)", need, workspace ? workspace_bytes : (size_t)0);
  if (need && (uintptr_t)workspace % 16) return fail(DDG_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
  const int parts = d.group ? d.cols / d.group : 1;
  const Arg args[] = {{"d_residual", d_residual, d.rows, d.cols, d.ld_residual, size, true},
                      {"d_y", d_y, d.rows, d.cols, d.ld_y, size, true},
                      gate_arg("d_gate", d, d_gate, true),
                      {"d_gain_y", d_gain_y, 1, d.cols, d.cols, 4, true},
                      {"d_gain_x", d_gain_x, 1, d.cols, d.cols, 4, true},
                      {"workspace", need ? workspace : nullptr, 1, (long)need, (long)need, 1, true},
                      {"y", y, d.rows, d.cols, d.ld_y, size, false},
                      {"rstd_y", rstd_y, d.rows, parts, parts, 4, false},
                      gate_arg("gate", d, gate, false),
                      {"x", x, d.rows, d.cols, d.ld_x, size, false},
                      {"rstd_x", rstd_x, d.rows, 1, 1, 4, false},
                      {"gain_y", gain_y, 1, d.cols, d.cols, 4, false},
                      {"gain_x", gain_x, 1, d.cols, d.cols, 4, false},
                      {"d_out", d_out, d.rows, d.cols, d.ld_out, size, false},
                      {"d_x", d_x, d.rows, d.cols, d.ld_x, size, false}};
  const Pair same[] = {{"d_residual", "d_x"}};
  CHECK(check_args(args, same));
  if (d.dry_run || (d.rows == 0 && !sums)) return DDG_OK;
  a.y = y; a.gate = gate; a.gain_y = gain_y; a.gain_x = gain_x; a.x = const_cast<void*>(x); a.rstd_y = const_cast<float*>(rstd_y);
  a.rstd_x = const_cast<float*>(rstd_x); a.d_out = d_out; a.d_x = d_x; a.d_residual = d_residual; a.d_y = d_y; a.d_gate = d_gate; a.d_gain_y = d_gain_y;
  a.d_gain_x = d_gain_x; a.partial = (float*)workspace;
  return done(gated_backward_launch(a, (hipStream_t)d.stream), "gated join backward");
}

size_t ddg_linear_attention_workspace(const ddg_linear_desc* desc, int backward) {
  ddg_linear_desc d;
  if (linear_desc(desc, &d) != DDG_OK) return 0;
  const size_t even = d.rows % d.sequences ? 0 : linear_bytes(d, backward != 0, false), ragged = linear_bytes(d, backward != 0, true);
  return even > ragged ? even : ragged;
}

ddg_status ddg_linear_attention(const ddg_linear_desc* desc, const void* q, const void* k, const void* v, const float* log_decay, const int32_t* starts,
                                const int32_t* slots, const float* state_in, void* o, float* state_out, void* workspace, size_t workspace_bytes) {
  ddg_linear_desc d;
  CHECK(linear_desc(desc, &d));
  if (!log_decay || (d.rows && (!q || !k || !v || !o))) return fail(DDG_ERR_INVALID_ARG, "q, k, v, log_decay and o must not be null");
  CHECK(check_sequences(d, starts, slots, state_in || state_out));
  const Cut c = cut_of(d, false, starts != nullptr);
  CHECK(check_grid(d, c));
  if (c.pieces && (!workspace || workspace_bytes < c.pieces))
    return fail(DDG_ERR_INVALID_ARG, "needs a workspace of %zu bytes (%zu)", c.pieces, workspace ? workspace_bytes : (size_t)0);
  if (c.pieces && (uintptr_t)workspace % 256) return fail(DDG_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
  const size_t size = dtype_size(d.dtype);
  const long cells = (long)d.heads * d.dim_k * d.dim_v;
  const Arg args[] = {{"o", o, d.rows, d.heads * d.dim_v, d.ld_o, size, true},
                      {"state_out", state_out, d.slots, cells, cells, 4, true},
                      {"workspace", c.pieces ? workspace : nullptr, 1, (long)c.pieces, (long)c.pieces, 1, true},
                      {"q", q, d.rows, d.heads * d.dim_k, d.ld_q, size, false},
                      {"k", k, d.rows, d.kv_heads * d.dim_k, d.ld_k, size, false},
                      {"v", v, d.rows, d.kv_heads * d.dim_v, d.ld_v, size, false},
                      {"log_decay", log_decay, d.heads, 1, 1, 4, false},
                      {"starts", starts, (long)d.sequences + 1, 1, 1, 4, false},
                      {"slots", slots, d.sequences, 1, 1, 4, false},
                      {"state_in", state_in, d.slots, cells, cells, 4, false}};
  const Pair same[] = {{"state_out", "state_in"}};
  CHECK(check_args(args, same));
  if (d.dry_run || (d.rows == 0 && !state_out)) return DDG_OK;
  LinearArgs a = linear_args(d, c, log_decay, starts, slots);
  LinearJob& j = a.job[0];
  const int share = d.heads / d.kv_heads;
  j.x = q; j.a = k; j.b = v; j.out = o; j.ld_x = d.ld_q; j.ld_a = d.ld_k; j.ld_b = d.ld_v; j.ld_out = d.ld_o;
  j.share_x = 1; j.share_a = share; j.share_b = share; j.K = d.dim_k; j.V = d.dim_v; j.slices = (int)slices_of(d.dim_v);
  j.inter = d.scale; j.intra = d.scale; j.update = 1.f; j.state_in = state_in; j.state_out = state_out; j.at_k = d.dim_v; j.at_v = 1;
  j.pieces = (float*)workspace;
  return done(linear_launch(a, 1, (hipStream_t)d.stream), "linear attention");
}

ddg_status ddg_linear_attention_backward(const ddg_linear_desc* desc, const void* q, const void* k, const void* v, const float* log_decay, const int32_t* starts,
                                         const int32_t* slots, const float* state_in, const void* d_o, const float* d_state_out, void* dq, void* dk, void* dv,
                                         float* d_state_in, void* workspace, size_t workspace_bytes) {
  ddg_linear_desc d;
  CHECK(linear_desc(desc, &d));
  if (!log_decay || (d.rows && (!q || !k || !v || !d_o))) return fail(DDG_ERR_INVALID_ARG, "q, k, v, log_decay and d_o must not be null");
  if (!dq && !dk && !dv && !d_state_in) return fail(DDG_ERR_INVALID_ARG, "nothing to compute: every gradient is null");
  CHECK(check_sequences(d, starts, slots, state_in || d_state_out || d_state_in));
  const Cut c = cut_of(d, true, starts != nullptr);
  CHECK(check_grid(d, c));
  const size_t need = linear_bytes(d, true, starts != nullptr);
  if (need && (!workspace || workspace_bytes < need))
    return fail(DDG_ERR_INVALID_ARG, "needs a workspace of %zu bytes (%zu)", need, workspace ? workspace_bytes : (size_t)0);
  if (need && (uintptr_t)workspace % 256) return fail(DDG_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
  const size_t size = dtype_size(d.dtype);
  const long cells = (long)d.heads * d.dim_k * d.dim_v;
  const Arg args[] = {{"dq", dq, d.rows, d.heads * d.dim_k, d.ld_q, size, true},
                      {"dk", dk, d.rows, d.kv_heads * d.dim_k, d.ld_k, size, true},
                      {"dv", dv, d.rows, d.kv_heads * d.dim_v, d.ld_v, size, true},
                      {"d_state_in", d_state_in, d.slots, cells, cells, 4, true},
                      {"workspace", need ? workspace : nullptr, 1, (long)need, (long)need, 1, true},
                      {"q", q, d.rows, d.heads * d.dim_k, d.ld_q, size, false},
                      {"k", k, d.rows, d.kv_heads * d.dim_k, d.ld_k, size, false},
                      {"v", v, d.rows, d.kv_heads * d.dim_v, d.ld_v, size, false},
                      {"d_o", d_o, d.rows, d.heads * d.dim_v, d.ld_o, size, false},
                      {"log_decay", log_decay, d.heads, 1, 1, 4, false},
                      {"starts", starts, (long)d.sequences + 1, 1, 1, 4, false},
                      {"slots", slots, d.sequences, 1, 1, 4, false},
                      {"state_in", state_in, d.slots, cells, cells, 4, false},
                      {"d_state_out", d_state_out, d.slots, cells, cells, 4, false}};
  CHECK(check_args(args, NONE));
  if (d.dry_run || (d.rows == 0 && !d_state_in)) return DDG_OK;
  LinearArgs a = linear_args(d, c, log_decay, starts, slots);
  const int share = d.heads / d.kv_heads;
  unsigned char* ws = (unsigned char*)workspace;
  float* const dk_heads = (float*)(ws + 3 * c.pieces);
  float* const dv_heads = (float*)(ws + 3 * c.pieces + shared_bytes(d, d.dim_k));
  int jobs = 0;
  auto next = [&]() -> LinearJob& {
    LinearJob& j = a.job[jobs];
    j.pieces = (float*)(ws + jobs * c.pieces);
    ++jobs;
    return j;
  };
  if (dq) {                                                // dq_t = scale S_t do_t: the forward walk with keys and values in each other's place
    LinearJob& j = next();
    j.x = d_o; j.a = v; j.b = k; j.out = dq; j.ld_x = d.ld_o; j.ld_a = d.ld_v; j.ld_b = d.ld_k; j.ld_out = d.ld_q;
    j.share_x = 1; j.share_a = share; j.share_b = share; j.K = d.dim_v; j.V = d.dim_k;
    j.inter = d.scale; j.intra = d.scale; j.update = 1.f; j.state_in = state_in; j.at_k = 1; j.at_v = d.dim_v;
  }
  if (dk) {                                                // dk_t = R_t v_t, from the end
    LinearJob& j = next();
    j.x = v; j.a = d_o; j.b = q; j.out = share > 1 ? dk_heads : dk; j.ld_x = d.ld_v; j.ld_a = d.ld_o; j.ld_b = d.ld_q;
    j.ld_out = share > 1 ? (long)d.heads * d.dim_k : d.ld_k; j.out_f32 = share > 1;
    j.share_x = share; j.share_a = 1; j.share_b = 1; j.K = d.dim_v; j.V = d.dim_k; j.back = true; j.late = true;
    j.inter = 1.f; j.intra = d.scale; j.update = d.scale; j.state_in = d_state_out; j.at_k = 1; j.at_v = d.dim_v;
  }
  if (dv || d_state_in) {                                  // dv_t = R_t^T k_t, from the end; R before the first row is the gradient of the state there
    LinearJob& j = next();
    j.x = k; j.a = q; j.b = d_o; j.out = share > 1 && dv ? dv_heads : dv; j.ld_x = d.ld_k; j.ld_a = d.ld_q; j.ld_b = d.ld_o;
    j.ld_out = share > 1 ? (long)d.heads * d.dim_v : d.ld_v; j.out_f32 = share > 1;
    j.share_x = share; j.share_a = 1; j.share_b = 1; j.K = d.dim_k; j.V = d.dim_v; j.back = true; j.late = true;
    j.inter = 1.f; j.intra = d.scale; j.update = d.scale; j.state_in = d_state_out; j.state_out = d_state_in; j.at_k = d.dim_v; j.at_v = 1;
  }
  for (int i = 0; i < jobs; ++i) a.job[i].slices = (int)slices_of(a.job[i].V);
  const hipStream_t s = (hipStream_t)d.stream;
  hipError_t e = linear_launch(a, jobs, s);
  if (e == hipSuccess && share > 1 && d.rows && (dk || dv)) {
    LinearShareArgs sum{};
    sum.starts = starts; sum.sequences = d.sequences; sum.rows = d.rows; sum.groups = d.kv_heads; sum.share = share; sum.dtype = d.dtype;
    int count = 0;
    if (dk) sum.of[count++] = {dk_heads, dk, d.ld_k, d.dim_k};
    if (dv) sum.of[count++] = {dv_heads, dv, d.ld_v, d.dim_v};
    e = linear_share_launch(sum, count, s);
  }
  return done(e, "linear attention backward");
}

ddg_status ddg_linear_attention_step(const ddg_linear_desc* desc, const void* q, const void* k, const void* v, const float* log_decay, const int32_t* slots,
                                     const float* state_in, void* o, float* state_out) {
  if (!desc) return fail(DDG_ERR_INVALID_ARG, "desc is null");
  ddg_linear_desc d = *desc;
  if (d.rows >= 0) d.sequences = d.rows ? d.rows : 1;
  CHECK(linear_desc(&d, &d));
  if (!log_decay || (d.rows && (!q || !k || !v || !o))) return fail(DDG_ERR_INVALID_ARG, "q, k, v, log_decay and o must not be null");
  if (d.rows) CHECK(check_sequences(d, nullptr, slots, state_in || state_out));
  if ((double)d.rows * d.heads > (double)GROUPS_MAX)
    return fail(DDG_ERR_SHAPE, "linear attention: %d rows of %d heads are more than a launch holds", d.rows, d.heads);
  const size_t size = dtype_size(d.dtype);
  const long cells = (long)d.heads * d.dim_k * d.dim_v;
  const Arg args[] = {{"o", o, d.rows, d.heads * d.dim_v, d.ld_o, size, true},
                      {"state_out", state_out, d.slots, cells, cells, 4, true},
                      {"q", q, d.rows, d.heads * d.dim_k, d.ld_q, size, false},
                      {"k", k, d.rows, d.kv_heads * d.dim_k, d.ld_k, size, false},
                      {"v", v, d.rows, d.kv_heads * d.dim_v, d.ld_v, size, false},
                      {"log_decay", log_decay, d.heads, 1, 1, 4, false},
                      {"slots", slots, d.rows, 1, 1, 4, false},
                      {"state_in", state_in, d.slots, cells, cells, 4, false}};
  const Pair same[] = {{"state_out", "state_in"}};
  CHECK(check_args(args, same));
  if (d.dry_run || d.rows == 0) return DDG_OK;
  const LinearStepArgs a{q, k, v, o, log_decay, slots, state_in, state_out, d.ld_q, d.ld_k, d.ld_v, d.ld_o,
                         d.rows, d.heads, d.heads / d.kv_heads, d.dim_k, d.dim_v, d.slots, d.dtype, d.scale, false};
  return done(linear_step_launch(a, (hipStream_t)d.stream), "linear attention step");
}

}  // extern "C"
