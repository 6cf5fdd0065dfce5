// What the operators between the joins of a token model (rotary positions, linear attention, the gated join) share between their checks
// (ddg_mixing.cpp) and their kernels: kernel arguments and launches. Every launch assumes what ddg_mixing.cpp has checked.
#pragma once
#include "ddg_kernels.h"

namespace ddg {

struct RotaryArgs {
  const void* x; void* y; const int* positions; const uint64_t* table;
  long ld_x, ld_y, first;
  int rows, heads, dim, rot, dtype;
  bool interleaved, inverse;
  float magnitude;
};
constexpr int ROTARY_DIM_MAX = 1024;
constexpr long ROTARY_FIRST_MAX = 1l << 48;    // four steps of the table make 2^-14 of a turn there, and sums with positions and rows stay inside 64 bits
hipError_t rotary_launch(const RotaryArgs& a, hipStream_t s);

enum Gate { GATE_NONE = 0, GATE_COLUMN = 1, GATE_PLAIN = 2, GATE_SIGMOID = 3, GATE_SILU = 4 };
struct GatedArgs {
  const void* y; const void* gate; const void* residual; const float* gain_y; const float* gain_x;   // gate: [rows][cols], or fp32 [cols] (GATE_COLUMN)
  void* x; void* out; float* rstd_y; float* rstd_x;             // forward: results; backward: x and both rstd are operands
  const void* d_out; const void* d_x;
  void* d_residual; void* d_y; void* d_gate; float* d_gain_y; float* d_gain_x; float* partial;   // partial: [3][gated_groups][cols in whole eights]
  long ld_y, ld_gate, ld_residual, ld_x, ld_out;
  int rows, cols, dtype, group, mode;
  float eps, scale, residual_scale;
  bool past;                                                   // results go past the caches (set by the launch)
};
constexpr int GATED_COLS_MAX = 8192;
int gated_groups(int rows, int cols);        // workgroups of the backward launch, each with rows of partial sums
hipError_t gated_forward_launch(const GatedArgs& a, hipStream_t s);
hipError_t gated_backward_launch(const GatedArgs& a, hipStream_t s);

// A walk over the rows of every sequence and head (from the last row on with `back`):
//   out_r = inter g^(r+1-late) x_r S + intra sum_{j<=r} g^(r-j) (x_r . a_j) b_j,   after n rows S' = g^n S + update sum_j g^(n-1-j+late) a_j b_j^T
struct LinearJob {
  const void* x; const void* a; const void* b; void* out;      // [rows][heads / share][K, K, V, V]
  long ld_x, ld_a, ld_b, ld_out;
  int share_x, share_a, share_b;                               // heads that share one of the operand's
  int K, V, slices;                                            // slices: pieces of 64 columns of V
  bool back, late, out_f32;
  float inter, intra, update;
  const float* state_in; float* state_out;                     // element (k, v) at k * at_k + v * at_v of a head's K * V
  long at_k, at_v;
  float* pieces;                                               // [pieces][heads][K][V]: states before each segment of a sequence that has several
};
struct LinearArgs {
  LinearJob job[3];
  const float* log_decay; const int* starts; const int* slots;
  int rows, sequences, heads, pool, segment, segments, dtype;  // segment: rows of one; segments: most there can be
  bool split, by_rows;                                         // sequences may have several segments; their pieces are numbered by rows alone
};
struct LinearStepArgs {
  const void* q; const void* k; const void* v; void* o; const float* log_decay; const int* slots; const float* state_in; float* state_out;
  long ld_q, ld_k, ld_v, ld_o;
  int rows, heads, share, K, V, pool, dtype;
  float scale;
  bool past;                                                   // states go past the caches (set by the launch)
};
constexpr int LINEAR_DIM_MAX = 256;
int linear_segment(int rows, int sequences, int walks, bool ragged, int dtype);   // rows of a segment; 0: sequences are not split
hipError_t linear_launch(const LinearArgs& a, int jobs, hipStream_t s);
hipError_t linear_step_launch(const LinearStepArgs& a, hipStream_t s);
// out [rows][groups][cols] = sums of `share` neighbouring heads of in [rows][groups * share][cols], fp32, in order; up to two of them
struct LinearShareArgs {
  struct One { const float* in; void* out; long ld; int cols; } of[2];
  const int* starts;
  int sequences, rows, groups, share, dtype;
};
hipError_t linear_share_launch(const LinearShareArgs& a, int count, hipStream_t s);

}  // namespace ddg
