// What the operators of token models share between their checks (ddg_token.cpp) and their kernels: kernel arguments and launches.
// Every launch assumes what ddg_token.cpp has checked.
#pragma once
#include "ddg_kernels.h"

namespace ddg {

// Dropout from a counter-based generator: `limit` of 65536 draws are dropped, the others multiplied by `scale`.
struct DropArgs { uint32_t limit; float scale; uint32_t key0, key1, step0, step1; };

struct DropoutArgs {
  const void* x; void* y;
  long ld_x, ld_y;
  int rows, cols, dtype;
  DropArgs drop;
};
hipError_t dropout_launch(const DropoutArgs& a, hipStream_t s);

struct JoinArgs {
  const void* y; const void* residual; const float* gain;    // forward: operands (residual, gain may be null)
  void* x; void* out; uint8_t* q; float* scale; float* rstd; // forward: results (out or q; x, rstd may be null)
  const void* d_out; const void* d_x;                        // backward: x, rstd, gain and these are operands (d_x may be null)
  void* d_residual; void* d_y; float* d_gain; float* partial;// backward: results (d_y, d_gain may be null); partial: [join_groups][cols]
  long ld_y, ld_residual, ld_x, ld_out;
  int rows, cols, dtype, group;
  float eps;
  DropArgs drop;
};
constexpr int JOIN_COLS_MAX = 32768;
int join_groups(int rows, int cols);         // workgroups of the backward launch, each with a row of partial sums
hipError_t join_forward_launch(const JoinArgs& a, hipStream_t s);
hipError_t join_backward_launch(const JoinArgs& a, hipStream_t s);

// Vocabulary loss. The plan holds what a call's sizes decide; offsets are bytes into the workspace.
struct VocabPlan {
  int tokens, dim, vocab, dtype;
  bool grads, dw_f32;
  bool pack_h, pack_w;       // operands whose rows are not 16-byte pieces are copied to ones that are
  bool planes;               // fp32 operands are taken apart into three bf16 planes each
  int dim_p;                 // width of the copies
  int panel, panels;         // tokens of a panel
  long ld_p;                 // elements between the rows of the panel's probabilities
  int cfg_z, cfg_dh, cfg_dw; // tiles of the three products
  int stat_cols, stats;      // columns that share a maximum and sum, and their number
  int splits, splits_dw;     // parts of the vocabulary that dh is summed over, of the tokens that dw is
  bool whole, pair;          // one tile holds the vocabulary and leaves P as it is read (not in planes); dh and dw are one launch
  bool acc;                  // dw is summed over panels in a buffer of the workspace
  size_t o_scalar, o_row, o_zt, o_stat, o_p, o_planes, o_part, o_part_dw, o_acc, o_h, o_w, bytes;
};
struct VocabArgs {
  const void* h; const void* w; const int32_t* target; const float* weight;
  float* loss; float* row_loss; float* lse; void* dh; void* dw; unsigned char* ws;
  long ld_h, ld_w, ld_dh, ld_dw;
};
void vocab_plan(VocabPlan* p);
hipError_t vocab_launch(const VocabPlan& p, const VocabArgs& a, hipStream_t s);

}  // namespace ddg
