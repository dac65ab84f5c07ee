// A step of drafted tokens: launch arguments of the rotation, tree, verification and row-moving kernels.
#pragma once

#include "kvc_serve.h"

namespace kvc {

// kvc_rotate (kvc_rotate.hip).
struct RotateRows {
  const char* in;
  char* out;
  int64_t in_token, in_head, out_token, out_head;  // bytes
};
struct RotateArgs {
  RotateRows rows[2];
  int32_t heads[2];
  int32_t num_rows, token0;   // tokens, and the first one of this launch
  int32_t pairs;              // rotated feature pairs
  int32_t copy;               // the features behind them are copied (they lie elsewhere in the result)
  double factor;
  double sign;                // -1: to -position
  const int32_t* positions;
  double turns[64][2];        // turns per position of each pair: rounded to 64 bits, and what that leaves
};
hipError_t launch_rotate(const RotateArgs& a, kvc_dtype dtype, int head_dim, int style, hipStream_t stream);

// kvc_tree (kvc_tree.hip).
struct TreeArgs {
  StepView step;
  const int32_t* parents;
  uint64_t* masks;
  int32_t words;
  int32_t* positions;
  int32_t seq0;  // first sequence of this launch
};
hipError_t launch_tree(TreeArgs a, hipStream_t stream);

// kvc_verify (kvc_verify.hip).
constexpr int kVerifyPiece = 2048;  // probabilities that a wave sums at a time
struct VerifyEnd {                  // where a sequence's walk ended
  double a;                         // what is left there: max(0, P - a Q)
  int32_t at;                       // the last accepted token's row, -1: the sequence is left out
  int32_t first, last;              // without draft probabilities: its children among these rows were rejected
  int32_t pad;
};
struct VerifyArgs {
  StepView step;
  const int32_t* parents;
  const int32_t* tokens;
  const float* target;
  const float* draft;
  int64_t target_stride, draft_stride;
  int32_t vocab, children, pieces;
  const float* uniforms;
  const float* last;
  int32_t* path;
  int32_t* counts;
  int32_t* chosen;
  VerifyEnd* ends;   // [num_seqs]
  double2* sums;     // [num_seqs][pieces]: what is left, and the whole
  int32_t seq0;
};
hipError_t launch_verify(VerifyArgs a, hipStream_t stream);

// kvc_keep (kvc_keep.hip).
struct KeepArgs {
  ServePool pv;
  StepView step;
  const int32_t* path;
  const int32_t* counts;
  int32_t num_layers;  // of this launch
  int32_t seq0;        // its first sequence
};
hipError_t launch_keep(const KeepArgs& a, const RowsLayers<kRowsLayers>& layers, kvc_dtype cache, int head_dim,
                       hipStream_t stream);

}  // namespace kvc
