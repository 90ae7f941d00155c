// Internal declarations of the gated-delta layer's kernels (matrix-state rule,
// short convolution) and of token scoring, shared with their C-ABI layer
// (layer_abi.cpp).  Not part of the public interface.
#pragma once

#include "precog_kernels.h"

namespace precog {

constexpr int kDeltaMaxK = 128;
constexpr int kDeltaMaxV = 256;
constexpr int kDeltaChainMax = 4;  // chain waves of a workgroup of the delta rule, 32 columns each
// Its prepare waves, one less than LDS has buffers: keys of up to 128 elements, or 64.
constexpr int delta_prepare_waves(bool in32, bool k128) { return in32 ? (k128 ? 1 : 3) : 4; }
constexpr float kDeltaErase = -256.f;  // log decays below it act as it: exp is 0 in fp32

// One gated-delta call.  Strides in elements; tokens of sequence b are
// [b * L, (b + 1) * L), or [starts[b], starts[b + 1]) clamped to [0, T].
struct DeltaParams {
  const void* q;
  const void* k;
  const void* v;
  const float* g;          // or null: 0
  const float* beta;       // or null: 1
  const int32_t* starts;   // or null
  const int32_t* idx;      // h0 rows of the sequences, or slots of a step; null: row b
  int64_t state_rows;      // rows of h0 that idx may name
  const void* h0;          // or null: zeros
  void* o;                 // or null: states only
  void* hT;                // or null; a step's states (h0 = hT)
  int64_t B, L, T;
  int64_t q_stride, k_stride, v_stride, h0_stride, hT_stride;
  int Hk, Hv, K, V;
  int norm;
  float eps, scale;
  int segments;            // of every sequence, 1: whole
  int phase;               // one of the following, set by launch_delta
  float* between;          // [B, segments, Hv, K, V] (workspace), segments > 1 only
  float* phi;              // [B, segments, Hv, K, K] (workspace)
};
constexpr int kWhole = 0, kSegmentEnds = 1, kSegments = 2;
hipError_t launch_delta(const DeltaParams& p, int in_dtype, int out_dtype, int state_dtype, int cus,
                        hipStream_t s);
hipError_t launch_delta_step(const DeltaParams& p, int in_dtype, int out_dtype, int state_dtype,
                             int cus, hipStream_t s);

struct ConvParams {
  const void* x;
  const float* w;          // [D, W]
  const float* bias;       // or null
  const int32_t* starts;   // or null
  const int32_t* idx;      // tail0 rows of the sequences, or slots of a step; null: row b
  int64_t tail_rows;
  const void* tail0;       // or null: zeros
  void* y;                 // or null: tails only
  void* tailT;             // or null; a step's tails (tail0 = tailT)
  int64_t B, L, T, D;
  int64_t x_stride;
  int W;
  int silu;
};
hipError_t launch_conv(const ConvParams& p, int in_dtype, int out_dtype, int cus, hipStream_t s);
hipError_t launch_conv_step(const ConvParams& p, int in_dtype, int out_dtype, hipStream_t s);

// Partial results of one workgroup's part of a row: maximum m, sum of
// exp(x - m), sum of exp(x - m) (x - m); then `top` candidates.
struct ScorePart {
  float m, s, t;
  int pad;
};
struct ScoreParams {
  const void* logits;
  const int32_t* token;    // or null
  float* logprob;
  float* entropy;          // or null
  int32_t* top_id;
  float* top_logprob;
  ScorePart* part;         // [T, splits] (workspace), splits > 1 only
  float* cand_val;         // [T, splits, top] (workspace)
  int32_t* cand_id;        // [T, splits, top] (workspace)
  int64_t T, V, row_stride;
  int top;
  int splits;              // workgroups of a row
  int64_t span;            // tokens of each of them
};
constexpr int kScoreMaxTop = 64;
constexpr int kScoreTile = 4 * 64 * 8;  // tokens that a workgroup takes at a time
hipError_t launch_score(const ScoreParams& p, int dtype, hipStream_t s);

}  // namespace precog
