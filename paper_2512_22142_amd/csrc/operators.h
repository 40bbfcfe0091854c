// Launch interface of the operators around the GEMMs: norms, bias gradient, log probabilities, AdamW.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "cleave.h"

namespace cleave {

// ---- root-mean-square norm ---------------------------------------------------

struct NormArgs {
  const void* x;
  const void* residual;    // null: h = x
  const float* weight;
  void* y;                 // x's type, or e4m3 with `scales`
  float* scales;           // null: y has x's type
  void* sum_out;           // h in x's type; may be null
  float* inv_rms;          // may be null
  int64_t rows, cols;
  int64_t ldx, ldr, ldy, lds;   // elements
  float eps;
};
hipError_t launch_rms_norm(const NormArgs& args, int dtype, hipStream_t stream);

// Rows of partial sums (each `cols` floats) that the gradient's first launch leaves for its second.
int rms_norm_partial_rows(int64_t rows, int64_t cols);
struct NormBackwardArgs {
  const void* dy;
  const void* h;
  const void* dsum;        // null: none
  const float* weight;
  const float* inv_rms;
  void* dx;
  float* partials;         // rms_norm_partial_rows x cols
  int64_t rows, cols;
  int64_t lddy, ldh, ldds, lddx;
};
// dx and the partial sums of the weight's gradient.
hipError_t launch_rms_norm_backward(const NormBackwardArgs& args, int dtype, int partial_rows, hipStream_t stream);

// ---- layer norm --------------------------------------------------------------

struct LayerNormArgs {
  const void* x;
  const void* residual;    // null: h = x
  const float* weight;
  const float* bias;       // may be null
  void* y;                 // x's type, or e4m3 with `scales`
  float* scales;           // null: y has x's type
  void* sum_out;           // h in x's type; may be null
  float* mean;             // may be null
  float* inv_std;          // may be null
  int64_t rows, cols;
  int64_t ldx, ldr, ldy, lds;   // elements
  float eps;
};
hipError_t launch_layer_norm(const LayerNormArgs& args, int dtype, hipStream_t stream);

// Rows of partial sums (the weight's, then the bias's, each in whole quads) that the gradient's first launch leaves for its second, at most.
int layer_norm_partial_rows(int64_t rows, int64_t cols);
struct LayerNormBackwardArgs {
  const void* dy;
  const void* h;
  const void* dsum;        // null: none
  const float* weight;
  const float* mean;
  const float* inv_std;
  void* dx;
  float* partials;         // layer_norm_partial_rows rows
  float* dweight;
  float* dbias;            // null: none
  int64_t rows, cols;
  int64_t lddy, ldh, ldds, lddx;
};
hipError_t launch_layer_norm_backward(const LayerNormBackwardArgs& args, int dtype, hipStream_t stream);

// ---- sums of columns ---------------------------------------------------------

// out[c] = sum over `rows` rows of in[., c], in a fixed order.
struct ColumnSumArgs {
  const void* in;
  int64_t ld;              // elements
  int64_t rows, cols;
  float* out;
  float* partials;         // chunks x cols where chunks > 1
  int chunks;
};
// Chunks of rows that are summed apart.
int column_sum_chunks(int64_t rows, int64_t cols);
// out[c] = sum of `n` contiguous rows of partial sums.
hipError_t launch_join_rows(const float* rows, int n, int64_t cols, float* out, hipStream_t stream);
hipError_t launch_column_sum(const ColumnSumArgs& args, int dtype, hipStream_t stream);

// ---- log probabilities of tokens ---------------------------------------------

constexpr int kMostTop = 32;      // most likely tokens of a row that are given
constexpr int kMostParts = 8;     // of a row
struct LogProbArgs {
  const void* logits;
  const int64_t* ids;      // null: no log probabilities
  float* logp;             // null, with ids
  float* lse;              // may be null
  float* entropy;          // may be null
  int64_t* top_ids;        // rows x n_top
  float* top_logp;
  float* workspace;        // parts > 1
  int64_t rows, cols, ld;
  float scale;
  int n_top, parts;
  int chunk;               // columns of a part
};
int log_probs_parts(int64_t rows, int64_t cols, int64_t n_top);
hipError_t launch_log_probs(const LogProbArgs& args, int dtype, hipStream_t stream);

struct LogProbBackwardArgs {
  const void* logits;
  const int64_t* ids;      // null, with dlogp
  const float* lse;
  const float* dlogp;
  const float* entropy;    // null, with dentropy
  const float* dentropy;
  void* dlogits;
  int64_t rows, cols, ld, ldd;
  float scale;
  int parts;               // workgroups of a row, and the |lse| that far rows begin at (filled in at the launch)
  float near;
};
hipError_t launch_log_probs_backward(const LogProbBackwardArgs& args, int dtype, hipStream_t stream);

// ---- AdamW over many tensors -------------------------------------------------

// Elements of an 8-bit state that share a scale.
constexpr int kStateBlock = 256;
// Elements that one workgroup updates.
constexpr int kAdamChunk = 4096;

struct AdamTensor {
  float* w;
  const void* g;
  void* m;                 // fp32, or e4m3 with scales
  void* v;                 // fp32, or the square root as e4m3 with scales
  float* m_scale;
  float* v_scale;
  uint16_t* copy;          // bf16; may be null
  uint64_t n;              // elements
};
static_assert(sizeof(AdamTensor) == 64, "AdamTensor is 64 bytes");
constexpr int kAdamTensors = 56;   // per launch
struct AdamWArgs {
  AdamTensor tensors[kAdamTensors];
  uint32_t chunk_end[kAdamTensors];   // chunks of the tensors up to and with this one
  int n_tensors;
  const float* grad_scale;            // device, may be null
  float lr, beta1, one_minus_beta1, beta2, one_minus_beta2, eps, weight_decay, inv_bias1, inv_bias2;
};
static_assert(sizeof(AdamWArgs) <= 4096, "kernel arguments stay within 4 KB");
hipError_t launch_adamw(const AdamWArgs& args, uint32_t chunks, int grad_dtype, bool states_8bit, hipStream_t stream);

}  // namespace cleave
