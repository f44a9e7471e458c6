// Arguments of the kernels behind psa_qk_norm_rope and its gradient (not part of the public ABI).
#pragma once
#include "psa_common.cuh"

namespace psa {

constexpr int kNormRopeBwdBlocks = 444;   // most blocks a tensor in a gradient launch, each with a partial sum per weight

struct NormRopeArgs {
  double turns[64];                 // quarter turns per unit of position of every pair, axis after axis
  Divisor by_tokens, by_w, by_h;
  double origin[3], step[3];        // positions: origin + step * index
  int pairs[3];                     // pairs of the first axis, of the first two, of all three
  int H, W;
  long long n_video;                // tokens of the sequence that are rotated: T * H * W
  long long first_token;            // of the sequence
  int n_tokens, n_all, n_heads;     // tokens of a batch element, of all of them
  int parts, slots, stages;         // groups of a token and tensor; tokens of a block; sets of rows in shared memory
  int tensors;                      // 2: a block takes q and k, 1: one of them
  int weight_dtype, weight_head;    // weight_head: 1 if every head has weights of its own
  int weight_cols;                  // weights
  float eps, inv_count;             // inv_count: 1 / values of a mean
  const void* in[2];                // q and k (either may be missing)
  const void* grad[2];              // gradients of the outputs
  void* out[2];                     // outputs, or gradients of the inputs
  const void* weight[2];
  float* dw_part;                   // [tensors][blocks][weight_cols]
  long long in_batch, in_head, in_token, out_batch, out_head, out_token, dx_batch, dx_head, dx_token;   // strides, in elements
};

// Launches the forward pass or the gradient.  The arguments have been checked; parts, slots, stages and tensors are chosen here.
cudaError_t launch_norm_rope(NormRopeArgs& a, const psa_qk& prob, bool halves, bool backward, int n_sms, float* q_dw, float* k_dw, cudaStream_t st,
                             int* launches);

}  // namespace psa
