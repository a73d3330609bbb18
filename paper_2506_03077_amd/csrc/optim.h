// Launchers of the optimizer step: only enqueue work on `st`; arguments are checked by the callers in optim_api.hip.
#pragma once
#include "common.h"

namespace sbp {

constexpr int ADAMW_BLOCK = 256;                            // elements that share the scale of an 8-bit state
constexpr int ADAMW_TABLE = 40, NORM_TABLE = 128;           // tensors of a launch: what its arguments hold (less than 4 KB)
// Elements of a workgroup: one pass, without a loop.  In a loop of passes the loads of one wait for the instructions of the one before: this / a loop over 8192 / over 32768, 545 M weights
// with 8-bit states 938 / 1038 / 1084 us, 238 M of them in 111 tensors 515 / 563 / 611, 233 M with fp32 states 1338 / 1330 / 1388.
constexpr int64_t ADAMW_SPAN = 2048;
constexpr int64_t ADAMW_MOST = (int64_t)1 << 34;            // ... of a launch: its threads are counted in 32 bits
constexpr int NORM_WORKGROUPS = 2048;                       // ... of a norm: that many workgroups, and one more per tensor
constexpr int64_t NORM_SPAN = 8192;                         // ... of at least so many elements, and a multiple of it

// From this many elements on (of a call) gradients, weights and 8-bit states pass the caches by: what a call leaves there is not read before it has been replaced.  Norm, step and
// another reader of the weights one after the other, through the caches / past them: 8-bit states, bf16 weights and gradients, 20 M elements 128 / 137 us, 63 M 381 / 383, 210 M 1302 / 1255;
// 545 M in a step alone 945 / 900.  32-bit states go through the caches at any size: 210 M elements 2215 / 2268 us.
constexpr int64_t OPTIM_PAST = (int64_t)1 << 27;

struct AdamwTensor {
  int64_t n;
  double weight_decay;
  void* param; float* master; void* grad; void *m, *v; uint8_t *m_scale, *v_scale;
  uint32_t first_group;        // workgroups of the tensors before it
  uint32_t index;              // of the call's tensors
  float keep;                  // 1 - lr weight_decay, without `now`
  int32_t dtype, grad_dtype;
};
struct AdamwNow { double lr; int32_t step, pad; };
struct AdamwArgs {
  double lr;
  double log1, log2;           // of beta1 and beta2 (-infinity for 0)
  float beta1, rest1, beta2, rest2, root2, root_rest2, eps;      // 1 - beta1, 1 - beta2, the roots of beta2 and 1 - beta2
  float bias1, bias2;          // lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t), without `now`
  uint32_t seed;
  int32_t step;
  const float* grad_scale;
  const AdamwNow* now;
  int32_t eight, zero_grads;
  int32_t past;                // OPTIM_PAST elements or more (8-bit states)
};
// n <= ADAMW_TABLE tensors, ADAMW_MOST elements together, first_group filled in here; tensors of no elements are left out by the caller
hipError_t adamw_step(const AdamwArgs& a, const AdamwTensor* t, int n, hipStream_t st);

struct NormTensor { const void* grad; int64_t n; uint32_t first_group; int32_t dtype; };
// Sums of squares of n <= NORM_TABLE tensors, one fp64 for every `span` elements (a multiple of NORM_SPAN) of a tensor, into part[0 ..]; returns their
// number in n_parts
hipError_t norm_parts(const NormTensor* t, int n, int64_t span, bool past, double* part, int* n_parts, hipStream_t st);
// norm = sqrt(sum of part[0 .. n)), scale (or NULL) = min(1, max_norm / norm)
hipError_t norm_finish(const double* part, int n, float max_norm, float* norm, float* scale, hipStream_t st);

}  // namespace sbp
