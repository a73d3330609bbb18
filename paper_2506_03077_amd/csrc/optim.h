// Launchers of the optimizer step: only enqueue work on `st`; arguments are checked by the callers in optim_api.hip.
#pragma once
#include "common.h"

namespace sbp {

constexpr int ADAMW_BLOCK = 256;                            // elements that share the scale of an 8-bit state
constexpr int ADAMW_TABLE = 40, NORM_TABLE = 128;           // tensors of a launch: what its arguments hold (less than 4 KB)
constexpr int64_t ADAMW_SPAN = 8192;                        // elements of a workgroup
constexpr int NORM_WORKGROUPS = 2048;                       // ... of a norm: that many workgroups, and one more per tensor
constexpr int64_t NORM_SPAN = 8192;                         // ... of at least so many elements

struct AdamwTensor {
  int64_t n;
  double weight_decay;
  void* param; float* master; void* grad; void *m, *v; uint8_t *m_scale, *v_scale;
  uint32_t first_group;        // workgroups of the tensors before it
  uint32_t index;              // of the call's tensors
  int32_t dtype, grad_dtype;
};
struct AdamwNow { double lr; int32_t step, pad; };
struct AdamwArgs {
  double lr, beta1, beta2, eps;
  float bias1, bias2;          // lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
  uint32_t seed;
  int32_t step;
  const float* grad_scale;
  const AdamwNow* now;
  int32_t eight, zero_grads;
};
// n <= ADAMW_TABLE tensors, first_group filled in here; tensors of no elements are left out by the caller
hipError_t adamw_step(const AdamwArgs& a, const AdamwTensor* t, int n, hipStream_t st);

struct NormTensor { const void* grad; int64_t n; uint32_t first_group; int32_t dtype; };
// Sums of squares of n <= NORM_TABLE tensors, one fp64 for every `span` elements (a multiple of 2048) of a tensor, into part[0 ..]; returns their
// number in n_parts
hipError_t norm_parts(const NormTensor* t, int n, int64_t span, double* part, int* n_parts, hipStream_t st);
// norm = sqrt(sum of part[0 .. n)), scale (or NULL) = min(1, max_norm / norm)
hipError_t norm_finish(const double* part, int n, float max_norm, float* norm, float* scale, hipStream_t st);

}  // namespace sbp
