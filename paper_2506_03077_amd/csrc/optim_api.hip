// C ABI of the optimizer step: validation and the host loops over tables of tensors.  Nothing is allocated or synchronised; no
// device code, so that the tests can build it with a host compiler.
#include "../../include/streambp.h"
#include "optim.h"

#include <algorithm>
#include <cmath>

using namespace sbp;

namespace {

#define HIPCHK(expr)                                                                       \
  do {                                                                                     \
    hipError_t e__ = (expr);                                                               \
    if (e__ != hipSuccess)                                                                 \
      return fail(SBP_ERR_HIP, "%s failed: %s (%s:%d)", #expr, hipGetErrorString(e__), __FILE__, __LINE__); \
  } while (0)

static_assert(sizeof(AdamwNow) == sizeof(sbp_adamw_now), "the device's view of sbp_adamw_now");
static_assert(ADAMW_BLOCK == SBP_STATE_BLOCK, "the block of the public header");

constexpr int64_t MOST_ELEMENTS = (int64_t)1 << 44;

bool valid_dtype(int dt) { return dt == SBP_F32 || dt == SBP_BF16; }
bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

int64_t sum_of(int32_t n, const sbp_adamw_tensor* t) {
  int64_t s = 0;
  for (int i = 0; i < n; ++i) s += t[i].n;
  return s;
}

int32_t check_table(int32_t n, const sbp_adamw_tensor* t) {
  if (n < 0) return fail(SBP_ERR_SHAPE, "n_tensors must be >= 0");
  if (n > 0 && !t) return fail(SBP_ERR_NULL, "the table of tensors is NULL");
  int64_t total = 0;      // (more than any memory: the sums of workgroups below stay far from their types' ends)
  for (int i = 0; i < n; ++i) {
    if (t[i].n < 0 || t[i].n > ADAMW_MOST) return fail(SBP_ERR_SHAPE, "tensor %d: n = %lld is outside [0, 2^34]", i, (long long)t[i].n);
    if ((total += t[i].n) > MOST_ELEMENTS) return fail(SBP_ERR_SHAPE, "tensor %d: more than 2^44 elements together", i);
    if (t[i].n == 0) continue;
    if (!valid_dtype(t[i].grad_dtype)) return fail(SBP_ERR_UNSUPPORTED, "tensor %d: grad_dtype %d not supported", i, t[i].grad_dtype);
    if (!t[i].grad) return fail(SBP_ERR_NULL, "tensor %d: grad is NULL", i);
    if (!aligned(t[i].grad, dtype_size(t[i].grad_dtype))) return fail(SBP_ERR_UNSUPPORTED, "tensor %d: grad is not aligned to its elements", i);
  }
  return SBP_OK;
}

int32_t check_adamw(const sbp_adamw_cfg* c, int32_t n, const sbp_adamw_tensor* t, bool now) {
  if (!c) return fail(SBP_ERR_NULL, "cfg is NULL");
  if (c->state != SBP_STATE_F32 && c->state != SBP_STATE_8BIT) return fail(SBP_ERR_UNSUPPORTED, "state %d not supported", c->state);
  if (!now && c->step < 1) return fail(SBP_ERR_SHAPE, "step must be >= 1");
  if (!now && !(c->lr >= 0.0 && std::isfinite(c->lr))) return fail(SBP_ERR_SHAPE, "lr must be >= 0 and finite");
  if (!(c->beta1 >= 0.0 && c->beta1 < 1.0) || !(c->beta2 >= 0.0 && c->beta2 < 1.0)) return fail(SBP_ERR_SHAPE, "beta1 and beta2 must be in [0, 1)");
  if (!(c->eps >= 0.0 && std::isfinite(c->eps))) return fail(SBP_ERR_SHAPE, "eps must be >= 0 and finite");
  if (c->zero_grads != 0 && c->zero_grads != 1) return fail(SBP_ERR_SHAPE, "zero_grads must be 0 or 1");
  if (int32_t rc = check_table(n, t)) return rc;
  for (int i = 0; i < n; ++i) {
    const sbp_adamw_tensor& x = t[i];
    if (!(x.weight_decay >= 0.0 && std::isfinite(x.weight_decay))) return fail(SBP_ERR_SHAPE, "tensor %d: weight_decay must be >= 0 and finite", i);
    if (x.n == 0) continue;
    if (!valid_dtype(x.dtype)) return fail(SBP_ERR_UNSUPPORTED, "tensor %d: dtype %d not supported", i, x.dtype);
    if (x.master && x.dtype != SBP_BF16) return fail(SBP_ERR_UNSUPPORTED, "tensor %d: a master copy belongs to a bf16 param", i);
    const bool eight = c->state == SBP_STATE_8BIT;
    if (!x.param || !x.m || !x.v) return fail(SBP_ERR_NULL, "tensor %d: param, m and v must be non-NULL", i);
    if (eight && (!x.m_scale || !x.v_scale)) return fail(SBP_ERR_NULL, "tensor %d: 8-bit states need m_scale and v_scale", i);
    if (!eight && (x.m_scale || x.v_scale)) return fail(SBP_ERR_UNSUPPORTED, "tensor %d: fp32 states have no scales", i);
    if (!aligned(x.param, dtype_size(x.dtype)) || !aligned(x.master, 4) || (!eight && (!aligned(x.m, 4) || !aligned(x.v, 4))))
      return fail(SBP_ERR_UNSUPPORTED, "tensor %d: a pointer is not aligned to its elements", i);
  }
  return SBP_OK;
}

}  // namespace

extern "C" {

int32_t streambp_adamw_step(const sbp_adamw_cfg* c, int32_t n_tensors, const sbp_adamw_tensor* tensors, const float* grad_scale,
                            const sbp_adamw_now* now, void* hip_stream) {
  if (int32_t rc = check_adamw(c, n_tensors, tensors, now != nullptr)) return rc;
  if (!aligned(grad_scale, 4) || !aligned(now, 8)) return fail(SBP_ERR_UNSUPPORTED, "grad_scale or now is not aligned to its elements");
  AdamwArgs a{};
  a.lr = c->lr; a.eps = (float)c->eps;
  a.beta1 = (float)c->beta1; a.rest1 = (float)(1.0 - c->beta1);
  a.beta2 = (float)c->beta2; a.rest2 = (float)(1.0 - c->beta2); a.root2 = (float)std::sqrt(c->beta2); a.root_rest2 = (float)std::sqrt(1.0 - c->beta2);
  a.seed = c->seed; a.step = c->step; a.grad_scale = grad_scale; a.now = (const AdamwNow*)now;
  a.eight = c->state == SBP_STATE_8BIT; a.zero_grads = c->zero_grads;
  a.log1 = std::log(c->beta1); a.log2 = std::log(c->beta2);
  if (!now) {
    // 1 - b^t by expm1, exact for b next to 1 too; b = 0: 1 + expm1(-infinity) of no effect
    a.bias1 = (float)(c->lr / -std::expm1(c->step * a.log1));
    a.bias2 = (float)(1.0 / std::sqrt(-std::expm1(c->step * a.log2)));
  }
  a.past = a.eight && sum_of(n_tensors, tensors) >= OPTIM_PAST;
  AdamwTensor table[ADAMW_TABLE];
  int n = 0;
  int64_t elements = 0;
  auto flush = [&]() {
    const hipError_t e = n > 0 ? adamw_step(a, table, n, (hipStream_t)hip_stream) : hipSuccess;
    n = 0;
    elements = 0;
    return e;
  };
  for (int i = 0; i < n_tensors; ++i) {
    const sbp_adamw_tensor& x = tensors[i];
    if (x.n == 0) continue;
    if (n == ADAMW_TABLE || elements + x.n > ADAMW_MOST) HIPCHK(flush());
    table[n++] = AdamwTensor{x.n, x.weight_decay, x.param, x.master, x.grad, x.m, x.v, (uint8_t*)x.m_scale, (uint8_t*)x.v_scale, 0, (uint32_t)i, (float)(1.0 - c->lr * x.weight_decay), x.dtype, x.grad_dtype};
    elements += x.n;
  }
  HIPCHK(flush());
  return SBP_OK;
}

size_t streambp_grad_norm_workspace_bytes(int32_t n_tensors) {
  return n_tensors < 0 ? 0 : align_up(((size_t)NORM_WORKGROUPS + n_tensors) * sizeof(double), 256);
}

int32_t streambp_grad_norm(int32_t n_tensors, const sbp_adamw_tensor* tensors, float max_norm, float* norm, float* grad_scale, void* workspace,
                           size_t workspace_bytes, void* hip_stream) {
  if (int32_t rc = check_table(n_tensors, tensors)) return rc;
  if (!(max_norm >= 0.f) || !std::isfinite(max_norm)) return fail(SBP_ERR_SHAPE, "max_norm must be >= 0 and finite");
  if (!norm || !workspace) return fail(SBP_ERR_NULL, "norm and workspace must be non-NULL");
  if (!aligned(norm, 4) || !aligned(grad_scale, 4)) return fail(SBP_ERR_UNSUPPORTED, "norm or grad_scale is not aligned to its elements");
  if (!aligned(workspace, 256)) return fail(SBP_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  if (workspace_bytes < streambp_grad_norm_workspace_bytes(n_tensors)) return fail(SBP_ERR_WORKSPACE, "workspace too small");
  const int64_t total = sum_of(n_tensors, tensors);
  // (every tensor has at most one span that is not full: no more than NORM_WORKGROUPS + n_tensors of them)
  const int64_t span = std::max<int64_t>(NORM_SPAN, align_up((size_t)cdiv(total, NORM_WORKGROUPS), NORM_SPAN));
  NormTensor table[NORM_TABLE];
  int n = 0, parts = 0;
  for (int i = 0; i < n_tensors; ++i) {
    if (tensors[i].n > 0) table[n++] = NormTensor{tensors[i].grad, tensors[i].n, 0, tensors[i].grad_dtype};
    if (n == NORM_TABLE || (i == n_tensors - 1 && n > 0)) {
      int more = 0;
      HIPCHK(norm_parts(table, n, span, total >= OPTIM_PAST, (double*)workspace + parts, &more, (hipStream_t)hip_stream));
      parts += more;
      n = 0;
    }
  }
  HIPCHK(norm_finish((const double*)workspace, parts, max_norm, norm, grad_scale, (hipStream_t)hip_stream));
  return SBP_OK;
}

}  // extern "C"
