// The host layer of the optimizer step (csrc/optim_api.hip) built with a host compiler: the launchers here write down what they are given, and the driver holds
// it against the call.  Every tensor has its workgroups once, under its own index; a launch takes no more than its table and its threads allow; the sums of
// the norm stay inside the workspace, which is allocated exactly.
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <random>
#include <string>
#include <vector>

#include "../../include/streambp.h"
#include "optim.h"

namespace sbp {

static std::vector<AdamwTensor> seen;
static std::vector<NormTensor> summed;
static int launches, parts_finished;
static AdamwArgs last;

int32_t fail(int32_t code, const char* fmt, ...) { (void)fmt; return code; }

static void expect(bool ok, const char* what) {
  if (!ok) { printf("FAILED: %s\n", what); exit(1); }
}

hipError_t adamw_step(const AdamwArgs& a, const AdamwTensor* t, int n, hipStream_t) {
  int64_t elements = 0;
  for (int i = 0; i < n; ++i) { elements += t[i].n; seen.push_back(t[i]); expect(t[i].n > 0, "an empty tensor was launched"); }
  expect(n >= 1 && n <= ADAMW_TABLE && elements <= ADAMW_MOST, "a launch of more than it takes");
  last = a;
  ++launches;
  return hipSuccess;
}
hipError_t norm_parts(const NormTensor* t, int n, int64_t span, bool, double* part, int* n_parts, hipStream_t) {
  expect(n >= 1 && n <= NORM_TABLE && span >= NORM_SPAN && span % NORM_SPAN == 0, "a table or span the kernel does not take");
  int64_t groups = 0;
  for (int i = 0; i < n; ++i) { groups += cdiv(t[i].n, span); summed.push_back(t[i]); }
  expect(groups * 256 < (int64_t)1 << 32, "more threads than a launch has");
  for (int64_t i = 0; i < groups; ++i) part[i] = 1.0;
  *n_parts = (int)groups;
  return hipSuccess;
}
hipError_t norm_finish(const double* part, int n, float, float* norm, float* scale, hipStream_t) {
  double s = 0.0;
  for (int i = 0; i < n; ++i) s += part[i];
  parts_finished = (int)s;
  *norm = 1.f;
  if (scale) *scale = 1.f;
  return hipSuccess;
}

}  // namespace sbp

using namespace sbp;

static void one(std::mt19937_64& rng, int n_tensors, int largest_log2) {
  std::vector<sbp_adamw_tensor> t(n_tensors);
  int64_t filled = 0;
  for (auto& x : t) {
    memset(&x, 0, sizeof x);
    x.n = rng() % 5 == 0 ? 0 : (int64_t)(rng() >> (63 - rng() % (largest_log2 + 1)));
    if (x.n > ((int64_t)1 << 34)) x.n = (int64_t)1 << 34;
    x.dtype = x.grad_dtype = SBP_F32;
    x.weight_decay = 0.01 * (double)(&x - t.data());
    x.param = x.grad = x.m = x.v = (void*)(uintptr_t)(4096 + 16 * (&x - t.data()));      // (never read)
    filled += x.n > 0;
  }
  seen.clear(); summed.clear(); launches = 0;
  sbp_adamw_cfg c{};
  c.state = SBP_STATE_F32; c.step = 3; c.lr = 1e-3; c.beta1 = 0.0; c.beta2 = 0.99; c.eps = 1e-8;
  expect(streambp_adamw_step(&c, n_tensors, t.data(), nullptr, nullptr, nullptr) == SBP_OK, "the step was refused");
  expect((int64_t)seen.size() == filled, "a tensor is missing or there twice");
  for (const auto& s : seen) expect(s.param == t[s.index].param && s.n == t[s.index].n && s.weight_decay == t[s.index].weight_decay, "a tensor has another's index");
  for (size_t i = 1; i < seen.size(); ++i) expect(seen[i].index > seen[i - 1].index, "an index is there twice");
  if (filled) expect(last.bias1 == 1e-3f && last.bias2 > 5.7f && last.bias2 < 5.9f, "the corrections of the step");      // 1 / sqrt(1 - 0.99^3) = 5.80
  const size_t bytes = streambp_grad_norm_workspace_bytes(n_tensors);
  char* ws = (char*)aligned_alloc(256, bytes);
  float norm[1], scale[1];
  expect(streambp_grad_norm(n_tensors, t.data(), 1.f, norm, scale, ws, bytes, nullptr) == SBP_OK, "the norm was refused");
  expect((int64_t)summed.size() == filled && parts_finished <= NORM_WORKGROUPS + n_tensors, "sums of the norm");
  free(ws);
}

int main(int argc, char** argv) {
  std::mt19937_64 rng(7);
  if (argc > 1 && std::string(argv[1]) == "planted") {      // a workspace shorter than the call says: the sums behind its end must be reported
    std::vector<sbp_adamw_tensor> t(1);
    memset(&t[0], 0, sizeof t[0]);
    t[0].n = (int64_t)1 << 30; t[0].grad_dtype = SBP_F32; t[0].grad = (void*)(uintptr_t)4096;
    char* ws = (char*)aligned_alloc(256, 1024);
    float norm[1];
    streambp_grad_norm(1, t.data(), 0.f, norm, nullptr, ws, streambp_grad_norm_workspace_bytes(1), nullptr);
    free(ws);
    printf("not reported\n");
    return 0;
  }
  int cases = 0;
  for (int largest : {3, 12, 20, 30, 35})
    for (int n : {0, 1, 39, 40, 41, 128, 129, 1000}) { one(rng, n, largest); ++cases; }
  printf("OK: %d cases\n", cases);
  return 0;
}
