// Internal launch interface between the C ABI of the operators on logits
// (logit_api.hip) and their kernels (logit_logprobs.hip, logit_distill.hip).
// The host has checked extents, pointers and sizes.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>

namespace streamkl {

// Rows r = b N + n of V logits; strides in elements.
struct LogitRows {
  const void* x;
  long long sb, sn;
  int B, N, V, dtype;
};

constexpr int kMostTop = 128;          // alternatives of a row
constexpr int kMostList = 128;         // entries of a teacher's list
constexpr int kMostParts = 32;         // parts that a row is cut into
constexpr int kMostVocab = 1 << 22;

// How a pass cuts its rows: parts of `chunks` 16-byte chunks each (a multiple of 4), `threads` a workgroup.
struct LogitPlan {
  int threads, parts, chunks;
};

// A grid of n workgroups: an axis holds less than 2^32 threads.
inline dim3 logit_grid(long long n) {
  constexpr long long most = 1 << 21;
  return n <= most ? dim3((unsigned)n) : dim3((unsigned)most, (unsigned)((n + most - 1) / most));
}

struct LogprobArgs {
  LogitRows rows;
  const void* tokens;
  int tokens64;
  float scale;
  int top;
  LogitPlan plan;
  void* workspace;
  float *logp, *entropy, *lse, *lse_err, *top_logp;
  int* top_ids;
  hipStream_t stream;
};

struct LogprobGradArgs {
  LogitRows rows;
  const void* tokens;
  int tokens64;
  float scale;
  LogitPlan plan;
  const float *lse, *lse_err, *entropy, *dlogp, *dentropy, *dlse;
  void* dx;
  long long dsb, dsn;
  hipStream_t stream;
};

// What the kernels of a distillation need of a row after the forward pass.
struct DistillStats {
  float x0;       // a logit that those of the list are taken relative to
  float r;        // the same for the others
  double lse;     // log sum_j exp(s2 (x_j - x0)); -inf: the row has no loss
  double rest;    // d loss / d z_j = rest exp(s2 (x_j - r)) for tokens outside the list
  double total;   // of the list: see the kernels
};

struct DistillArgs {
  LogitRows rows;
  const void* ids;
  int ids64;
  const void* teacher;
  int teacher_dtype, K;
  float s1, s2;
  int rest, reverse;
  LogitPlan plan;
  void* workspace;
  float* loss;
  DistillStats* stats;
  // gradient: row r has the upstream gradient weight[r] factor *dfactor (each 1 where null)
  const float* weight;
  float factor;
  const float* dfactor;
  int done_if_one;   // nothing to do where *dfactor is 1
  void* dx;
  long long dsb, dsn;
  hipStream_t stream;
};

LogitPlan logprob_plan(long long rows, int V, int dtype, int top);
size_t logprob_workspace(long long rows, const LogitPlan& p, int top);
hipError_t launch_logprob(const LogprobArgs& a);
LogitPlan logprob_grad_plan(long long rows, int V, int dtype);
hipError_t launch_logprob_grad(const LogprobGradArgs& a);

LogitPlan distill_plan(long long rows, int V, int dtype, int rest);
size_t distill_workspace(long long rows, const LogitPlan& p);
hipError_t launch_distill(const DistillArgs& a);
LogitPlan distill_grad_plan(long long rows, int V, int dtype);
hipError_t launch_distill_grad(const DistillArgs& a);
// Loss and gradient in one kernel, for sizes that it holds.
bool distill_step_fits(long long rows, int V, int dtype);
hipError_t launch_distill_step(const DistillArgs& a);
hipError_t launch_weighted_sum(const float* loss, const float* weight, float factor, long long rows, float* total,
                               hipStream_t stream);

}  // namespace streamkl
