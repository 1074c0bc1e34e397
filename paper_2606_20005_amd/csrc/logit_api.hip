// C ABI of the operators on rows of logits: argument checks and sizes
// (streamkl_token_logprobs_*, streamkl_topk_distill_*).
#include <cmath>
#include <cstdint>

#include "logit_launch.hpp"
#include "streamkl.h"

using namespace streamkl;

namespace {

constexpr long long kMostRows = 0x7fff0000LL;
constexpr long long kMostWorkgroups = 1LL << 36;   // of the two axes of a grid

bool aligned_to(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool known_type(int t) { return t == STREAMKL_BF16 || t == STREAMKL_F16 || t == STREAMKL_F32; }
uintptr_t size_of(int t) { return t == STREAMKL_F32 ? 4 : 2; }
bool known_scale(float s) { return std::isfinite(s) && s >= 0x1p-64f && s <= 0x1p64f; }

bool countable(int B, int N, long long parts) {
  const long long rows = (long long)B * N;
  return rows <= kMostRows && rows * parts <= kMostWorkgroups;
}

int check_logits(const streamkl_logits* x) {
  if (!x || x->B < 0 || x->N < 0 || !known_type(x->dtype)) return STREAMKL_ERR_INVALID_ARG;
  if (x->V < 0 || x->sb < 0 || x->sn < 0) return STREAMKL_ERR_INVALID_ARG;
  if (x->V > kMostVocab || (long long)x->B * x->N > kMostRows) return STREAMKL_ERR_UNSUPPORTED;
  if (x->B == 0 || x->N == 0) return STREAMKL_OK;
  if (x->V < 1 || !x->data || !aligned_to(x->data, size_of(x->dtype))) return STREAMKL_ERR_INVALID_ARG;
  return STREAMKL_OK;
}

// Rows of gradients: none overlaps another.
int check_grads(const streamkl_logits* x, const void* dx, long long sb, long long sn) {
  if (!dx || !aligned_to(dx, size_of(x->dtype)) || sb < 0 || sn < 0) return STREAMKL_ERR_INVALID_ARG;
  const long long V = x->V, N = x->N, B = x->B;
  constexpr long long far = 1LL << 60;
  if (sb > far || sn > far / N) return sb > far || sn > far ? STREAMKL_ERR_INVALID_ARG : STREAMKL_ERR_UNSUPPORTED;
  if (N > 1 && sn < V) return STREAMKL_ERR_INVALID_ARG;
  if (B > 1 && sb < V) return STREAMKL_ERR_INVALID_ARG;
  if (N > 1 && B > 1 && sb < (N - 1) * sn + V && (sb > far / B || sn < (B - 1) * sb + V)) return STREAMKL_ERR_INVALID_ARG;
  return STREAMKL_OK;
}

LogitRows rows_of(const streamkl_logits* x) {
  return LogitRows{x->data, x->sb, x->sn, x->B, x->N, x->V, x->dtype};
}

bool empty(const streamkl_logits* x) { return x->B == 0 || x->N == 0; }

int check_teacher(const streamkl_logits* x, const streamkl_teacher_list* t, int direction) {
  if (!t || t->K < 1 || !known_type(t->dtype) || (t->ids64 != 0 && t->ids64 != 1) || (t->rest != 0 && t->rest != 1))
    return STREAMKL_ERR_INVALID_ARG;
  if (direction != STREAMKL_KL_FWD && direction != STREAMKL_KL_REV) return STREAMKL_ERR_INVALID_ARG;
  if (!known_scale(t->scale) || (t->rest && t->scale != 1.f)) return STREAMKL_ERR_INVALID_ARG;
  if (t->K > kMostList || (direction == STREAMKL_KL_REV && !t->rest)) return STREAMKL_ERR_UNSUPPORTED;
  if (empty(x)) return STREAMKL_OK;
  if (!t->ids || !aligned_to(t->ids, t->ids64 ? 8 : 4) || !t->values || !aligned_to(t->values, size_of(t->dtype)))
    return STREAMKL_ERR_INVALID_ARG;
  return STREAMKL_OK;
}

DistillArgs distill_args(const streamkl_logits* x, const streamkl_teacher_list* t, float scale, int direction,
                         hipStream_t stream) {
  DistillArgs a = {};
  a.rows = rows_of(x);
  a.ids = t->ids;
  a.ids64 = t->ids64;
  a.teacher = t->values;
  a.teacher_dtype = t->dtype;
  a.K = t->K;
  a.s1 = t->scale;
  a.s2 = scale;
  a.rest = t->rest;
  a.reverse = direction == STREAMKL_KL_REV;
  a.factor = 1.f;
  a.stream = stream;
  return a;
}

int status(hipError_t e) { return e == hipSuccess ? STREAMKL_OK : STREAMKL_ERR_HIP; }

int check_workspace(const void* workspace, size_t bytes, size_t need) {
  return need && (!workspace || !aligned_to(workspace, 16) || bytes < need) ? STREAMKL_ERR_INVALID_ARG : STREAMKL_OK;
}

}  // namespace

extern "C" size_t streamkl_token_logprobs_workspace_bytes(int B, int N, int V, int dtype, int top) {
  if (B < 0 || N < 0 || V < 1 || V > kMostVocab || !known_type(dtype) || top < 0 || top > kMostTop || top > V) return 0;
  const long long rows = (long long)B * N;
  if (rows > kMostRows) return 0;
  return logprob_workspace(rows, logprob_plan(rows, V, dtype == STREAMKL_F32, top), top);
}

extern "C" int streamkl_token_logprobs_fwd(const streamkl_logits* x, const void* tokens, int tokens64, float scale, int top,
                                           void* workspace, size_t workspace_bytes, float* logp, float* entropy,
                                           float* lse, float* lse_err, float* top_logp, int* top_ids,
                                           hipStream_t stream) {
  int st = check_logits(x);
  if (st != STREAMKL_OK) return st;
  if (!known_scale(scale) || (tokens64 != 0 && tokens64 != 1) || top < 0) return STREAMKL_ERR_INVALID_ARG;
  if (top > kMostTop) return STREAMKL_ERR_UNSUPPORTED;
  if (empty(x)) return STREAMKL_OK;
  if (top > x->V || !tokens != !logp || !aligned_to(tokens, tokens64 ? 8 : 4)) return STREAMKL_ERR_INVALID_ARG;
  if (top > 0 && (!top_logp || !top_ids)) return STREAMKL_ERR_INVALID_ARG;
  for (const void* p : {(const void*)logp, (const void*)entropy, (const void*)lse, (const void*)lse_err,
                        (const void*)top_logp, (const void*)top_ids})
    if (!aligned_to(p, 4)) return STREAMKL_ERR_INVALID_ARG;
  if (!logp && !entropy && !lse && !lse_err && top == 0) return STREAMKL_ERR_INVALID_ARG;
  LogprobArgs a = {};
  a.rows = rows_of(x);
  const long long rows = (long long)x->B * x->N;
  a.plan = logprob_plan(rows, x->V, x->dtype == STREAMKL_F32, top);
  if (!countable(x->B, x->N, a.plan.parts)) return STREAMKL_ERR_UNSUPPORTED;
  st = check_workspace(workspace, workspace_bytes, logprob_workspace(rows, a.plan, top));
  if (st != STREAMKL_OK) return st;
  a.tokens = tokens;
  a.tokens64 = tokens64;
  a.scale = scale;
  a.top = top;
  a.workspace = workspace;
  a.logp = logp;
  a.entropy = entropy;
  a.lse = lse;
  a.lse_err = lse_err;
  a.top_logp = top_logp;
  a.top_ids = top_ids;
  a.stream = stream;
  return status(launch_logprob(a));
}

extern "C" int streamkl_token_logprobs_bwd(const streamkl_logits* x, const void* tokens, int tokens64, float scale,
                                           const float* lse, const float* lse_err, const float* entropy,
                                           const float* dlogp, const float* dentropy, const float* dlse, void* dx,
                                           long long dx_sb, long long dx_sn, hipStream_t stream) {
  int st = check_logits(x);
  if (st != STREAMKL_OK) return st;
  if (!known_scale(scale) || (tokens64 != 0 && tokens64 != 1)) return STREAMKL_ERR_INVALID_ARG;
  if (empty(x)) return STREAMKL_OK;
  st = check_grads(x, dx, dx_sb, dx_sn);
  if (st != STREAMKL_OK) return st;
  if (!lse || (dlogp && !tokens) || (dentropy && !entropy) || !aligned_to(tokens, tokens64 ? 8 : 4))
    return STREAMKL_ERR_INVALID_ARG;
  for (const float* p : {lse, lse_err, entropy, dlogp, dentropy, dlse})
    if (!aligned_to(p, 4)) return STREAMKL_ERR_INVALID_ARG;
  LogprobGradArgs a = {};
  a.rows = rows_of(x);
  a.plan = grad_plan(x->V, x->dtype == STREAMKL_F32);
  if (!countable(x->B, x->N, a.plan.parts)) return STREAMKL_ERR_UNSUPPORTED;
  a.tokens = tokens;
  a.tokens64 = tokens64;
  a.scale = scale;
  a.lse = lse;
  a.lse_err = lse_err;
  a.entropy = entropy;
  a.dlogp = dlogp;
  a.dentropy = dentropy;
  a.dlse = dlse;
  a.dx = dx;
  a.dsb = dx_sb;
  a.dsn = dx_sn;
  a.stream = stream;
  return status(launch_logprob_grad(a));
}

extern "C" size_t streamkl_topk_distill_workspace_bytes(int B, int N, int V, int dtype, int rest) {
  if (B < 0 || N < 0 || V < 1 || V > kMostVocab || !known_type(dtype)) return 0;
  const long long rows = (long long)B * N;
  if (rows > kMostRows) return 0;
  return distill_workspace(rows, distill_plan(rows, V, dtype == STREAMKL_F32, rest != 0));
}

namespace {

// Arguments of a forward pass; its checks.
int distill_forward(const streamkl_logits* x, const streamkl_teacher_list* t, float scale, int direction, void* workspace,
                    size_t workspace_bytes, float* loss, void* stats, hipStream_t stream, DistillArgs* a) {
  int st = check_logits(x);
  if (st == STREAMKL_OK) st = check_teacher(x, t, direction);
  if (st == STREAMKL_OK && !known_scale(scale)) st = STREAMKL_ERR_INVALID_ARG;
  if (st != STREAMKL_OK || empty(x)) return st;
  if (!loss || !aligned_to(loss, 4) || !stats || !aligned_to(stats, 8)) return STREAMKL_ERR_INVALID_ARG;
  *a = distill_args(x, t, scale, direction, stream);
  const long long rows = (long long)x->B * x->N;
  a->plan = distill_plan(rows, x->V, x->dtype == STREAMKL_F32, t->rest != 0);
  if (!countable(x->B, x->N, a->plan.parts)) return STREAMKL_ERR_UNSUPPORTED;
  a->workspace = workspace;
  a->loss = loss;
  a->stats = static_cast<DistillStats*>(stats);
  return check_workspace(workspace, workspace_bytes, distill_workspace(rows, a->plan));
}

}  // namespace

extern "C" int streamkl_topk_distill_fwd(const streamkl_logits* x, const streamkl_teacher_list* t, float scale,
                                         int direction, void* workspace, size_t workspace_bytes, float* loss, void* stats,
                                         hipStream_t stream) {
  DistillArgs a;
  const int st = distill_forward(x, t, scale, direction, workspace, workspace_bytes, loss, stats, stream, &a);
  if (st != STREAMKL_OK || empty(x)) return st;
  return status(launch_distill(a));
}

extern "C" int streamkl_topk_distill_bwd(const streamkl_logits* x, const streamkl_teacher_list* t, float scale,
                                         int direction, const void* stats, const float* dloss, float factor,
                                         const float* dfactor, int done_if_one, void* dx, long long dx_sb, long long dx_sn,
                                         hipStream_t stream) {
  int st = check_logits(x);
  if (st == STREAMKL_OK) st = check_teacher(x, t, direction);
  if (st == STREAMKL_OK && (!known_scale(scale) || (done_if_one != 0 && done_if_one != 1) || (done_if_one && !dfactor)))
    st = STREAMKL_ERR_INVALID_ARG;
  if (st != STREAMKL_OK || empty(x)) return st;
  st = check_grads(x, dx, dx_sb, dx_sn);
  if (st != STREAMKL_OK) return st;
  if (!stats || !aligned_to(stats, 8) || !aligned_to(dloss, 4) || !aligned_to(dfactor, 4)) return STREAMKL_ERR_INVALID_ARG;
  DistillArgs a = distill_args(x, t, scale, direction, stream);
  a.plan = grad_plan(x->V, x->dtype == STREAMKL_F32);
  if (!countable(x->B, x->N, a.plan.parts)) return STREAMKL_ERR_UNSUPPORTED;
  a.stats = const_cast<DistillStats*>(static_cast<const DistillStats*>(stats));
  a.weight = dloss;
  a.factor = factor;
  a.dfactor = dfactor;
  a.done_if_one = done_if_one;
  a.dx = dx;
  a.dsb = dx_sb;
  a.dsn = dx_sn;
  return status(launch_distill_grad(a));
}

extern "C" int streamkl_topk_distill_step(const streamkl_logits* x, const streamkl_teacher_list* t, float scale,
                                          int direction, void* workspace, size_t workspace_bytes, const float* weight,
                                          float factor, float* loss, void* stats, void* dx, long long dx_sb,
                                          long long dx_sn, hipStream_t stream) {
  DistillArgs a;
  int st = distill_forward(x, t, scale, direction, workspace, workspace_bytes, loss, stats, stream, &a);
  if (st != STREAMKL_OK || empty(x)) return st;
  st = check_grads(x, dx, dx_sb, dx_sn);
  if (st != STREAMKL_OK) return st;
  if (!aligned_to(weight, 4)) return STREAMKL_ERR_INVALID_ARG;
  const LogitPlan back = grad_plan(x->V, x->dtype == STREAMKL_F32);
  if (!countable(x->B, x->N, back.parts)) return STREAMKL_ERR_UNSUPPORTED;
  a.weight = weight;
  a.factor = factor;
  a.dx = dx;
  a.dsb = dx_sb;
  a.dsn = dx_sn;
  if (distill_step_fits((long long)x->B * x->N, x->V, x->dtype == STREAMKL_F32)) return status(launch_distill_step(a));
  st = status(launch_distill(a));
  if (st != STREAMKL_OK) return st;
  a.plan = back;
  return status(launch_distill_grad(a));
}

extern "C" int streamkl_topk_distill_total(const float* loss, const float* weight, float factor, long long rows,
                                           float* total, hipStream_t stream) {
  if (rows < 0 || !total || !aligned_to(total, 4) || !aligned_to(weight, 4)) return STREAMKL_ERR_INVALID_ARG;
  if (rows > 0 && (!loss || !aligned_to(loss, 4))) return STREAMKL_ERR_INVALID_ARG;
  return status(launch_weighted_sum(loss, weight, factor, rows, total, stream));
}
