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

constexpr int kGroup = 16;             // logits of a group, whose maximum is kept
constexpr int kMostGroups = 8448;      // of a part with alternatives: 135168 logits
constexpr int kMostMarks = 33792;      // chunks of a part with marks

// The most 16-byte chunks that a row of any alignment has.
inline int chunks_of(int V, bool f32) {
  const int epc = f32 ? 4 : 8;
  return (V + epc - 1 + epc - 1) / epc;
}

// A row in parts of a multiple of 4 chunks.
inline LogitPlan cut(int chunks, long long parts) {
  LogitPlan p;
  p.chunks = (int)((chunks + parts - 1) / parts + 3) / 4 * 4;
  p.parts = (chunks + p.chunks - 1) / p.chunks;
  p.threads = 256;
  return p;
}

// Forward passes: a workgroup a row; two a CU where rows are fewer, as long as a part has 8192 logits, and no more chunks
// in a part than its workgroup's LDS has room for.
inline LogitPlan forward_plan(long long rows, int V, bool f32, int most_chunks) {
  const int epc = f32 ? 4 : 8, chunks = chunks_of(V, f32);
  long long parts = rows ? 512 / rows : 1;
  const long long useful = ((long long)V + 8191) / 8192, least = ((long long)chunks + most_chunks - 1) / most_chunks;
  if (parts > useful) parts = useful;
  if (parts < least) parts = least;
  if (parts < 1) parts = 1;
  if (parts > kMostParts) parts = kMostParts;
  LogitPlan p = cut(chunks, parts);
  if ((long long)p.chunks * epc > 16384) p.threads = 512;
  return p;
}

inline LogitPlan logprob_plan(long long rows, int V, bool f32, int top) {
  return forward_plan(rows, V, f32, top > 0 ? kMostGroups * kGroup / (f32 ? 4 : 8) : 1 << 30);
}

inline LogitPlan distill_plan(long long rows, int V, bool f32, bool rest) {
  return forward_plan(rows, V, f32, rest ? kMostMarks : 1 << 30);
}

// Backward passes: parts of at most 32768 logits.
inline LogitPlan grad_plan(int V, bool f32) { return cut(chunks_of(V, f32), ((long long)V + 32767) / 32768); }

// The sums of a part.
struct LogprobPart {
  float r, l, a;
};
struct DistillPart {
  float r, l;
};

// Sums of all parts, then their keys.
__host__ __device__ inline size_t logprob_part_bytes(long long rows, const LogitPlan& p) {
  return ((size_t)rows * p.parts * sizeof(LogprobPart) + 15) / 16 * 16;
}
inline size_t logprob_workspace(long long rows, const LogitPlan& p, int top) {
  return p.parts <= 1 ? 0 : logprob_part_bytes(rows, p) + (size_t)rows * p.parts * top * 8;
}
inline size_t distill_workspace(long long rows, const LogitPlan& p) {
  return p.parts <= 1 ? 0 : (size_t)rows * p.parts * sizeof(DistillPart);
}

// Whether a distillation step runs as one kernel, a workgroup a row, or as a forward and a backward pass in parts: for few
// long rows parts fill the chip (one kernel and three, us: 4096 logits, 1 row 8.8 and 12.7; 32000, 1 row 15.5 and 19.4;
// 128000, 16 rows 25 and 21, 64 rows 25.8 both, 128 rows 28 and 34; 262144, 128 rows 61 and 49, 256 rows 68 and 81). Rows
// whose marks, a byte a chunk, are more than LDS is kept for take two passes as well: float32 from some 135000 logits on.
inline bool distill_step_fits(long long rows, int V, bool f32) {
  const int chunks = chunks_of(V, f32);
  return chunks <= kMostMarks && (chunks <= 8192 || rows * 128 >= chunks);
}

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

hipError_t launch_logprob(const LogprobArgs& a);
hipError_t launch_logprob_grad(const LogprobGradArgs& a);

hipError_t launch_distill(const DistillArgs& a);
hipError_t launch_distill_grad(const DistillArgs& a);
// Loss and gradient in one kernel, for sizes that it holds.
hipError_t launch_distill_step(const DistillArgs& a);
hipError_t launch_weighted_sum(const float* loss, const float* weight, float factor, long long rows, float* total,
                               hipStream_t stream);

}  // namespace streamkl
