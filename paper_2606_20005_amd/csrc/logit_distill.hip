// Divergence of a student's rows of logits from a teacher's best tokens
// (streamkl_topk_distill_fwd, streamkl_topk_distill_bwd,
// streamkl_topk_distill_step).
//
// z = s2 x is a student's row, q = exp(z - lse) its distribution over all V
// tokens, (id_k, t_k) the teacher's list.
//   With a rest (t are log probabilities): p_k = exp t_k, and one more bucket
//   holds what neither list nor row assigns to a listed token,
//       p_r = max(1 - sum p_k, 2^-24),   q_r = sum_{j not listed} q_j,
//   L = sum p_k (t_k - log q_k) + p_r (log p_r - log q_r), or the same with the
//   roles of p and q exchanged (reverse).
//   Without: p = softmax(s1 t) over the list, L = sum p_k (log p_k - log q_k).
// Gradients, with P = sum p_k (+ p_r), r = log q - log p of a bucket and
// Q = sum q_k + q_r (1 unless a token is listed twice):
//   dL/dz_j = q_j P - sum_{id_k = j} p_k                 listed
//           = exp(z_j - lse_r) (P q_r - p_r)             not listed (without a rest: q_j P)
//   reverse: q_j (sum_{id_k = j} (r_k + 1) - L - Q)      listed
//           = exp(z_j - lse_r) q_r (r_r + 1 - L - Q)     not listed
// with lse_r = log sum_{j not listed} exp z_j. That sum is formed over the
// logits that are not listed: as 1 - sum q_k it would lose all digits once a
// student is sure of listed tokens. The list of a row is a byte of marks per
// 16-byte chunk in LDS, and a chunk that holds a listed logit (at most K of
// thousands) takes another way through the sums.
//
// What belongs to a row (K terms) is formed by one wave in 64 bits: the terms
// cancel where student and teacher agree, and cost nothing beside the row.
//
// Bound: HBM. A logit is read once forward; the backward pass reads it again
// and writes its gradient.
#include "logit_rows.hpp"
#include "streamkl.h"

namespace streamkl {
namespace {

constexpr int kUnroll = 4;
constexpr int kMostMarks = 33792;        // chunks of a part
constexpr double kLeastRest = 0x1p-24;   // of the teacher's mass outside its list: less is the rounding of its t_k
static_assert(kMostList == 128, "a wave holds a list in two entries a lane");

__device__ __forceinline__ long long id_of(const DistillArgs& a, long long i) {
  return a.ids64 ? static_cast<const long long*>(a.ids)[i] : static_cast<const int*>(a.ids)[i];
}
__device__ __forceinline__ double teacher_of(const DistillArgs& a, long long i) {
  if (a.teacher_dtype == STREAMKL_F32) return (double)static_cast<const float*>(a.teacher)[i];
  if (a.teacher_dtype == STREAMKL_F16) return (double)(float)static_cast<const _Float16*>(a.teacher)[i];
  return (double)(float)static_cast<const __bf16*>(a.teacher)[i];
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) v += __shfl_xor(v, m);
  return v;
}
__device__ __forceinline__ double wave_max(double v) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const double o = __shfl_xor(v, m);
    v = o > v ? o : v;
  }
  return v;
}

// A row's list in LDS: ids that are tokens, -1 for the others.
struct List {
  int id[kMostList];
};

// A row's list as one wave holds it: lane l has the entries l and l + 64.
struct Entries {
  bool there[2];
  int id[2];
  float x[2];            // student's logit
  double t[2];           // teacher's log probability or logit

  // by one wave; `bad`: an id outside the vocabulary
  template <typename T>
  __device__ __forceinline__ void read(const DistillArgs& a, int r, const T* row, List& list, bool* some, bool* bad) {
    const int lane = threadIdx.x & 63;
    bool any = false, out = false;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int k = lane + 64 * i;
      there[i] = false;
      id[i] = -1;
      x[i] = 0.f;
      t[i] = 0.0;
      if (k < a.K) {
        const long long at = (long long)r * a.K + k, v = id_of(a, at);
        out |= v >= a.rows.V;
        there[i] = v >= 0 && v < a.rows.V;
        if (there[i]) {
          id[i] = (int)v;
          x[i] = (float)row[v];
          t[i] = teacher_of(a, at);
        }
      }
      list.id[k] = id[i];
      any |= there[i];
    }
    *some = __any(any);
    *bad = __any(out);
  }
  // the teacher's probabilities and their logarithms
  __device__ __forceinline__ void probabilities(const DistillArgs& a, double (&p)[2], double (&lp)[2]) const {
    double norm = 0.0;
    if (!a.rest) {
      double m = -INFINITY;
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (there[i]) m = fmax(m, (double)a.s1 * t[i]);
      m = wave_max(m);
      double sum = 0.0;
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (there[i]) sum += exp((double)a.s1 * t[i] - m);
      norm = m + log(wave_sum(sum));
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      lp[i] = there[i] ? (a.rest ? t[i] : (double)a.s1 * t[i] - norm) : 0.0;
      p[i] = there[i] ? exp(lp[i]) : 0.0;
    }
  }
};

// A row's loss and statistics from the sums over its logits (without the listed ones where there is a rest), by one wave.
template <typename T>
__device__ void finish_row(const DistillArgs& a, int r, const T* row, const Sums& sums, List& list) {
  Entries e;
  bool some, bad;
  e.read(a, r, row, list, &some, &bad);
  // the list is read by other lanes of this wave
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  // Everything relative to the largest of what there is (x0): absolute log-sum-exps would swallow the differences of rows
  // near the type's lowest value.
  const bool outside = sums.l != 0.f;
  float x0 = outside ? sums.r : kNegInf;
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (a.rest && e.there[i] && e.x[i] > x0) x0 = e.x[i];
  x0 = (float)wave_max((double)x0);
  const double s2 = (double)a.s2;
  // an empty row has x0 = -inf: its numbers are not used
  const double lse_r = outside ? s2 * ((double)sums.r - (double)x0) + log((double)sums.l) : (double)kNegInf;
  double lse = lse_r;
  if (a.rest) {   // with the listed logits, each token once
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int k = (threadIdx.x & 63) + 64 * i;
      bool first = e.there[i];
      for (int j = 0; j < a.K; ++j) first = first && !(j < k && list.id[j] == e.id[i]);
      if (first) sum += exp(s2 * ((double)e.x[i] - (double)x0));
    }
    lse = log(wave_sum(sum) + (outside ? exp(lse_r) : 0.0));
  }
  const bool empty = x0 == kNegInf;
  double p[2], lp[2];
  e.probabilities(a, p, lp);
  double loss = 0.0, rest = 0.0, total = 0.0;
  if (some && !empty) {
    double mass = wave_sum(p[0] + p[1]);
    const bool others = a.rest && outside;   // a bucket that nothing can fill is left out
    double pr = 0.0, lpr = 0.0;
    if (others) {
      pr = 1.0 - mass;
      pr = pr < kLeastRest ? kLeastRest : pr;
      lpr = log(pr);
    }
    const double lqr = lse_r - lse, qr = others ? exp(lqr) : 0.0;
    double terms = 0.0, qs = 0.0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (!e.there[i]) continue;
      const double lq = s2 * ((double)e.x[i] - (double)x0) - lse;
      if (a.reverse) {
        const double q = exp(lq);
        qs += q;
        terms += q == 0.0 ? 0.0 : q * (lq - lp[i]);
      } else {
        terms += p[i] == 0.0 ? 0.0 : p[i] * (lp[i] - lq);
      }
    }
    loss = wave_sum(terms);
    if (a.reverse) {
      if (others) loss += qr * (lqr - lpr);
      total = loss + wave_sum(qs) + qr;
      rest = others ? qr * (lqr - lpr + 1.0 - total) : 0.0;
    } else {
      if (others) loss += pr * (lpr - lqr);
      total = mass + pr;
      rest = a.rest ? (others ? total * qr - pr : 0.0) : total;
    }
    if (outside) rest /= (double)sums.l;
  }
  if (some && bad) loss = rest = total = (double)__builtin_nanf("");
  if ((threadIdx.x & 63) == 0) {
    a.loss[r] = (float)loss;
    a.stats[r] = DistillStats{x0, outside ? sums.r : 0.f, some && !empty ? lse : (double)kNegInf, rest, total};
  }
}

struct Part {
  float r, l;
};

template <typename T, int THREADS, bool REST>
__global__ void __launch_bounds__(THREADS)
distill_kernel(DistillArgs a) {
  __shared__ float red[3 * THREADS / 64];
  __shared__ List list;
  __shared__ int some_sh;
  extern __shared__ u32 marks[];   // REST: a byte per chunk of the part, a bit per listed logit
  int r, s;
  if (!grid_place((long long)a.rows.B * a.rows.N, a.plan.parts, &r, &s)) return;
  const Row<T> row(a.rows, r);
  const int c0 = s * a.plan.chunks, c1 = min(row.chunks, c0 + a.plan.chunks), tid = threadIdx.x;
  const float c = a.s2 * kLog2e, rise = kRise / c;
  if (tid == 0) some_sh = 0;
  if constexpr (REST)
    for (int i = tid; 4 * i < a.plan.chunks; i += THREADS) marks[i] = 0;
  __syncthreads();
  for (int k = tid; k < a.K; k += THREADS) {
    const long long v = id_of(a, (long long)r * a.K + k);
    if (v >= 0) some_sh = 1;
    if (REST && v >= 0 && v < row.V) {
      const int at = (int)v + row.ph, ch = at / kEpc<T> - c0;
      if (ch >= 0 && ch < c1 - c0) atomicOr(&marks[ch / 4], 1u << (8 * (ch % 4) + at % kEpc<T>));
    }
  }
  __syncthreads();
  Sums sums;
  if (some_sh) {   // a row without a list has no loss, whatever its logits
    const unsigned char* const mark = reinterpret_cast<const unsigned char*>(marks);
    each_turn<T, THREADS, kUnroll>(row, c0, c1, [&](int at, const u32x4(&raw)[kUnroll]) {
      float f[kUnroll][kEpc<T>], mx[kUnroll];
      u32 m[kUnroll] = {}, any = 0;
#pragma unroll
      for (int j = 0; j < kUnroll; ++j) {
        if constexpr (REST) {
          const int ch = at + j * THREADS;
          m[j] = ch < c1 ? mark[ch - c0] : 0;
          any |= m[j];
        }
        unpack<T>(raw[j], f[j]);
      }
      if (REST && __any(any != 0)) {
#pragma unroll
        for (int j = 0; j < kUnroll; ++j)
#pragma unroll
          for (int e = 0; e < kEpc<T>; ++e) f[j][e] = (m[j] >> e) & 1 ? kNegInf : f[j][e];
      }
#pragma unroll
      for (int j = 0; j < kUnroll; ++j) mx[j] = max_of<T>(f[j]);
      sums.expect(vmax(vmax3(mx[0], mx[1], mx[2]), mx[3]), c, rise);
    sums.template add<false>(f, c);
    });
  }
  sums = block_join<THREADS>(sums, c, red);
  if (a.plan.parts == 1) {
    if (tid < 64) finish_row(a, r, row.row, sums, list);
  } else if (tid == 0) {
    static_cast<Part*>(a.workspace)[(long long)r * a.plan.parts + s] = Part{sums.r, sums.l};
  }
}

// Joins the parts of a row.
template <typename T>
__global__ void __launch_bounds__(64)
distill_join_kernel(DistillArgs a) {
  __shared__ List list;
  int r, s;
  if (!grid_place((long long)a.rows.B * a.rows.N, 1, &r, &s)) return;
  const Row<T> row(a.rows, r);
  Sums sums;
  if ((int)threadIdx.x < a.plan.parts) {
    const Part p = static_cast<const Part*>(a.workspace)[(long long)r * a.plan.parts + threadIdx.x];
    sums.r = p.r;
    sums.l = p.l;
  }
  sums = wave_join(sums, a.s2 * kLog2e);
  finish_row(a, r, row.row, sums, list);
}

// The upstream gradient of a row.
__device__ __forceinline__ float upstream(const DistillArgs& a, int r) {
  float g = a.factor;
  if (a.weight) g *= a.weight[r];
  if (a.dfactor) g *= *a.dfactor;
  return g;
}

// Gradients of the listed logits of a row, by one wave: value[k] for entry k, in the units of x.
template <typename T>
__device__ void listed_gradients(const DistillArgs& a, int r, const T* row, const DistillStats& st, float g, List& list,
                                 float* add, float* value) {
  Entries e;
  bool some, bad;
  e.read(a, r, row, list, &some, &bad);
  double p[2], lp[2];
  e.probabilities(a, p, lp);
  double q[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int k = (threadIdx.x & 63) + 64 * i;
    const double lq = (double)a.s2 * ((double)e.x[i] - (double)st.x0) - st.lse;
    q[i] = e.there[i] ? exp(lq) : 0.0;
    // what the entry adds to its token: forward -p, reverse q (r + 1)
    add[k] = (float)(a.reverse ? (q[i] == 0.0 ? 0.0 : q[i] * (lq - lp[i] + 1.0)) : -p[i]);
  }
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int k = (threadIdx.x & 63) + 64 * i;
    double v = a.reverse ? (q[i] == 0.0 ? 0.0 : -q[i] * st.total) : q[i] * st.total;
    if (e.there[i])
      for (int j = 0; j < a.K; ++j) v += list.id[j] == e.id[i] ? (double)add[j] : 0.0;   // entries of one token
    value[k] = (float)(v * ((double)a.s2 * (double)g));
  }
}

// dx of a part of a row.
template <typename T, int THREADS>
__global__ void __launch_bounds__(THREADS)
distill_grad_kernel(DistillArgs a) {
  __shared__ List list;
  __shared__ float add[kMostList], value[kMostList];
  if (a.done_if_one && *a.dfactor == 1.f) return;
  int r, s;
  if (!grid_place((long long)a.rows.B * a.rows.N, a.plan.parts, &r, &s)) return;
  const Row<T> row(a.rows, r);
  const int c0 = s * a.plan.chunks, c1 = min(row.chunks, c0 + a.plan.chunks), tid = threadIdx.x;
  const int b = r / a.rows.N;
  T* const dx = static_cast<T*>(a.dx) + b * a.dsb + (r - b * a.rows.N) * a.dsn;
  const float g = upstream(a, r);
  const DistillStats st = a.stats[r];
  if (g == 0.f || st.lse == (double)kNegInf) {   // rows without an upstream gradient, a list or a token
    float z[kEpc<T>] = {};
    for (int ch = c0 + tid; ch < c1; ch += THREADS) store<T>(row, dx, ch, z);
    return;
  }
  // dx may be x: listed logits are read before anything is written, by the part that holds them as well
  if (tid < 64) listed_gradients(a, r, row.row, st, g, list, add, value);
  __syncthreads();
  const float c = a.s2 * kLog2e;
  const float at = st.r, w = (float)((double)a.s2 * (double)g * st.rest);
  each_turn<T, THREADS, kUnroll>(row, c0, c1, [&](int first, const u32x4(&raw)[kUnroll]) {
#pragma unroll
    for (int j = 0; j < kUnroll; ++j) {
      const int ch = first + j * THREADS;
      float f[kEpc<T>];
      unpack<T>(raw[j], f);
#pragma unroll
      for (int i = 0; i < kEpc<T>; ++i) f[i] = exp2_fast((f[i] - at) * c) * w;
      if (ch < c1) store<T>(row, dx, ch, f);
    }
  });
  __syncthreads();
  for (int k = tid; k < a.K; k += THREADS) {
    const int id = list.id[k], ch = id < 0 ? -1 : (id + row.ph) / kEpc<T>;
    if (ch >= c0 && ch < c1) dx[id] = (T)value[k];
  }
}

// total = sum of weight factor loss over the rows whose weight is not 0, by one workgroup.
constexpr int kSumThreads = 1024;

__global__ void __launch_bounds__(kSumThreads)
weighted_sum_kernel(const float* loss, const float* weight, float factor, long long rows, float* total) {
  __shared__ double red[kSumThreads / 64];
  double v = 0.0;
  for (long long i = threadIdx.x; i < rows; i += kSumThreads) {
    const float w = weight ? weight[i] : 1.f;
    v += w == 0.f ? 0.0 : (double)w * (double)loss[i];
  }
  v = wave_sum(v);
  if (threadIdx.x % 64 == 0) red[threadIdx.x / 64] = v;
  __syncthreads();
  if (threadIdx.x == 0) {
    double t = 0.0;
    for (int i = 0; i < kSumThreads / 64; ++i) t += red[i];
    *total = (float)(t * (double)factor);
  }
}

template <int THREADS, typename T>
void run_fwd(const DistillArgs& a, dim3 grid) {
  if (a.rest)
    distill_kernel<T, THREADS, true><<<grid, dim3(THREADS), (size_t)a.plan.chunks, a.stream>>>(a);
  else
    distill_kernel<T, THREADS, false><<<grid, dim3(THREADS), 0, a.stream>>>(a);
}

}  // namespace

LogitPlan distill_plan(long long rows, int V, int dtype, int rest) {
  const int epc = dtype == STREAMKL_F32 ? 4 : 8, chunks = chunks_of(V, dtype);
  long long parts = rows ? 512 / rows : 1;
  const long long useful = ((long long)V + 8191) / 8192;
  if (parts > useful) parts = useful;
  const long long least = rest ? (chunks + kMostMarks - 1) / kMostMarks : 1;
  if (parts < least) parts = least;
  if (parts < 1) parts = 1;
  if (parts > kMostParts) parts = kMostParts;
  LogitPlan p;
  p.chunks = (int)((chunks + parts - 1) / parts + 3) / 4 * 4;
  p.parts = (chunks + p.chunks - 1) / p.chunks;
  p.threads = (long long)p.chunks * epc <= 16384 ? 256 : 512;
  return p;
}

size_t distill_workspace(long long rows, const LogitPlan& p) {
  return p.parts <= 1 ? 0 : (size_t)rows * p.parts * sizeof(Part);
}

hipError_t launch_distill(const DistillArgs& a) {
  const long long rows = (long long)a.rows.B * a.rows.N;
  const dim3 grid = logit_grid(rows * a.plan.parts);
  by_type(a.rows.dtype, [&](auto t) {
    if (a.plan.threads == 256)
      run_fwd<256, decltype(t)>(a, grid);
    else
      run_fwd<512, decltype(t)>(a, grid);
    if (a.plan.parts > 1) distill_join_kernel<decltype(t)><<<logit_grid(rows), dim3(64), 0, a.stream>>>(a);
  });
  return hipGetLastError();
}

LogitPlan distill_grad_plan(long long rows, int V, int dtype) {
  const int chunks = chunks_of(V, dtype);
  const long long parts = ((long long)V + 32767) / 32768;
  LogitPlan p;
  p.chunks = (int)((chunks + parts - 1) / parts + 3) / 4 * 4;
  p.parts = (chunks + p.chunks - 1) / p.chunks;
  p.threads = 256;
  return p;
}

hipError_t launch_distill_grad(const DistillArgs& a) {
  const dim3 grid = logit_grid((long long)a.rows.B * a.rows.N * a.plan.parts);
  by_type(a.rows.dtype, [&](auto t) {
    distill_grad_kernel<decltype(t), 256><<<grid, dim3(256), 0, a.stream>>>(a);
  });
  return hipGetLastError();
}

hipError_t launch_weighted_sum(const float* loss, const float* weight, float factor, long long rows, float* total,
                               hipStream_t stream) {
  weighted_sum_kernel<<<dim3(1), dim3(kSumThreads), 0, stream>>>(loss, weight, factor, rows, total);
  return hipGetLastError();
}

}  // namespace streamkl
