// Divergence of a student's rows of logits from a teacher's best tokens: what
// the kernels of logit_distill.hip (streamkl_topk_distill_fwd, _bwd) and
// logit_distill_step.hip (streamkl_topk_distill_step) do with a row's list.
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
// What belongs to a row (K terms) is formed by one wave. Log probabilities,
// their differences and the sums of the terms are held in 64 bits: they cancel
// where student and teacher agree (with float32 logarithms and exponentials
// the losses of 4094 rows were off by 4.5e-7 instead of 6e-8, for half a
// percent of the time). The probabilities that the differences are weighed
// with, and those of the gradients, are float32: p_k rounded once, q_k and q_r
// the exponential of a float32 exponent, off by 2^-24 |log2 q| of themselves,
// in terms of the size q |log q - log p|. What does not depend on the sums over the row is prepared while its
// logits are on their way.
#pragma once

#include "logit_rows.hpp"
#include "streamkl.h"

namespace streamkl {

constexpr double kLeastRest = 0x1p-24;   // of the teacher's mass outside its list: less is the rounding of its t_k
static_assert(kMostList == 128, "a wave holds a list in two entries a lane");

__device__ __forceinline__ long long id_of(const DistillArgs& a, long long i) {
  return a.ids64 ? static_cast<const long long*>(a.ids)[i] : static_cast<const int*>(a.ids)[i];
}
__device__ __forceinline__ float teacher_of(const DistillArgs& a, long long i) {
  if (a.teacher_dtype == STREAMKL_F32) return static_cast<const float*>(a.teacher)[i];
  if (a.teacher_dtype == STREAMKL_F16) return (float)static_cast<const _Float16*>(a.teacher)[i];
  return (float)static_cast<const __bf16*>(a.teacher)[i];
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) v += __shfl_xor(v, m);
  return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) v = fmaxf(v, __shfl_xor(v, m));
  return v;
}
// exp of a number formed in 64 bits
__device__ __forceinline__ float exp_of(double v) { return exp2_fast((float)(v * 1.4426950408889634074)); }

// Logits of a chunk that `marks` names count as -inf. Few chunks have some: of 64 in 16000, a wave meets one in every fifth
// of its own.
template <int E>
__device__ __forceinline__ void leave_out(float (&f)[E], u32 marks) {
  if (__any(marks != 0)) {
#pragma unroll
    for (int e = 0; e < E; ++e) f[e] = (marks >> e) & 1 ? kNegInf : f[e];
  }
}

// A row's list in LDS.
struct List {
  int id[kMostList];       // -1: no entry
  float x[kMostList];      // student's logit
  float t[kMostList];      // teacher's value
  double lp[kMostList];    // teacher's log probability
  float p[kMostList];      // and probability
  float add[kMostList];    // what an entry adds to the gradient of its token
  float value[kMostList];  // the gradient of its token
  double mass;             // sum of p
  int some, bad, twice;    // whether there are entries, one of them outside the vocabulary, a token with two
};

// Before: list.some = list.bad = list.twice = 0 and a barrier. Entries by the threads of a workgroup, f(entry, id) for each
// that is a token. After: a barrier.
template <typename T, int THREADS, typename F>
__device__ __forceinline__ void read_list(const DistillArgs& a, int r, const T* row, List& list, F f) {
  for (int k = threadIdx.x; k < kMostList; k += THREADS) {
    int id = -1;
    if (k < a.K) {
      const long long at = (long long)r * a.K + k, v = id_of(a, at);
      if (v >= 0) list.some = 1;
      if (v >= a.rows.V) list.bad = 1;
      if (v >= 0 && v < a.rows.V) {
        id = (int)v;
        f(k, id);
        list.t[k] = teacher_of(a, at);
        list.x[k] = (float)row[id];
      }
    }
    list.id[k] = id;
  }
}

__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// The teacher's side, by one wave: lp, p, mass and twice. Without a rest everything relative to the largest value: an absolute
// log-sum-exp would swallow log sum of a list near the type's lowest value (which is uniform), in 64 bits too.
__device__ __forceinline__ void teacher_side(const DistillArgs& a, List& list) {
  const int lane = threadIdx.x & 63;
  bool there[2];
  float t[2];
  double lp[2];
  double norm = 0.0;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    there[i] = list.id[lane + 64 * i] >= 0;
    t[i] = there[i] ? list.t[lane + 64 * i] : kNegInf;
    lp[i] = (double)t[i];   // with a rest s1 is 1
  }
  if (!a.rest) {
    const float m = wave_max(fmaxf(t[0], t[1]));
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      lp[i] = (double)a.s1 * ((double)t[i] - (double)m);
      if (there[i]) sum += exp(lp[i]);
    }
    norm = log(wave_sum(sum));
  }
  double mass = 0.0;
  bool twice = false;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int k = lane + 64 * i;
    lp[i] -= norm;
    // in 64 bits: the rest is what the sum of these leaves of 1
    const double p = there[i] ? exp(lp[i]) : 0.0;
    mass += p;
    list.lp[k] = lp[i];
    list.p[k] = (float)p;
    if (there[i])
      for (int j = 0; j < k; ++j) twice |= list.id[j] == list.id[k];
  }
  mass = wave_sum(mass);
  if (lane == 0) list.mass = mass;
  if (__any(twice) && lane == 0) list.twice = 1;
}

// Whether an earlier entry has the token of entry k.
__device__ __forceinline__ bool had_before(const List& list, int k) {
  bool had = false;
  if (list.twice)
    for (int j = 0; j < k; ++j) had |= list.id[j] == list.id[k];
  return had;
}

// A row's loss and statistics from the sums over its logits (without the listed ones where there is a rest), by one wave
// after teacher_side.
__device__ __forceinline__ DistillStats finish_row(const DistillArgs& a, const Sums& sums, const List& list, float* loss_out) {
  const int lane = threadIdx.x & 63;
  bool there[2];
  float x[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    there[i] = list.id[lane + 64 * i] >= 0;
    x[i] = there[i] ? list.x[lane + 64 * i] : kNegInf;
  }
  // Everything relative to the largest of what there is (x0): absolute log-sum-exps would swallow the differences of rows
  // near the type's lowest value.
  const bool outside = sums.l != 0.f;
  float x0 = outside ? sums.r : kNegInf;
  if (a.rest) x0 = wave_max(fmaxf(x0, fmaxf(x[0], x[1])));
  const bool empty = x0 == kNegInf;
  const double s2 = (double)a.s2;
  const double lse_r = outside ? s2 * ((double)sums.r - (double)x0) + log((double)sums.l) : (double)kNegInf;
  double lse = lse_r;
  if (a.rest) {   // with the listed logits, each token once
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (there[i] && !had_before(list, lane + 64 * i)) sum += exp(s2 * ((double)x[i] - (double)x0));
    lse = log(wave_sum(sum) + (outside ? exp(lse_r) : 0.0));
  }
  double loss = 0.0, rest = 0.0, total = 0.0;
  if (list.some && !empty) {
    const bool others = a.rest && outside;   // a bucket that nothing can fill is left out
    double pr = 0.0, lpr = 0.0;
    if (others) {
      pr = 1.0 - list.mass;
      pr = pr < kLeastRest ? kLeastRest : pr;
      lpr = log(pr);
    }
    const double lqr = lse_r - lse, qr = others ? (double)exp_of(lqr) : 0.0;
    double terms = 0.0, qs = 0.0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (!there[i]) continue;
      const double lq = s2 * ((double)x[i] - (double)x0) - lse, lp = list.lp[lane + 64 * i];
      const double p = (double)list.p[lane + 64 * i];
      if (a.reverse) {
        const double q = (double)exp_of(lq);
        qs += q;
        terms += q == 0.0 ? 0.0 : q * (lq - lp);
      } else {
        terms += p == 0.0 ? 0.0 : p * (lp - lq);
      }
    }
    loss = wave_sum(terms);
    if (a.reverse) {
      if (others) loss += qr * (lqr - lpr);
      total = loss + wave_sum(qs) + qr;
      rest = others ? qr * (lqr - lpr + 1.0 - total) : 0.0;
    } else {
      if (others) loss += pr * (lpr - lqr);
      total = list.mass + pr;
      rest = a.rest ? (others ? total * qr - pr : 0.0) : total;
    }
    if (outside) rest /= (double)sums.l;
  }
  if (!list.some || empty) lse = (double)kNegInf;
  // of an empty row too; maxima do not see a NaN, which is no sign of an empty row, and entries of probability 0 no infinity
  if (list.bad || __any(!(x[0] < -kNegInf) || !(x[1] < -kNegInf))) loss = rest = total = lse = (double)__builtin_nanf("");
  *loss_out = (float)loss;
  return DistillStats{x0, outside ? sums.r : 0.f, lse, rest, total};
}

// Gradients of the listed logits in the units of x, for the upstream gradient g, by one wave after teacher_side.
__device__ __forceinline__ void listed_gradients(const DistillArgs& a, const DistillStats& st, float g, List& list) {
  const int lane = threadIdx.x & 63;
  const double s2 = (double)a.s2;
  double base[2], v[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int k = lane + 64 * i;
    const bool there = list.id[k] >= 0;
    const double lq = there ? s2 * ((double)list.x[k] - (double)st.x0) - st.lse : 0.0;
    const double q = there ? (double)exp_of(lq) : 0.0;
    // what the entry adds to its token: forward -p, reverse q (r + 1)
    const double add = a.reverse ? (q == 0.0 ? 0.0 : q * (lq - list.lp[k] + 1.0)) : -(double)list.p[k];
    list.add[k] = (float)add;
    base[i] = a.reverse ? (q == 0.0 ? 0.0 : -q * st.total) : q * st.total;
    v[i] = base[i] + add;
  }
  wave_fence();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int k = lane + 64 * i, id = list.id[k];
    if (list.twice && id >= 0) {   // the entries of one token all come to the same value: any of them may be written last
      v[i] = base[i];
      for (int j = 0; j < a.K; ++j) v[i] += list.id[j] == id ? (double)list.add[j] : 0.0;
    }
    list.value[k] = (float)(v[i] * (s2 * (double)g));
  }
}

// The upstream gradient of a row.
__device__ __forceinline__ float upstream(const DistillArgs& a, int r) {
  float g = a.factor;
  if (a.weight) g *= a.weight[r];
  if (a.dfactor) g *= *a.dfactor;
  return g;
}

}  // namespace streamkl
