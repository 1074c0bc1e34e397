// Log probabilities of given tokens, entropies and top alternatives of rows of
// logits (streamkl_token_logprobs_fwd, streamkl_token_logprobs_bwd).
//
// With z = s x one row, lse = log sum exp z and p = exp(z - lse),
//   logp = z_tok - lse,   H = -sum p log p,   and the `top` largest z - lse.
// Backward, for upstream gradients g (logp), h (H) and e (lse):
//   dx_j = s [ g (j == tok) + p_j (e - g - h (log p_j + H)) ].
//
// Bound: HBM. A logit is read once (twice with a backward pass, and its
// gradient written); forward with entropies 10 vector instructions a logit and 4
// issue slots for the exponential keep the vector unit as busy (8192 x 128000
// bf16: 350 us, 6.0 TB/s, where a kernel that only reads reaches 6.2). A workgroup takes a row, or a part of one where rows are
// few; the parts are joined by a second kernel.
//
// Alternatives. While a row streams by, the maximum of every 16 consecutive
// logits (a group) goes to LDS and every thread keeps its own. The `top`-th
// largest of 256 maxima over disjoint sets of logits is a bound that at least
// `top` logits reach, and few more do; it is found by bisection in one wave.
// Only the groups that reach it are read again, their logits that reach it are
// ranked by counting, each against all. All of it is compared as keys of value
// and place, so that equal logits rank by place and the outcome does not
// depend on the order of arrival. Where too many groups reach the bound (rows
// of equal logits), the `top` groups with the largest keys are found by
// bisection over all groups instead: the alternatives lie in them, since each
// group that a logit's own group ranks behind holds a logit that ranks before
// it. Many candidates (2048 at most) are thinned out by bisection before they
// are ranked. 8192 rows of 128000 bf16, the best 64: noise 386 us (358 without
// alternatives), equal logits 589 us (1731 without thinning out); 16384 rows of
// 2000 zeros, the best one: 242 us (6993).
#include "logit_rows.hpp"
#include "streamkl.h"

namespace streamkl {
namespace {

constexpr int kUnroll = 4;
constexpr int kMostHits = 512, kMostCands = 2048;  // kMostTop groups hold at most kMostCands logits
constexpr int kFewCands = 128;                     // more than `top`, that are ranked against all without thinning out
static_assert(kMostTop * kGroup <= kMostCands && kMostTop <= kMostHits, "");

// The order of logits as numbers: larger for larger values, -0 as 0, 0 for a NaN.
__device__ __forceinline__ u32 key_of(float x) {
  const u32 b = __builtin_bit_cast(u32, x + 0.f);
  return x != x ? 0u : b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float value_of(u32 k) {
  return __builtin_bit_cast(float, k ^ ((k >> 31) ? 0x80000000u : 0xffffffffu));
}
// Value, then place: a larger one ranks first.
__device__ __forceinline__ u64 rank_key(u32 key, u32 place) { return ((u64)key << 32) | (u32)~place; }

template <typename T>
struct TopShared {
  T group[kMostGroups];   // their maxima, which are logits
  u64 cand[kMostCands];
  int hit[kMostHits];
  u32 most[512];     // keys of the threads' maxima
  u64 least[8], last[8];   // of the waves' candidates
  int hits, cands, count[2];
  u32 bound, largest;
};

// The largest t with at least `top` of 256 keys >= t (or one that up to top / 8 more reach), by one wave, and the largest key.
// `most` holds 512 keys or, padded with zeros, fewer.
__device__ __forceinline__ u32 bound_of(const u32* most, int top, u32* largest) {
  const int lane = threadIdx.x;
  u32 k[4], lo = 0xffffffffu, hi = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const u32 a = most[64 * i + lane], b = most[256 + 64 * i + lane];
    k[i] = a > b ? a : b;
    lo = k[i] < lo ? k[i] : lo;
    hi = k[i] > hi ? k[i] : hi;
  }
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const u32 l = (u32)__shfl_xor((int)lo, m), h = (u32)__shfl_xor((int)hi, m);
    lo = l < lo ? l : lo;
    hi = h > hi ? h : hi;
  }
  *largest = hi;
  // all 256 reach lo; kMostTop <= 256
  while (lo < hi) {
    const u32 mid = lo + (hi - lo) / 2 + 1;
    int n = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) n += __popcll(__ballot(k[i] >= mid));
    if (n < top) {
      hi = mid - 1;
    } else {
      lo = mid;
      if (n <= top + top / 8) break;
    }
  }
  return lo;
}

// The sum over the workgroup of what its waves have counted (each all of its lanes the same), in every thread. All threads call
// it; `turn` counts the calls.
template <typename T>
__device__ __forceinline__ int add_up(TopShared<T>& sh, int turn, int wave_count) {
  if (threadIdx.x % 64 == 0) atomicAdd(&sh.count[turn & 1], wave_count);
  __syncthreads();
  const int total = sh.count[turn & 1];
  if (threadIdx.x == 0) sh.count[(turn + 1) & 1] = 0;
  __syncthreads();
  return total;
}

// How many groups satisfy `pred`.
template <typename T, int THREADS, typename P>
__device__ int count_groups(TopShared<T>& sh, int groups, int turn, P pred) {
  int n = 0;
  for (int b = 0; b < groups; b += THREADS) {
    const int g = b + threadIdx.x;
    n += __popcll(__ballot(g < groups && pred(g)));
  }
  return add_up(sh, turn, n);
}

// Leaves the first `top` of many candidates and at most 64 others: each is ranked against all that are left.
template <typename T, int THREADS>
__device__ void thin_out(TopShared<T>& sh, int top) {
  constexpr int EACH = kMostCands / THREADS, W = THREADS / 64;
  static_assert(W <= 8, "");
  const int tid = threadIdx.x, n = sh.cands;
  u64 k[EACH], lo = ~0ull, hi = 0;
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int at = i * THREADS + tid;
    k[i] = at < n ? sh.cand[at] : 0;   // no candidate's
    if (at < n) {
      lo = k[i] < lo ? k[i] : lo;
      hi = k[i] > hi ? k[i] : hi;
    }
  }
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const u64 l = (u64)__shfl_xor((long long)lo, m), h = (u64)__shfl_xor((long long)hi, m);
    lo = l < lo ? l : lo;
    hi = h > hi ? h : hi;
  }
  if (tid % 64 == 0) {
    sh.least[tid / 64] = lo;
    sh.last[tid / 64] = hi;
  }
  if (tid == 0) sh.count[0] = sh.count[1] = 0;
  __syncthreads();
  for (int w = 0; w < W; ++w) {
    lo = sh.least[w] < lo ? sh.least[w] : lo;
    hi = sh.last[w] > hi ? sh.last[w] : hi;
  }
  for (int turn = 0; lo < hi; ++turn) {   // at least `top` reach lo, fewer than that any key above hi
    const u64 mid = lo + (hi - lo) / 2 + 1;
    int c = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) c += __popcll(__ballot(k[i] >= mid));
    c = add_up(sh, turn, c);
    if (c < top) {
      hi = mid - 1;
    } else {
      lo = mid;
      if (c <= top + 64) break;
    }
  }
  if (tid == 0) sh.cands = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < EACH; ++i)
    if (k[i] >= lo) sh.cand[atomicAdd(&sh.cands, 1)] = k[i];
  __syncthreads();
}

// The candidates of a part: keys of all its logits that can be among the `top` first, in sh.cand (sh.cands of them), the
// first `top` among them for sure. group0 is the first group of the part.
template <typename T, int THREADS>
__device__ void find_candidates(TopShared<T>& sh, const Row<T>& row, int group0, int groups, int top) {
  const int tid = threadIdx.x;
  __syncthreads();   // group maxima and thread maxima are written
  if (tid < 64) {
    u32 largest;
    const u32 t = bound_of(sh.most, top, &largest);
    if (tid == 0) {
      sh.bound = t ? t : 1u;   // 0 is for no logit
      sh.largest = largest;
      sh.hits = sh.cands = 0;
      sh.count[0] = sh.count[1] = 0;
    }
  }
  __syncthreads();
  auto gather = [&](u32 bound, auto pred) {
    for (int g = tid; g < groups; g += THREADS) {
      if (pred(g, key_of((float)sh.group[g]))) {
        const int at = atomicAdd(&sh.hits, 1);
        if (at < kMostHits) sh.hit[at] = g;
      }
    }
    __syncthreads();
    const int hits = sh.hits;
    if (hits <= kMostHits) {
      for (int i = tid; i < hits * kGroup; i += THREADS) {
        const int j = (group0 + sh.hit[i / kGroup]) * kGroup + i % kGroup - row.ph;
        if (j >= 0 && j < row.V) {
          const u32 k = key_of((float)row.row[j]);
          if (k >= bound) {
            const int at = atomicAdd(&sh.cands, 1);
            if (at < kMostCands) sh.cand[at] = rank_key(k, (u32)j);
          }
        }
      }
    }
    __syncthreads();
    return hits <= kMostHits && sh.cands <= kMostCands;
  };
  const u32 bound = sh.bound;
  if (gather(bound, [&](int, u32 k) { return k >= bound; })) {
    if (sh.cands > top + kFewCands) thin_out<T, THREADS>(sh, top);
    return;
  }
  // too many reach it: the first `top` groups by key, then by place
  int turn = 0;
  u32 lo = bound, hi = sh.largest > bound ? sh.largest : bound;   // more than `top` groups reach lo
  while (lo < hi) {
    const u32 mid = lo + (hi - lo) / 2 + 1;
    if (count_groups<T, THREADS>(sh, groups, turn++, [&](int g) { return key_of((float)sh.group[g]) >= mid; }) < top)
      hi = mid - 1;
    else
      lo = mid;
  }
  const u32 v = lo;
  const int above = count_groups<T, THREADS>(sh, groups, turn++, [&](int g) { return key_of((float)sh.group[g]) > v; });
  int g0 = 0, g1 = groups - 1;        // the last group of key v that is taken
  while (g0 < g1) {
    const int mid = g0 + (g1 - g0) / 2;
    if (count_groups<T, THREADS>(sh, groups, turn++, [&](int g) { return g <= mid && key_of((float)sh.group[g]) == v; }) <
        top - above)
      g0 = mid + 1;
    else
      g1 = mid;
  }
  if (tid == 0) sh.hits = sh.cands = 0;
  __syncthreads();
  gather(v, [&](int g, u32 k) { return k > v || (k == v && g <= g0); });
  if (sh.cands > top + kFewCands) thin_out<T, THREADS>(sh, top);
}

// Ranks the candidates: f(rank, key) for the first `top`.
template <typename T, int THREADS, typename F>
__device__ __forceinline__ void rank_candidates(const TopShared<T>& sh, int top, F f) {
  const int n = sh.cands < kMostCands ? sh.cands : kMostCands;
  for (int i = threadIdx.x; i < n; i += THREADS) {
    const u64 k = sh.cand[i];
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += sh.cand[j] > k;
    if (rank < top) f(rank, k);
  }
}

// What a row's sums come to. Log probabilities are formed from the distance to the reference: a log-sum-exp near the
// type's lowest value would swallow them.
struct RowEnd {
  double r, log_l, scale;
  bool empty;
  __device__ __forceinline__ RowEnd(const Sums& s, float scale_)
      : r((double)s.r), log_l(log_of((double)s.l)), scale((double)scale_), empty(s.l == 0.f) {}
  __device__ __forceinline__ float logp(float x) const {
    return empty ? kNegInf : (float)(scale * ((double)x - r) - log_l);
  }
};

// A row's token and its logit.
struct Token {
  long long id;
  float x;
  __device__ __forceinline__ Token(const LogprobArgs& a, int r, const void* row) : id(-1), x(0.f) {
    if (!a.logp) return;
    id = a.tokens64 ? static_cast<const long long*>(a.tokens)[r] : static_cast<const int*>(a.tokens)[r];
    if (id < 0 || id >= a.rows.V) return;
    x = a.rows.dtype == STREAMKL_F32   ? static_cast<const float*>(row)[id]
        : a.rows.dtype == STREAMKL_F16 ? (float)static_cast<const _Float16*>(row)[id]
                                       : (float)static_cast<const __bf16*>(row)[id];
  }
};

__device__ __forceinline__ void finish_row(const LogprobArgs& a, int r, const Sums& sums, const RowEnd& end,
                                           const Token& token) {
  const double base = end.scale * end.r;   // exact
  const float lse = end.empty ? kNegInf : (float)(base + end.log_l);
  if (a.lse) a.lse[r] = lse;
  if (a.lse_err) a.lse_err[r] = end.empty ? 0.f : (float)((base - (double)lse) + end.log_l);
  // in units of log 2: log2 l - a / l
  if (a.entropy)
    a.entropy[r] = end.empty ? 0.f : (float)(end.log_l - 0.69314718055994530942 * ((double)sums.a / (double)sums.l));
  if (a.logp) a.logp[r] = token.id < 0 ? 0.f : token.id >= a.rows.V ? __builtin_nanf("") : end.logp(token.x);
}

__device__ __forceinline__ void write_top(const LogprobArgs& a, int r, int rank, u64 k, const RowEnd& end) {
  const long long at = (long long)r * a.top + rank;
  a.top_ids[at] = (int)~(u32)k;
  a.top_logp[at] = end.logp(value_of((u32)(k >> 32)));
}

// Places of a row's list that no logit took (it holds a NaN).
__device__ __forceinline__ void write_none(const LogprobArgs& a, int r, int rank) {
  const long long at = (long long)r * a.top + rank;
  a.top_ids[at] = -1;
  a.top_logp[at] = __builtin_nanf("");
}

struct NoShared {};

template <typename T, int THREADS, bool ENTROPY, bool TOP>
__global__ void __launch_bounds__(THREADS, 8)
logprob_kernel(LogprobArgs a) {
  __shared__ float red[3 * THREADS / 64];
  __shared__ std::conditional_t<TOP, TopShared<T>, NoShared> sh;
  int r, s;
  if (!grid_place((long long)a.rows.B * a.rows.N, a.plan.parts, &r, &s)) return;
  const Row<T> row(a.rows, r);
  const int c0 = s * a.plan.chunks, c1 = min(row.chunks, c0 + a.plan.chunks), tid = threadIdx.x;
  const float c = a.scale * kLog2e, rise = kRise / c;
  Sums sums;
  float most = kNegInf;
  each_turn<T, THREADS, kUnroll, true>(row, c0, c1, [&](int at, const auto& turn) {
    constexpr int N = std::decay_t<decltype(turn)>::N;
    float f[N][kEpc<T>], mx[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      unpack<T>(turn.raw[j], f[j]);
      mx[j] = max_of<T>(f[j]);
    }
    const float mm = max_all(mx);
    if constexpr (TOP) {
      most = vmax(most, mm);
      constexpr int CPG = kGroup / kEpc<T>;   // lanes that share a group
#pragma unroll
      for (int j = 0; j < N; ++j) {
        float g = vmax_xor1(mx[j]);
        if constexpr (CPG == 4) g = vmax_xor2(g);
        const int ch = at + j * THREADS;
        if (ch < c1 && tid % CPG == 0) sh.group[(ch - c0) / CPG] = (T)g;
      }
    }
    sums.expect(mm, c, rise);
    sums.template add<ENTROPY>(f, c);
  });
  if constexpr (TOP) {
    for (int i = tid; i < 512; i += THREADS) sh.most[i] = i == tid ? key_of(most) : 0u;
  }
  sums = block_join<THREADS>(sums, c, red);
  const RowEnd end(sums, a.scale);
  const int top = a.top;
  if constexpr (TOP) {
    constexpr int CPG = kGroup / kEpc<T>;
    find_candidates<T, THREADS>(sh, row, c0 / CPG, (c1 - c0 + CPG - 1) / CPG, top);
  }
  if (a.plan.parts == 1) {
    if (tid == 0) finish_row(a, r, sums, end, Token(a, r, row.row));
    if constexpr (TOP) {
      for (int i = sh.cands + tid; i < top; i += THREADS) write_none(a, r, i);
      rank_candidates<T, THREADS>(sh, top, [&](int rank, u64 k) { write_top(a, r, rank, k, end); });
    }
  } else {
    const long long i = (long long)r * a.plan.parts + s;
    if (tid == 0) static_cast<LogprobPart*>(a.workspace)[i] = LogprobPart{sums.r, sums.l, sums.a};
    if constexpr (TOP) {
      u64* keys = reinterpret_cast<u64*>(static_cast<char*>(a.workspace) +
                                         logprob_part_bytes((long long)a.rows.B * a.rows.N, a.plan)) + i * top;
      for (int q = sh.cands + tid; q < top; q += THREADS) keys[q] = 0;   // ranks behind any logit
      rank_candidates<T, THREADS>(sh, top, [&](int rank, u64 k) { keys[rank] = k; });
    }
  }
}

// Joins the parts of a row. Sums by one lane a part. Every part has sorted keys, `per` of them at or before its per-th, so
// that `top` keys rank at or before the last of these: only keys up to there are looked at, and each is ranked against all
// others of them (or, where they are many, among the sorted lists). Everything is on its way before anything is waited for:
// the kernel is latency (16 rows of 16 parts, 20 alternatives: 18 us with the bound by one thread and a search in every
// list, 6 us so).
constexpr int kJoinThreads = 256, kJoinCands = 512;

__global__ void __launch_bounds__(kJoinThreads)
logprob_join_kernel(LogprobArgs a) {
  extern __shared__ u64 keys[];   // [parts][top]
  __shared__ u64 cand[kJoinCands];
  __shared__ u64 bound;
  __shared__ float joined[2];
  __shared__ int cands;
  int r, s;
  if (!grid_place((long long)a.rows.B * a.rows.N, 1, &r, &s)) return;
  const int tid = threadIdx.x, parts = a.plan.parts, top = a.top, n = parts * top;
  const float c = a.scale * kLog2e;
  const u64* const from =
      reinterpret_cast<const u64*>(static_cast<const char*>(a.workspace) +
                                   logprob_part_bytes((long long)a.rows.B * a.rows.N, a.plan)) +
      (long long)r * n;
  if (tid < 64) {
    const int b = r / a.rows.N;
    const long long at = b * a.rows.sb + (r - b * a.rows.N) * a.rows.sn;
    Sums sums;
    u64 least = ~0ull;
    if (tid < parts) {
      const LogprobPart p = static_cast<const LogprobPart*>(a.workspace)[(long long)r * parts + tid];
      sums.r = p.r;
      sums.l = p.l;
      sums.a = p.a;
      if (top) least = from[tid * top + (top + parts - 1) / parts - 1];
    }
    const Token token(a, r, static_cast<const char*>(a.rows.x) + at * (a.rows.dtype == STREAMKL_F32 ? 4 : 2));
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
      const u64 o = (u64)__shfl_xor((long long)least, m);
      least = o < least ? o : least;
    }
    sums = lanes_join<64>(sums, c);
    if (tid == 0) {
      joined[0] = sums.r;
      joined[1] = sums.l;
      bound = least ? least : 1;
      cands = 0;
      finish_row(a, r, sums, RowEnd(sums, a.scale), token);
    }
  }
  if (top == 0) return;
  for (int i = tid; i < n; i += kJoinThreads) keys[i] = from[i];
  for (int i = tid; i < top; i += kJoinThreads) write_none(a, r, i);
  __syncthreads();
  const u64 first = bound;
  for (int i = tid; i < n; i += kJoinThreads) {
    if (keys[i] >= first) {
      const int at = atomicAdd(&cands, 1);
      if (at < kJoinCands) cand[at] = keys[i];
    }
  }
  __syncthreads();
  Sums sums;
  sums.r = joined[0];
  sums.l = joined[1];
  const RowEnd end(sums, a.scale);
  if (cands <= kJoinCands) {
    const int m = cands;
    for (int i = tid; i < m; i += kJoinThreads) {
      const u64 k = cand[i];
      int rank = 0;
      for (int j = 0; j < m; ++j) rank += cand[j] > k;
      if (rank < top) write_top(a, r, rank, k, end);
    }
    return;
  }
  for (int i = tid; i < n; i += kJoinThreads) {
    const u64 k = keys[i];
    if (k < first) continue;
    int rank = 0;
    for (int p = 0; p < parts && rank < top; ++p) {
      int lo = 0, hi = top;   // keys of part p that rank before k
      while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (keys[p * top + mid] > k)
          lo = mid + 1;
        else
          hi = mid;
      }
      rank += lo;
    }
    if (rank < top) write_top(a, r, rank, k, end);
  }
}

// A row's sums (no entropy), in every thread.
template <typename T, int THREADS>
__device__ __forceinline__ Sums row_sums(const Row<T>& row, float c, float* red) {
  const float rise = kRise / c;
  Sums sums;
  each_turn<T, THREADS, kUnroll, false>(row, 0, row.chunks, [&](int, const auto& turn) {
    constexpr int N = std::decay_t<decltype(turn)>::N;
    float f[N][kEpc<T>], mx[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      unpack<T>(turn.raw[j], f[j]);
      mx[j] = max_of<T>(f[j]);
    }
    sums.expect(max_all(mx), c, rise);
    sums.template add<false>(f, c);
  });
  return block_join<THREADS>(sums, c, red);
}

// dx of a part of a row. A log-sum-exp is what the forward call handed over: its float32 value and what that rounding left
// off. From kFarLse on the latter is as large as log l itself or larger, and further out it swallows log l whole, while the
// place of the row's logits cannot be told from lse / scale any more: the sums of such a row are formed again.
constexpr float kFarLse = 0x1p24f;

template <typename T, int THREADS>
__global__ void __launch_bounds__(THREADS, 8)
logprob_grad_kernel(LogprobGradArgs a) {
  __shared__ float red[3 * THREADS / 64];
  int r, s;
  if (!grid_place((long long)a.rows.B * a.rows.N, a.plan.parts, &r, &s)) return;
  r = a.rows.B * a.rows.N - 1 - r;   // the last rows first: the forward pass left them in the cache
  const Row<T> row(a.rows, r);
  int c0 = s * a.plan.chunks, c1 = min(row.chunks, c0 + a.plan.chunks);
  const int b = r / a.rows.N;
  T* const dx = static_cast<T*>(a.dx) + b * a.dsb + (r - b * a.rows.N) * a.dsn;
  long long tok = -1;
  if (a.tokens)
    tok = a.tokens64 ? static_cast<const long long*>(a.tokens)[r] : static_cast<const int*>(a.tokens)[r];
  const float g = a.dlogp && tok >= 0 ? a.dlogp[r] : 0.f;
  const float h = a.dentropy ? a.dentropy[r] : 0.f, e = a.dlse ? a.dlse[r] : 0.f;
  const float lse = a.lse[r], c = a.scale * kLog2e;
  const bool none = (g == 0.f && h == 0.f && e == 0.f) || lse == kNegInf;
  if (none) {
    float z[kEpc<T>] = {};
    for (int ch = c0 + threadIdx.x; ch < c1; ch += THREADS) store<T>(row, dx, ch, z);
    return;
  }
  float at, f, log_f;   // p_j = 2^u_j f, u_j = (x_j - at) c
  if (__builtin_fabsf(lse) < kFarLse) {
    const Exponent x(lse, a.lse_err ? a.lse_err[r] : 0.f, a.scale);
    at = x.at;
    f = x.f;
    log_f = logf(f);
  } else {   // by the first workgroup alone, the others would write what it reads where dx is x
    if (s != 0) return;
    c0 = 0;
    c1 = row.chunks;
    const Sums sums = row_sums<T, THREADS>(row, c, red);
    at = sums.r;
    f = 1.f / sums.l;
    log_f = -logf(sums.l);
  }
  // dx_j = p_j (p1 + p2 u_j) + (j == tok) hit
  const float H = h == 0.f ? 0.f : a.entropy[r];
  float p1 = a.scale * f * (e - g - h * (H + log_f));
  const float p2 = -a.scale * f * h * kLn2, hit = a.scale * g;
  if (tok >= row.V && g != 0.f) p1 = __builtin_nanf("");   // entropy and log-sum-exp do not depend on the token
  const int tok_at = tok >= 0 && tok < row.V ? (int)tok + row.ph : -1;
  const int tok_chunk = tok_at >= 0 ? tok_at / kEpc<T> : -1;
  each_turn<T, THREADS, kUnroll, false>(row, c0, c1, [&](int first, const auto& turn) {
#pragma unroll
    for (int j = 0; j < std::decay_t<decltype(turn)>::N; ++j) {
      const int ch = first + j * THREADS;
      float d[kEpc<T>];
      unpack<T>(turn.raw[j], d);
#pragma unroll
      for (int i = 0; i < kEpc<T>; ++i) {
        float u = (d[i] - at) * c;
        u = u < kFloor ? kFloor : u;
        d[i] = exp2_fast(u) * __builtin_fmaf(p2, u, p1);
      }
      if (ch == tok_chunk) {
#pragma unroll
        for (int i = 0; i < kEpc<T>; ++i) d[i] += i == tok_at % kEpc<T> ? hit : 0.f;
      }
      if (ch < c1) store<T>(row, dx, ch, d);
    }
  });
}

// ---------------------------------------------------------------------------
// Launches
// ---------------------------------------------------------------------------

template <int THREADS, typename T>
void run_fwd(const LogprobArgs& a, dim3 grid) {
  if (a.top > 0) {
    if (a.entropy)
      logprob_kernel<T, THREADS, true, true><<<grid, dim3(THREADS), 0, a.stream>>>(a);
    else
      logprob_kernel<T, THREADS, false, true><<<grid, dim3(THREADS), 0, a.stream>>>(a);
  } else if (a.entropy) {
    logprob_kernel<T, THREADS, true, false><<<grid, dim3(THREADS), 0, a.stream>>>(a);
  } else {
    logprob_kernel<T, THREADS, false, false><<<grid, dim3(THREADS), 0, a.stream>>>(a);
  }
}

}  // namespace

hipError_t launch_logprob(const LogprobArgs& a) {
  const long long rows = (long long)a.rows.B * a.rows.N;
  const dim3 grid = logit_grid(rows * a.plan.parts);
  by_type(a.rows.dtype, [&](auto t) {
    if (a.plan.threads == 256)
      run_fwd<256, decltype(t)>(a, grid);
    else
      run_fwd<512, decltype(t)>(a, grid);
  });
  if (a.plan.parts > 1)
    logprob_join_kernel<<<logit_grid(rows), dim3(kJoinThreads), a.plan.parts * a.top * sizeof(u64), a.stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_logprob_grad(const LogprobGradArgs& a) {
  const dim3 grid = logit_grid((long long)a.rows.B * a.rows.N * a.plan.parts);
  by_type(a.rows.dtype, [&](auto t) {
    logprob_grad_kernel<decltype(t), 256><<<grid, dim3(256), 0, a.stream>>>(a);
  });
  return hipGetLastError();
}

}  // namespace streamkl
