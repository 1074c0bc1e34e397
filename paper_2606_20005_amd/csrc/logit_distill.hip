// Divergence of a student's rows of logits from a teacher's best tokens
// (streamkl_topk_distill_fwd, streamkl_topk_distill_bwd); logit_distill.hpp has
// the mathematics. A logit is read once forward; the backward pass reads it
// again and writes its gradient. A workgroup takes a row, or a part of one
// where rows are few (forward; the parts are joined by a second kernel) or
// long (backward).
#include "logit_distill.hpp"

namespace streamkl {
namespace {

constexpr int kUnroll = 4;

template <typename T, int THREADS, bool REST>
__global__ void __launch_bounds__(THREADS, 8)
distill_kernel(DistillArgs a) {
  __shared__ float red[3 * THREADS / 64];
  __shared__ List list;
  extern __shared__ u32 marks[];   // REST: a byte per chunk of the part, a bit per listed logit
  int r, s;
  if (!grid_place((long long)a.rows.B * a.rows.N, a.plan.parts, &r, &s)) return;
  const Row<T> row(a.rows, r);
  const int c0 = s * a.plan.chunks, c1 = min(row.chunks, c0 + a.plan.chunks), tid = threadIdx.x;
  const float c = a.s2 * kLog2e, rise = kRise / c;
  if (tid == 0) list.some = list.bad = list.twice = 0;
  if constexpr (REST)
    for (int i = tid; 4 * i < a.plan.chunks; i += THREADS) marks[i] = 0;
  __syncthreads();
  read_list<T, THREADS>(a, r, row.row, list, [&](int, int id) {
    const int at = id + row.ph, ch = at / kEpc<T> - c0;
    if (REST && ch >= 0 && ch < c1 - c0) atomicOr(&marks[ch / 4], 1u << (8 * (ch % 4) + at % kEpc<T>));
  });
  __syncthreads();
  Sums sums;
  if (list.some) {   // a row without a list has no loss, whatever its logits
    const unsigned char* const mark = reinterpret_cast<const unsigned char*>(marks);
    each_turn<T, THREADS, kUnroll, true>(row, c0, c1, [&](int at, const auto& turn) {
      constexpr int N = std::decay_t<decltype(turn)>::N;
      float f[N][kEpc<T>], mx[N];
#pragma unroll
      for (int j = 0; j < N; ++j) {
        unpack<T>(turn.raw[j], f[j]);
        if constexpr (REST) {
          const int ch = at + j * THREADS;
          leave_out(f[j], ch < c1 ? mark[ch - c0] : 0u);
        }
        mx[j] = max_of<T>(f[j]);
      }
      sums.expect(max_all(mx), c, rise);
      sums.template add<false>(f, c);
    });
  }
  if (a.plan.parts == 1 && tid < 64) teacher_side(a, list);
  sums = block_join<THREADS>(sums, c, red);
  if (a.plan.parts == 1) {
    if (tid < 64) {
      float loss;
      const DistillStats st = finish_row(a, sums, list, &loss);
      if (tid == 0) {
        a.loss[r] = loss;
        a.stats[r] = st;
      }
    }
  } else if (tid == 0) {
    static_cast<DistillPart*>(a.workspace)[(long long)r * a.plan.parts + s] = DistillPart{sums.r, sums.l};
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
  if (threadIdx.x == 0) list.some = list.bad = list.twice = 0;
  __syncthreads();
  Sums sums;
  if ((int)threadIdx.x < a.plan.parts) {
    const DistillPart p = static_cast<const DistillPart*>(a.workspace)[(long long)r * a.plan.parts + threadIdx.x];
    sums.r = p.r;
    sums.l = p.l;
  }
  read_list<T, 64>(a, r, row.row, list, [](int, int) {});
  __syncthreads();
  teacher_side(a, list);
  __syncthreads();
  sums = lanes_join<64>(sums, a.s2 * kLog2e);
  float loss;
  const DistillStats st = finish_row(a, sums, list, &loss);
  if (threadIdx.x == 0) {
    a.loss[r] = loss;
    a.stats[r] = st;
  }
}

// dx of a part of a row.
template <typename T, int THREADS>
__device__ __forceinline__ void part_gradients(const DistillArgs& a, int r, int s, List& list) {
  r = a.rows.B * a.rows.N - 1 - r;   // the last rows first: the forward pass left them in the cache
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
  __syncthreads();   // the list of the part before is done with
  // dx may be x: the listed logits of a part are read before it writes, those of other parts are read but not used
  if (tid == 0) list.some = list.bad = list.twice = 0;
  __syncthreads();
  read_list<T, THREADS>(a, r, row.row, list, [](int, int) {});
  __syncthreads();
  if (tid < 64) {
    teacher_side(a, list);
    wave_fence();
    listed_gradients(a, st, g, list);
  }
  const float c = a.s2 * kLog2e, at = st.r, w = (float)((double)a.s2 * (double)g * st.rest);
  each_turn<T, THREADS, kUnroll, false>(row, c0, c1, [&](int first, const auto& turn) {
#pragma unroll
    for (int j = 0; j < std::decay_t<decltype(turn)>::N; ++j) {
      const int ch = first + j * THREADS;
      float f[kEpc<T>];
      unpack<T>(turn.raw[j], f);
#pragma unroll
      for (int i = 0; i < kEpc<T>; ++i) f[i] = exp2_fast((f[i] - at) * c) * w;
      if (ch < c1) store<T>(row, dx, ch, f);
    }
  });
  __syncthreads();
  for (int k = tid; k < a.K; k += THREADS) {
    const int id = list.id[k], ch = id < 0 ? -1 : (id + row.ph) / kEpc<T>;
    if (ch >= c0 && ch < c1) dx[id] = (T)list.value[k];
  }
}

// One part a workgroup; FEW, where there may be nothing to do: few workgroups that take several (65536 that only look at the
// factor took 15 us).
constexpr int kFewWorkgroups = 2048;

template <typename T, int THREADS, bool FEW>
__global__ void __launch_bounds__(THREADS, FEW ? 4 : 8)
distill_grad_kernel(DistillArgs a) {
  __shared__ List list;
  int r, s;
  if constexpr (!FEW) {
    if (grid_place((long long)a.rows.B * a.rows.N, a.plan.parts, &r, &s)) part_gradients<T, THREADS>(a, r, s, list);
  } else {
    if (*a.dfactor == 1.f) return;
    const long long n = (long long)a.rows.B * a.rows.N * a.plan.parts;
    for (long long i = blockIdx.x; i < n; i += gridDim.x)
      part_gradients<T, THREADS>(a, (int)(i / a.plan.parts), (int)(i % a.plan.parts), list);
  }
}

// total = sum of weight factor loss over the rows whose weight is not 0, by one workgroup.
constexpr int kSumThreads = 1024;

__global__ void __launch_bounds__(kSumThreads)
weighted_sum_kernel(const float* loss, const float* weight, float factor, long long rows, float* total) {
  __shared__ double red[kSumThreads / 64];
  // eight loads of each in flight
  constexpr int ahead = 8;
  double v = 0.0;
  for (long long i = threadIdx.x; i < rows; i += ahead * kSumThreads) {
    float w[ahead], l[ahead];
#pragma unroll
    for (int u = 0; u < ahead; ++u) {
      const long long at = i + u * kSumThreads;
      w[u] = at < rows ? (weight ? weight[at] : 1.f) : 0.f;
      l[u] = at < rows ? loss[at] : 0.f;
    }
#pragma unroll
    for (int u = 0; u < ahead; ++u) v += w[u] == 0.f ? 0.0 : (double)w[u] * (double)l[u];
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

hipError_t launch_distill_grad(const DistillArgs& a) {
  const long long n = (long long)a.rows.B * a.rows.N * a.plan.parts;
  by_type(a.rows.dtype, [&](auto t) {
    if (a.done_if_one)
      distill_grad_kernel<decltype(t), 256, true>
          <<<dim3((unsigned)(n < kFewWorkgroups ? n : kFewWorkgroups)), dim3(256), 0, a.stream>>>(a);
    else
      distill_grad_kernel<decltype(t), 256, false><<<logit_grid(n), dim3(256), 0, a.stream>>>(a);
  });
  return hipGetLastError();
}

hipError_t launch_weighted_sum(const float* loss, const float* weight, float factor, long long rows, float* total,
                               hipStream_t stream) {
  weighted_sum_kernel<<<dim3(1), dim3(kSumThreads), 0, stream>>>(loss, weight, factor, rows, total);
  return hipGetLastError();
}

}  // namespace streamkl
