// The kernels that join the partials of the split differential-attention forward.
#include "diff_launch.hpp"

namespace streamkl {

namespace {

constexpr int kFewSplits = 8;

__device__ __forceinline__ float inverse_sum(float l) { return l > 0.f || l != l ? 1.f / l : 0.f; }

// Writes four columns of an output row from its joined maps.
__device__ __forceinline__ void write_joined(const DiffArgs& a, long long row, int col4, bool ok, f32x4 o1, float f1,
                                             f32x4 o2, float f2, float lam) {
  bf16x4 r, r2;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float v2 = ok ? o2[j] * f2 : 0.f;
    r2[j] = (__bf16)v2;
    r[j] = (__bf16)(ok ? __builtin_fmaf(-lam, v2, o1[j] * f1) : 0.f);
  }
  *reinterpret_cast<bf16x4*>(a.out + row * a.dv + 4 * col4) = r;
  if (a.out2) *reinterpret_cast<bf16x4*>(a.out2 + row * a.dv + 4 * col4) = r2;
}

// Joins the partials of output rows (see diff_fwd.hpp) where there are few of
// each: one wave per row, four columns a lane. (One workgroup per row took 80
// us for 48056 rows of two partials, of which their bytes are 44.)
__global__ void __launch_bounds__(kThreads) diff_merge_few_kernel(const DiffArgs a) {
  const int lane = threadIdx.x & 63;
  const long long rows = (long long)a.B * a.H * a.NQ;
  const long long row = (long long)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
  if (row >= rows) return;
  const int bh = (int)(row / a.NQ), i = (int)(row - (long long)bh * a.NQ), b = bh / a.H, h = bh - b * a.H;
  const bool ok = i < clamp_len(a.q_len, b, a.NQ);
  const int S = a.splits, cols = a.dv / 4;
  const float* po = a.part + row * S * 2 * a.dv;
  const float* pm = a.part + rows * S * 2 * a.dv + row * S * 4;
  float ref[2][kFewSplits], top[2] = {kNegInf, kNegInf}, sum[2] = {0.f, 0.f};
  f32x4 o[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
  if (ok) {
#pragma unroll
    for (int s = 0; s < kFewSplits; ++s) {
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        ref[m][s] = s < S ? pm[(s * 2 + m) * 2] : kNegInf;
        top[m] = fmaxf(top[m], ref[m][s]);
      }
    }
#pragma unroll
    for (int s = 0; s < kFewSplits; ++s) {
      if (s < S) {
#pragma unroll
        for (int m = 0; m < 2; ++m) {
          const float f = ref[m][s] == kNegInf ? 0.f : exp2_fast(ref[m][s] - top[m]);
          sum[m] = __builtin_fmaf(f, pm[(s * 2 + m) * 2 + 1], sum[m]);
          if (lane < cols) o[m] += reinterpret_cast<const f32x4*>(po + (s * 2 + m) * a.dv)[lane] * f;
        }
      }
    }
  }
  if (lane < cols) write_joined(a, row, lane, ok, o[0], inverse_sum(sum[0]), o[1], inverse_sum(sum[1]), a.lam[h]);
  if (lane < 2) {
    float* lse = lane ? a.lse2 : a.lse1;
    const float t = lane ? top[1] : top[0], l = lane ? sum[1] : sum[0];
    if (lse) lse[row] = !ok || l == 0.f ? kNegInf : diff_lse(l, t);
  }
}

// The same for many partials of few rows: one workgroup per row, whose groups
// of lanes share the splits.
__global__ void __launch_bounds__(kThreads) diff_merge_kernel(const DiffArgs a) {
  __shared__ float w[2][kDiffMaxSplits];
  __shared__ float top[2], total[2];
  __shared__ f32x4 acc[2][kThreads];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const long long row = blockIdx.x;
  const int bh = (int)(row / a.NQ), i = (int)(row - (long long)bh * a.NQ), b = bh / a.H, h = bh - b * a.H;
  const bool ok = i < clamp_len(a.q_len, b, a.NQ);
  const int S = a.splits, cols = a.dv / 4;   // 8 to 64, a multiple of 8
  const long long rows = (long long)a.B * a.H * a.NQ;
  const float* po = a.part + row * S * 2 * a.dv;
  const float* pm = a.part + rows * S * 2 * a.dv + row * S * 4;
  if (wave < 2) {   // wave m: the joint reference and sum of map m
    float t = kNegInf;
    if (ok)
      for (int s = lane; s < S; s += 64) t = fmaxf(t, pm[(s * 2 + wave) * 2]);
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) t = fmaxf(t, __shfl_xor(t, x));
    float sum = 0.f;
    for (int s = lane; s < S; s += 64) {
      float f = 0.f;
      if (ok) {
        const float r = pm[(s * 2 + wave) * 2];
        f = r == kNegInf ? 0.f : exp2_fast(r - t);
        sum = __builtin_fmaf(f, pm[(s * 2 + wave) * 2 + 1], sum);
      }
      w[wave][s] = f;
    }
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) sum += __shfl_xor(sum, x);
    if (lane == 0) {
      top[wave] = t;
      total[wave] = sum;
    }
  }
  __syncthreads();
  const int groups = kThreads / cols, grp = tid / cols, col = tid - grp * cols;
  f32x4 o1 = {0.f, 0.f, 0.f, 0.f}, o2 = o1;
  if (ok && grp < groups) {
    for (int s = grp; s < S; s += groups) {
      const f32x4* p = reinterpret_cast<const f32x4*>(po + (long long)s * 2 * a.dv);
      o1 += p[col] * w[0][s];
      o2 += p[cols + col] * w[1][s];
    }
  }
  acc[0][tid] = o1;
  acc[1][tid] = o2;
  __syncthreads();
  if (tid < cols) {
    for (int g = 1; g < groups; ++g) {
      o1 += acc[0][g * cols + tid];
      o2 += acc[1][g * cols + tid];
    }
    write_joined(a, row, tid, ok, o1, inverse_sum(total[0]), o2, inverse_sum(total[1]), a.lam[h]);
  }
  if (tid < 2) {
    float* lse = tid ? a.lse2 : a.lse1;
    if (lse) lse[row] = !ok || total[tid] == 0.f ? kNegInf : diff_lse(total[tid], top[tid]);
  }
}

}  // namespace

hipError_t launch_diff_merge(const DiffArgs& a) {
  const long long rows = (long long)a.B * a.H * a.NQ;
  if (a.splits <= kFewSplits && rows >= 8 * kCus)   // fewer waves than that would not hide a walk over the partials
    hipLaunchKernelGGL(diff_merge_few_kernel, dim3((unsigned)((rows + kThreads / 64 - 1) / (kThreads / 64))),
                       dim3(kThreads), 0, a.stream, a);
  else
    hipLaunchKernelGGL(diff_merge_kernel, dim3((unsigned)rows), dim3(kThreads), 0, a.stream, a);
  return hipGetLastError();
}

}  // namespace streamkl
