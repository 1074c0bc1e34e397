// Instantiations of the differential-attention backward, the kernel that
// prepares the row statistics and the one that sums dlam.
#include "diff_bwd.hpp"
#include "diff_launch.hpp"

namespace streamkl {

namespace {

// One wave per 32-row tile of a head: D_1 = dO . (O + lam O_2) and
// D_2 = dO . O_2 of its rows, 8 columns a lane, then the statistics in the
// form the kernels use (diff_bwd.hpp). Bound by reading dO, O and O_2 once.
__global__ void __launch_bounds__(kThreads) diff_bwd_prep_kernel(const DiffArgs a, const uint16_t* __restrict__ o,
                                                                 const uint16_t* __restrict__ o2, long long tiles,
                                                                 int ntq, int tpr) {
  const int lane = threadIdx.x & 63;
  const long long tile = (long long)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
  if (tile >= tiles) return;
  const long long bh = tile / ntq;
  const int row0 = (int)(tile - bh * ntq) * kDiffTile, b = (int)(bh / a.H), h = (int)(bh - (long long)b * a.H);
  const int qlen = clamp_len(a.q_len, b, a.NQ);
  const float lam = a.lam[h], l2lam = __builtin_amdgcn_logf(fabsf(lam) < 0x1p-126f ? fabsf(lam) * 0x1p64f : fabsf(lam)) -
                                      (fabsf(lam) < 0x1p-126f ? 64.f : 0.f);   // -inf at 0
  float* st = a.stats + tile * kDiffStatsTile;
  const int c = lane & (tpr - 1), rpw = 64 / tpr;
  for (int r = lane / tpr; r < kDiffTile; r += rpw) {
    const int row = row0 + r;
    const bool ok = row < qlen;
    float s1 = 0.f, s2 = 0.f;
    if (ok && 8 * c < a.dv) {
      const long long at = (bh * a.NQ + row) * a.dv + 8 * c;
      const bf16x8 g = *reinterpret_cast<const bf16x8*>(a.dout + at), x = *reinterpret_cast<const bf16x8*>(o + at);
      const bf16x8 y = *reinterpret_cast<const bf16x8*>(o2 + at);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        s1 = __builtin_fmaf((float)g[e], (float)x[e], s1);
        s2 = __builtin_fmaf((float)g[e], (float)y[e], s2);
      }
    }
    for (int m = 1; m < tpr; m <<= 1) {
      s1 += __shfl_xor(s1, m);
      s2 += __shfl_xor(s2, m);
    }
    if (c == 0) {
      float e1 = kNegInf, e2 = kNegInf;
      if (ok) {
        e1 = a.lse1[bh * a.NQ + row];
        e2 = a.lse2[bh * a.NQ + row];
      }
      const bool none = e1 == kNegInf || e2 == kNegInf;   // sees nothing: P = 0, and no NaN from its sums
      st[r] = none ? __builtin_inff() : e1 * kLog2e;
      st[kDiffTile + r] = none ? __builtin_inff() : e2 * kLog2e - l2lam;
      st[2 * kDiffTile + r] = none ? 0.f : __builtin_fmaf(lam, s2, s1);
      st[3 * kDiffTile + r] = none ? 0.f : lam < 0.f ? -s2 : s2;
    }
  }
}

// dlam_h = -sum of its blocks' partial sums, one workgroup per head.
__global__ void __launch_bounds__(kThreads) diff_bwd_dlam_kernel(const DiffArgs a, int T) {
  __shared__ float red[kThreads / 64];
  const int h = blockIdx.x, tid = threadIdx.x;
  float s = 0.f;
  for (int i = tid; i < a.B * T; i += kThreads) {
    const int b = i / T;
    s += a.dlam_part[((long long)b * a.H + h) * T + (i - b * T)];
  }
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) s += __shfl_xor(s, m);
  if ((tid & 63) == 0) red[tid >> 6] = s;
  __syncthreads();
  if (tid == 0) a.dlam[h] = -((red[0] + red[1]) + (red[2] + red[3]));
}

int row_blocks(int NQ) { return (NQ + DiffBwdCfg<64, 64>::ROWS - 1) / DiffBwdCfg<64, 64>::ROWS; }

template <typename F>
hipError_t by_dims(int d, int dv, F f) {
  auto by_dv = [&](auto kd) {
    switch (diff_value_dim(dv)) {
      case 64: return f(kd, std::integral_constant<int, 64>{});
      case 128: return f(kd, std::integral_constant<int, 128>{});
      default: return f(kd, std::integral_constant<int, 256>{});
    }
  };
  return diff_key_dim(d) == 64 ? by_dv(std::integral_constant<int, 64>{}) : by_dv(std::integral_constant<int, 128>{});
}

}  // namespace

size_t diff_bwd_stats_floats(int B, int H, int NQ) {
  return (size_t)B * H * ((NQ + kDiffTile - 1) / kDiffTile) * kDiffStatsTile;
}

size_t diff_bwd_dlam_floats(int B, int H, int NQ) { return (size_t)B * H * row_blocks(NQ); }

hipError_t launch_diff_bwd_prep(const DiffArgs& a) {
  const int ntq = (a.NQ + kDiffTile - 1) / kDiffTile;
  const long long tiles = (long long)a.B * a.H * ntq;
  const int chunks = a.dv / 8, tpr = chunks <= 4 ? 4 : chunks <= 8 ? 8 : chunks <= 16 ? 16 : 32;
  hipLaunchKernelGGL(diff_bwd_prep_kernel, dim3((unsigned)((tiles + 3) / 4)), dim3(kThreads), 0, a.stream, a, a.out,
                     a.out2, tiles, ntq, tpr);
  return hipGetLastError();
}

hipError_t launch_diff_bwd_dq(const DiffArgs& a) {
  return by_dims(a.d, a.dv, [&](auto kd, auto kv) {
    hipLaunchKernelGGL((diff_bwd_dq_kernel<kd.value, kv.value>),
                       dim3((unsigned)((long long)a.B * a.H * row_blocks(a.NQ))), dim3(kThreads), 0, a.stream, a);
    return hipGetLastError();
  });
}

hipError_t launch_diff_bwd_dkv(const DiffArgs& a) {
  return by_dims(a.d, a.dv, [&](auto kd, auto kv) {
    hipLaunchKernelGGL((diff_bwd_dkv_kernel<kd.value, kv.value>),
                       dim3((unsigned)((long long)a.B * a.HK * row_blocks(a.NK))), dim3(kThreads), 0, a.stream, a);
    return hipGetLastError();
  });
}

hipError_t launch_diff_bwd_dlam(const DiffArgs& a) {
  hipLaunchKernelGGL(diff_bwd_dlam_kernel, dim3((unsigned)a.H), dim3(kThreads), 0, a.stream, a, row_blocks(a.NQ));
  return hipGetLastError();
}

}  // namespace streamkl
