// The small kernels of the differential-attention backward: row statistics,
// the sum of dlam, the sum of partial gradients.
#include "diff_bwd.hpp"
#include "diff_launch.hpp"

namespace streamkl {

namespace {

// One workgroup per 32-row tile of a head: D_1 = dO . (O + lam O_2) and
// D_2 = dO . O_2 of its rows, 8 columns a lane, then the statistics in the
// form the kernels use (diff_bwd.hpp). Bound by reading dO, O and O_2 once (32
// heads x 4096, dv 128: 100 MB in 21 us; with one wave a tile short grids took
// three times as long).
__global__ void __launch_bounds__(kThreads) diff_bwd_prep_kernel(const DiffArgs a, const uint16_t* __restrict__ o,
                                                                 const uint16_t* __restrict__ o2, int ntq, int tpr) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const long long tile = blockIdx.x;
  const long long bh = tile / ntq;
  const int row0 = (int)(tile - bh * ntq) * kDiffTile, b = (int)(bh / a.H), h = (int)(bh - (long long)b * a.H);
  const int qlen = clamp_len(a.q_len, b, a.NQ);
  const float lam = a.lam[h], l2lam = __builtin_amdgcn_logf(fabsf(lam) < 0x1p-126f ? fabsf(lam) * 0x1p64f : fabsf(lam)) -
                                      (fabsf(lam) < 0x1p-126f ? 64.f : 0.f);   // -inf at 0
  float* st = a.stats + tile * kDiffStatsTile;
  const int c = lane & (tpr - 1), rpw = 64 / tpr;
  for (int r = wave * rpw + lane / tpr; r < kDiffTile; r += rpw * (kThreads / 64)) {
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
      const float d1 = __builtin_fmaf(lam, s2, s1);
      st[2 * kDiffTile + r] = none ? 0.f : -d1;
      st[3 * kDiffTile + r] = none ? 0.f : lam < 0.f ? d1 - s2 : s2 - d1;
    }
  }
}

// dlam_h = -sum of its blocks' partial sums, one workgroup per head.
__global__ void __launch_bounds__(kThreads) diff_bwd_dlam_kernel(const DiffArgs a, int T) {
  __shared__ double red[kThreads / 64];
  const int h = blockIdx.x, tid = threadIdx.x;
  double s = 0.;
  for (int i = tid; i < a.B * T; i += kThreads) {
    const int b = i / T;
    s += a.dlam_part[((long long)b * a.H + h) * T + (i - b * T)];
  }
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) s += __shfl_xor(s, m);
  if ((tid & 63) == 0) red[tid >> 6] = s;
  __syncthreads();
  if (tid == 0) a.dlam[h] = (float)-((red[0] + red[1]) + (red[2] + red[3]));
}

// Sum of n partial arrays in their order, `each` floats apart: `count` values
// of one gradient, a multiple of 4.
template <bool BF16>
__global__ void __launch_bounds__(kThreads) diff_bwd_join_kernel(const float* __restrict__ part, long long each, int n,
                                                                 void* __restrict__ out, long long count) {
  for (long long i = ((long long)blockIdx.x * kThreads + threadIdx.x) * 4; i < count;
       i += (long long)gridDim.x * kThreads * 4) {
    f32x4 s = *reinterpret_cast<const f32x4*>(part + i);
    for (int j = 1; j < n; ++j) s += *reinterpret_cast<const f32x4*>(part + j * each + i);
    if (BF16) {
      bf16x4 r;
#pragma unroll
      for (int e = 0; e < 4; ++e) r[e] = (__bf16)s[e];
      uint32_t* o = reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(out) + i);   // 4-byte aligned
      const uint64_t bits = __builtin_bit_cast(uint64_t, r);
      o[0] = (uint32_t)bits;
      o[1] = (uint32_t)(bits >> 32);
    } else {
      float* o = static_cast<float*>(out) + i;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = s[e];
    }
  }
}

hipError_t join(const float* part, long long each, int n, void* out, long long count, bool bf16, hipStream_t st) {
  if (!out || count == 0) return hipSuccess;
  const long long blocks = (count / 4 + kThreads - 1) / kThreads;
  const dim3 grid((unsigned)(blocks < 16 * kCus ? blocks : 16 * kCus));
  if (bf16)
    hipLaunchKernelGGL(diff_bwd_join_kernel<true>, grid, dim3(kThreads), 0, st, part, each, n, out, count);
  else
    hipLaunchKernelGGL(diff_bwd_join_kernel<false>, grid, dim3(kThreads), 0, st, part, each, n, out, count);
  return hipGetLastError();
}

}  // namespace

size_t diff_bwd_stats_floats(int B, int H, int NQ) {
  return (size_t)B * H * ((NQ + kDiffTile - 1LL) / kDiffTile) * kDiffStatsTile;
}

size_t diff_bwd_dlam_floats(int B, int H, int NQ, int q_splits) {
  return ((size_t)B * H * 2 * diff_row_blocks(NQ) * q_splits + 1) / 2 * 4;   // a double each, blocks of 64 rows
}

hipError_t launch_diff_bwd_prep(const DiffArgs& a) {
  const int ntq = (a.NQ + kDiffTile - 1) / kDiffTile;
  const long long tiles = (long long)a.B * a.H * ntq;
  const int chunks = a.dv / 8, tpr = chunks <= 4 ? 4 : chunks <= 8 ? 8 : chunks <= 16 ? 16 : 32;
  hipLaunchKernelGGL(diff_bwd_prep_kernel, dim3((unsigned)tiles), dim3(kThreads), 0, a.stream, a, a.out, a.out2, ntq,
                     tpr);
  return hipGetLastError();
}

hipError_t launch_diff_bwd_dlam(const DiffArgs& a) {
  hipLaunchKernelGGL(diff_bwd_dlam_kernel, dim3((unsigned)a.H), dim3(kThreads), 0, a.stream, a,
                     a.row_blocks * a.q_splits);
  return hipGetLastError();
}

hipError_t launch_diff_bwd_join_q(const DiffArgs& a) {
  const long long each = (long long)a.B * a.H * a.NQ * a.d;
  const bool half = a.bf16_grads != 0;
  hipError_t e = join(a.grad_part, 2 * each, a.q_splits, a.dq1, each, half, a.stream);
  if (e == hipSuccess) e = join(a.grad_part + each, 2 * each, a.q_splits, a.dq2, each, half, a.stream);
  return e;
}

hipError_t launch_diff_bwd_join_k(const DiffArgs& a) {
  const long long keys = (long long)a.B * a.HK * a.NK, each = keys * (2 * a.d + a.dv);
  const bool half = a.bf16_grads != 0;
  hipError_t e = join(a.grad_part, each, a.k_splits, a.dk1, keys * a.d, half, a.stream);
  if (e == hipSuccess) e = join(a.grad_part + keys * a.d, each, a.k_splits, a.dk2, keys * a.d, half, a.stream);
  if (e == hipSuccess) e = join(a.grad_part + keys * 2 * a.d, each, a.k_splits, a.dv_out, keys * a.dv, half, a.stream);
  return e;
}

}  // namespace streamkl
