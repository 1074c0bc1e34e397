// Backward kernels of differential attention.
//
// With dP = dO V^T (one product for both maps), D_t = dO . O_t per row:
//   dS_1 = P_1 (dP - D_1),   dS_2 = -lam P_2 (dP - D_2),
//   dQ_t = s dS_t K_t,  dK_t = s dS_t^T Q_t,  dV = (P_1 - lam P_2)^T dO,
//   dlam_h = -sum_rows sum_j P_2 dP.
// The probabilities are recomputed from the saved log-sum-exps. A query-owned
// kernel writes dQ_1, dQ_2 and the sums for dlam, a key-owned kernel dK_1,
// dK_2 and dV: every output has one owner, there are no atomics, and results
// are reproducible bit for bit. That costs 16 d + 6 dv operations a pair where
// a single pass with atomic adds would need 12 d + 4 dv.
//
// The logit tile of the first contraction lies in the registers as the A
// operand of the second (its 16-row k-blocks are a permutation of the 32
// rows); the other operand comes from the streamed tile by transpose reads.
//
// Rounding: the logit gradients and P_1 - lam P_2 to bf16 as operands of the
// second contraction (each term is off by at most 2^-8 of itself), gradients
// once when they are written. D_t is formed from the bf16 outputs O and O_2;
// dlam is not: P_2 dP is summed in float32 from the recomputed values.
//
// Prepared statistics (diff_bwd_prep_kernel): for every head and 32-row tile
// 4 x 32 floats,
//   [0] LSE_1 log2 e                    [1] LSE_2 log2 e - log2 |lam|
//   [2] D_1                             [3] sign(lam) D_2
// so that 2^(c s_2 - [1]) is |lam| P_2 without a multiply; rows that do not
// exist or see nothing have +inf offsets (P = 0).
#pragma once

#include "diff_common.hpp"
#include "kl_bwd.hpp"

namespace streamkl {

constexpr int kDiffStatsTile = 4 * kDiffTile;   // floats per tile

template <int D, int DV>
struct DiffBwdCfg {
  static constexpr int NW = 4, NT = 64 * NW, ROWS = 32 * NW;
  static constexpr int CD = D / 8, CV = DV / 8;
  static constexpr int STAGE = DiffDma<D, DV, NT>::CHUNKS;
  // registers: gradients, resident rows, three logit tiles, about 64 for the rest
  static constexpr int REGS_Q = D + (2 * D + DV) / 4 + 48 + 64;
  static constexpr int REGS_K = D + DV / 2 + (2 * D + DV) / 4 + 48 + 64;
  static constexpr int WAVES_Q = REGS_Q <= 256 ? 2 : 1, WAVES_K = REGS_K <= 256 ? 2 : 1;
};

// One 32 x 32 block of raw products streamed x resident: A = rows of the
// streamed tile (matrix at `tile`), B = resident operands.
template <int D>
__device__ __forceinline__ f32x16 diff_product(const u32x4* tile, const bf16x8 (&op)[D / 16], int lane) {
  f32x16 s = zero16();
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks)
    s = mfma32(lds_row8<D / 8>(tile, lane & 31, 2 * ks + (lane >> 5)), op[ks], s);
  return s;
}

// ---------------------------------------------------------------------------
// dQ: workgroup = 128 query rows of one head, streams tiles [K_1 | K_2 | V].
// ---------------------------------------------------------------------------
template <int D, int DV>
__global__ void __launch_bounds__(kThreads, (DiffBwdCfg<D, DV>::WAVES_Q)) diff_bwd_dq_kernel(const DiffArgs a) {
  using C = DiffBwdCfg<D, DV>;
  __shared__ u32x4 st0[C::STAGE];
  __shared__ u32x4 st1[C::STAGE];
  __shared__ float red[C::NW];
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int T = (a.NQ + C::ROWS - 1) / C::ROWS;
  int bh, blk;
  if (a.causal) {
    causal_block(blockIdx.x, gridDim.x, T, kCus * C::WAVES_Q, bh, blk);
    blk = T - 1 - blk;
  } else {
    const int x = xcd_logical(blockIdx.x, gridDim.x);
    bh = x / T;
    blk = x - bh * T;
  }
  const int b = bh / a.H, h = bh - b * a.H, hk = h / (a.H / a.HK);
  const int qlen = clamp_len(a.q_len, b, a.NQ), klen = clamp_len(a.kv_len, b, a.NK);
  const int off = klen - qlen;
  const float c = a.scale * kLog2e;
  auto limit_of = [&](int i) { return a.causal ? min(max(off + i + 1, 0), klen) : klen; };
  const int r0 = blk * C::ROWS, rw = r0 + 32 * wave, row = rw + (lane & 31);
  const int t_end = r0 < qlen ? (limit_of(min(r0 + C::ROWS, qlen) - 1) + kDiffTile - 1) / kDiffTile : 0;
  const int wave_min = limit_of(rw), wave_max = rw < qlen ? limit_of(min(rw + 32, qlen) - 1) : 0;

  const bool ok = row < qlen;
  const int limit = ok ? limit_of(row) : klen;
  bf16x8 q1[D / 16], q2[D / 16], go[DV / 16];
  auto row_of = [&](const DiffRows& x) {
    return x.p + (ok ? (long long)b * x.sb + (long long)h * x.sh + (long long)row * x.sn : 0);
  };
  load_row_operand<D>(q1, row_of(a.q1), ok, half, a.d);
  load_row_operand<D>(q2, row_of(a.q2), ok, half, a.d);
  const long long ri = (long long)bh * a.NQ + row;
  load_row_operand<DV>(go, a.dout + (ok ? ri * a.dv : 0), ok, half, a.dv);
  const int ntq = (a.NQ + kDiffTile - 1) / kDiffTile;
  const float lam = a.lam[h];
  float ls1 = __builtin_inff(), ls2 = ls1, d1 = 0.f, d2 = 0.f;
  if (ok) {
    const float* st = a.stats + ((long long)bh * ntq + row / kDiffTile) * kDiffStatsTile + row % kDiffTile;
    d1 = st[2 * kDiffTile];
    d2 = lam < 0.f ? -st[3 * kDiffTile] : st[3 * kDiffTile];
    const float e1 = a.lse1[ri], e2 = a.lse2[ri];
    ls1 = e1 == kNegInf ? __builtin_inff() : e1 * kLog2e;
    ls2 = e2 == kNegInf ? __builtin_inff() : e2 * kLog2e;
  }
  wait_vmem();   // before the tile loop: a first use inside it would wait on every trip

  f32x16 g1[D / 32], g2[D / 32];
#pragma unroll
  for (int n = 0; n < D / 32; ++n) {
    g1[n] = zero16();
    g2[n] = zero16();
  }
  float dl = 0.f;   // sum of P_2 dP

  const uint32_t bk1 = (uint32_t)a.k1.sn * 2u, bk2 = (uint32_t)a.k2.sn * 2u, bv = (uint32_t)a.v.sn * 2u;
  const uint16_t* k1 = a.k1.p + (long long)b * a.k1.sb + (long long)hk * a.k1.sh;
  const uint16_t* k2 = a.k2.p + (long long)b * a.k2.sb + (long long)hk * a.k2.sh;
  const uint16_t* vv = a.v.p + (long long)b * a.v.sb + (long long)hk * a.v.sh;
  const DiffDma<D, DV, C::NT> dma(tid, a.d, a.dv, bk1, bk2, bv);
  const TrCols<D> tr(lane);
  auto load = [&](int t, u32x4* stage) {
    dma.issue(tile_rsrc(k1, t * kDiffTile, klen, bk1, a.d), tile_rsrc(k2, t * kDiffTile, klen, bk2, a.d),
              tile_rsrc(vv, t * kDiffTile, klen, bv, a.dv), stage, wave);
  };

  auto tile = [&](const u32x4* stage, int t) {
    const int k0 = t * kDiffTile;
    if (k0 >= wave_max) return;
    f32x16 s1 = diff_product<D>(stage, q1, lane);
    f32x16 s2 = diff_product<D>(stage + kDiffTile * C::CD, q2, lane);
    const f32x16 dp = diff_product<DV>(stage + 2 * kDiffTile * C::CD, go, lane);
    if (k0 + kDiffTile > wave_min) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const bool seen = k0 + 8 * (i >> 2) + 4 * half + (i & 3) < limit;
        s1[i] = seen ? s1[i] : kNegInf;
        s2[i] = seen ? s2[i] : kNegInf;
      }
    }
    float e1[16], e2[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float p1 = exp2_fast(__builtin_fmaf(s1[i], c, -ls1)), p2 = exp2_fast(__builtin_fmaf(s2[i], c, -ls2));
      e1[i] = p1 * (dp[i] - d1);
      e2[i] = p2 * (dp[i] - d2);
      dl = __builtin_fmaf(p2, dp[i], dl);
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const bf16x8 a1 = pack8(e1 + 8 * u), a2 = pack8(e2 + 8 * u);
#pragma unroll
      for (int n = 0; n < D / 32; ++n) g1[n] = mfma32(a1, tr.read(stage, 0, n, u), g1[n]);
#pragma unroll
      for (int n = 0; n < D / 32; ++n) g2[n] = mfma32(a2, tr.read(stage, kDiffTile * C::CD * 16, n, u), g2[n]);
    }
  };

  if (t_end > 0) load(0, st0);
  wait_vmem();
  barrier_no_fence();
  auto step = [&](const u32x4* cur, u32x4* nxt, int t) {
    if (t + 1 < t_end) load(t + 1, nxt);
    tile(cur, t);
    wait_vmem();
    wait_lds();
    barrier_no_fence();
  };
  for (int t = 0; t < t_end; t += 2) {
    step(st0, st1, t);
    if (t + 1 < t_end) step(st1, st0, t + 1);
  }

  const size_t rows = (size_t)bh * a.NQ;
  if (a.dq1) write_grad<D>(a.dq1, a.bf16_grads != 0, g1, rows, rw, a.NQ, a.scale, lane, a.d);
  if (a.dq2) write_grad<D>(a.dq2, a.bf16_grads != 0, g2, rows, rw, a.NQ, -a.scale * lam, lane, a.d);
  if (a.dlam) {
    if (!ok) dl = 0.f;
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) dl += __shfl_xor(dl, x);
    if (lane == 0) red[wave] = dl;
    __syncthreads();
    if (tid == 0) a.dlam_part[(long long)bh * T + blk] = (red[0] + red[1]) + (red[2] + red[3]);
  }
}

// ---------------------------------------------------------------------------
// dK, dV: workgroup = 128 keys of one key head, streams tiles [Q_1 | Q_2 | dO]
// of 32 rows, one query head of the group after the other, with their
// prepared statistics.
// ---------------------------------------------------------------------------
template <int D, int DV>
__global__ void __launch_bounds__(kThreads, (DiffBwdCfg<D, DV>::WAVES_K)) diff_bwd_dkv_kernel(const DiffArgs a) {
  using C = DiffBwdCfg<D, DV>;
  __shared__ u32x4 st0[C::STAGE];
  __shared__ u32x4 st1[C::STAGE];
  __shared__ f32x4 stat[2][4][kDiffTile / 4];
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int T = (a.NK + C::ROWS - 1) / C::ROWS, G = a.H / a.HK;
  int bk, blk;
  if (a.causal) {
    causal_block(blockIdx.x, gridDim.x, T, kCus * C::WAVES_K, bk, blk);   // rank 0: the first keys, seen by the most rows
  } else {
    const int x = xcd_logical(blockIdx.x, gridDim.x);
    bk = x / T;
    blk = x - bk * T;
  }
  const int b = bk / a.HK, hk = bk - b * a.HK;
  const int qlen = clamp_len(a.q_len, b, a.NQ), klen = clamp_len(a.kv_len, b, a.NK);
  const int off = klen - qlen;
  const float c = a.scale * kLog2e;
  const int kb0 = blk * C::ROWS, kw = kb0 + 32 * wave, key = kw + (lane & 31);

  // row tiles that see a key of the block, for every head of the group
  const int t_all = (qlen + kDiffTile - 1) / kDiffTile;
  const int t_first = !a.causal ? 0 : min(max(kb0 - off, 0) / kDiffTile, t_all);
  const int per = kb0 < klen ? t_all - t_first : 0, t_end = per * G;

  const bool ok = key < klen;
  bf16x8 k1[D / 16], k2[D / 16], vv[DV / 16];
  auto row_of = [&](const DiffRows& x) {
    return x.p + (ok ? (long long)b * x.sb + (long long)hk * x.sh + (long long)key * x.sn : 0);
  };
  load_row_operand<D>(k1, row_of(a.k1), ok, half, a.d);
  load_row_operand<D>(k2, row_of(a.k2), ok, half, a.d);
  load_row_operand<DV>(vv, row_of(a.v), ok, half, a.dv);
  wait_vmem();   // before the tile loop: a first use inside it would wait on every trip

  f32x16 g1[D / 32], g2[D / 32], gv[DV / 32];
#pragma unroll
  for (int n = 0; n < D / 32; ++n) {
    g1[n] = zero16();
    g2[n] = zero16();
  }
#pragma unroll
  for (int n = 0; n < DV / 32; ++n) gv[n] = zero16();

  const uint32_t bq1 = (uint32_t)a.q1.sn * 2u, bq2 = (uint32_t)a.q2.sn * 2u, bo = (uint32_t)a.dv * 2u;
  const DiffDma<D, DV, C::NT> dma(tid, a.d, a.dv, bq1, bq2, bo);
  const TrCols<D> trd(lane);
  const TrCols<DV> trv(lane);
  const int ntq = (a.NQ + kDiffTile - 1) / kDiffTile;
  // step u: head hk G + u / per, row tile t_first + u % per. The loads run one
  // step ahead, so each side keeps its own place.
  int lg = 0, lt = 0;
  auto load = [&](u32x4* stage, int buf) {
    const int h = hk * G + lg, row0 = (t_first + lt) * kDiffTile;
    const long long bh = (long long)b * a.H + h;
    dma.issue(tile_rsrc(a.q1.p + (long long)b * a.q1.sb + (long long)h * a.q1.sh, row0, qlen, bq1, a.d),
              tile_rsrc(a.q2.p + (long long)b * a.q2.sb + (long long)h * a.q2.sh, row0, qlen, bq2, a.d),
              tile_rsrc(a.dout + bh * a.NQ * a.dv, row0, qlen, bo, a.dv), stage, wave);
#if defined(__HIP_DEVICE_COMPILE__)
    if (wave == 0) {
      const rsrc_t rs = make_rsrc(a.stats + (bh * ntq + t_first + lt) * kDiffStatsTile, kDiffStatsTile * 4u);
      float* dst = reinterpret_cast<float*>(&stat[buf][0][0]);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void*)dst, 4, 4u * lane, 0, 0, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void*)(dst + 64), 4, 4u * lane + 256u, 0, 0, 0);
    }
#endif
    if (++lt == per) {
      lt = 0;
      ++lg;
    }
  };

  int cg = 0, ct = 0;
  float nsign = a.lam[hk * G] < 0.f ? 1.f : -1.f;   // -sign(lam) of the current head
  auto tile = [&](const u32x4* stage, int buf) {
    const int r0 = (t_first + ct) * kDiffTile;
    const int rlast = min(r0 + kDiffTile, qlen) - 1;
    const bool active = kw < klen && (!a.causal || rlast + off >= kw);
    if (active) {
      const u32x4* to = stage + 2 * kDiffTile * C::CD;
      f32x16 s1 = diff_product<D>(stage, k1, lane);
      f32x16 s2 = diff_product<D>(stage + kDiffTile * C::CD, k2, lane);
      const f32x16 dp = diff_product<DV>(to, vv, lane);
      if ((a.causal && kw + 31 > r0 + off) || kw + 32 > klen) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const bool seen = ok && (!a.causal || key <= r0 + 8 * (i >> 2) + 4 * half + (i & 3) + off);
          s1[i] = seen ? s1[i] : kNegInf;
          s2[i] = seen ? s2[i] : kNegInf;
        }
      }
      float p[16], e1[16], e2[16];
#pragma unroll
      for (int qd = 0; qd < 4; ++qd) {
        const f32x4 l1 = stat[buf][0][2 * qd + half], l2 = stat[buf][1][2 * qd + half];
        const f32x4 d1 = stat[buf][2][2 * qd + half], d2 = stat[buf][3][2 * qd + half];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int i = 4 * qd + j;
          const float p1 = exp2_fast(__builtin_fmaf(s1[i], c, -l1[j]));
          const float p2 = exp2_fast(__builtin_fmaf(s2[i], c, -l2[j]));   // |lam| P_2
          p[i] = __builtin_fmaf(nsign, p2, p1);
          e1[i] = p1 * (dp[i] - d1[j]);
          e2[i] = p2 * __builtin_fmaf(nsign, dp[i], d2[j]);
        }
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const bf16x8 ap = pack8(p + 8 * u), a1 = pack8(e1 + 8 * u), a2 = pack8(e2 + 8 * u);
#pragma unroll
        for (int n = 0; n < DV / 32; ++n)
          gv[n] = mfma32(ap, trv.read(stage, 2 * kDiffTile * C::CD * 16, n, u), gv[n]);
#pragma unroll
        for (int n = 0; n < D / 32; ++n) g1[n] = mfma32(a1, trd.read(stage, 0, n, u), g1[n]);
#pragma unroll
        for (int n = 0; n < D / 32; ++n) g2[n] = mfma32(a2, trd.read(stage, kDiffTile * C::CD * 16, n, u), g2[n]);
      }
    }
    if (++ct == per) {
      ct = 0;
      if (++cg < G) nsign = a.lam[hk * G + cg] < 0.f ? 1.f : -1.f;
    }
  };

  if (t_end > 0) load(st0, 0);
  wait_vmem();
  barrier_no_fence();
  auto step = [&](const u32x4* cur, u32x4* nxt, int t, int buf) {
    if (t + 1 < t_end) load(nxt, buf ^ 1);
    tile(cur, buf);
    wait_vmem();
    wait_lds();
    barrier_no_fence();
  };
  for (int t = 0; t < t_end; t += 2) {
    step(st0, st1, t, 0);
    if (t + 1 < t_end) step(st1, st0, t + 1, 1);
  }

  const size_t rows = (size_t)bk * a.NK;
  const bool half_type = a.bf16_grads != 0;
  if (a.dk1) write_grad<D>(a.dk1, half_type, g1, rows, kw, a.NK, a.scale, lane, a.d);
  if (a.dk2) write_grad<D>(a.dk2, half_type, g2, rows, kw, a.NK, a.scale, lane, a.d);
  if (a.dv_out) write_grad<DV>(a.dv_out, half_type, gv, rows, kw, a.NK, 1.f, lane, a.dv);
}

}  // namespace streamkl
