// Query-owned kernel of the differential-attention backward with 16 rows a
// wave: the sums of diff_bwd_dq_kernel on the 16x16x32 MFMA, two waves per SIMD
// where 32 rows a wave leave room for one. See diff_bwd_keys16.hpp.
// dQ with 32 and 16 rows a wave, us: 4 x 12 heads x 1021 ragged, d 96/160, 62 and 54;
// 16 heads x 4096 causal, 64/192, 159 and 149, 128/192, 209 and 202; 8 heads x 6007, 128/128,
// 399 and 388; 16 heads x 4096, 96/96, 284 and 276, 128/256, 404 and 396.
// Where 32 rows leave room for two waves, they are ahead: 64/128, 249 and 262 (250 with three
// waves of 16 rows), 64/64, 193 and 215.
#pragma once

#include "diff_bwd_16.hpp"

namespace streamkl {

template <int D, int DV>
constexpr bool kDiffRows16 = DiffBwdCfg<D, DV>::WAVES_Q == 1;

template <int D, int DV>
__global__ void __launch_bounds__(kThreads, 2) diff_bwd_dq16_kernel(const DiffArgs a) {
  using C = Diff16Cfg<D, DV, 0>;
  constexpr int KD = D / 32, KV = DV / 32, ND = D / 16;
  __shared__ u32x4 st0[C::TR * C::STAGE];
  __shared__ u32x4 st1[C::TR * C::STAGE];
  __shared__ u32x4 st2[C::STAGES == 3 ? C::TR * C::STAGE : 1];
  __shared__ double red[kThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63, quad = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int T = (a.NQ + C::ROWS - 1) / C::ROWS;
  int bh, blk;
  if (a.causal) {
    causal_block(blockIdx.x, gridDim.x, T, 2 * kCus, bh, blk);
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
  const int r0 = blk * C::ROWS, rw = r0 + 16 * wave, row = rw + (lane & 15);
  int t_end = r0 < qlen ? (limit_of(min(r0 + C::ROWS, qlen) - 1) + kDiffTile - 1) / kDiffTile : 0, t_begin = 0;
  if (a.q_splits > 1) {
    const int each = (t_end + a.q_splits - 1) / a.q_splits;
    t_begin = min(t_end, (int)blockIdx.y * each);
    t_end = min(t_end, t_begin + each);
  }
  const int wave_min = limit_of(rw), wave_max = rw < qlen ? limit_of(min(rw + 16, qlen) - 1) : 0;

  const bool ok = row < qlen;
  const int limit = ok ? limit_of(row) : klen;
  bf16x8 q1[KD], q2[KD], go[KV];
  auto row_of = [&](const DiffRows& x) {
    return x.p + (ok ? (long long)b * x.sb + (long long)h * x.sh + (long long)row * x.sn : 0);
  };
  load_resident16(q1, row_of(a.q1), ok, quad);
  load_resident16(q2, row_of(a.q2), ok, quad);
  const long long ri = (long long)bh * a.NQ + row;
  load_resident16(go, a.dout + (ok ? ri * DV : 0), ok, quad);
  const int ntq = (a.NQ + kDiffTile - 1) / kDiffTile;
  const float lam = a.lam[h];
  const int lift = klen > 1 ? 31 - __builtin_clz(klen) : 0;   // P_2 is formed times 2^lift
  float ls1 = __builtin_inff(), ls2 = ls1, d1 = 0.f, d2 = 0.f;
  if (ok) {
    const float* st = a.stats + ((long long)bh * ntq + row / kDiffTile) * kDiffStatsTile + row % kDiffTile;
    d1 = -st[2 * kDiffTile];
    d2 = leading_bits(d1 + (lam < 0.f ? -st[3 * kDiffTile] : st[3 * kDiffTile]));
    const float e1 = a.lse1[ri], e2 = a.lse2[ri];
    ls1 = e1 == kNegInf ? __builtin_inff() : e1 * kLog2e;
    ls2 = e2 == kNegInf ? __builtin_inff() : e2 * kLog2e - (float)lift;
  }
  negate_odd_rows(go, d1, d2, lane);
  wait_vmem();   // before the tile loop: a first use inside it would wait on every trip

  f32x4 g1[ND], g2[ND];
#pragma unroll
  for (int n = 0; n < ND; ++n) g1[n] = g2[n] = f32x4{0.f, 0.f, 0.f, 0.f};
  double dl = 0.;   // 2^lift times the sum of P_2 (dP - D_2)

  const uint32_t bk1 = (uint32_t)a.k1.sn * 2u, bk2 = (uint32_t)a.k2.sn * 2u, bv = (uint32_t)a.v.sn * 2u;
  const uint16_t* k1 = a.k1.p + (long long)b * a.k1.sb + (long long)hk * a.k1.sh;
  const uint16_t* k2 = a.k2.p + (long long)b * a.k2.sb + (long long)hk * a.k2.sh;
  const uint16_t* vv = a.v.p + (long long)b * a.v.sb + (long long)hk * a.v.sh;
  const typename C::Dma dma(tid, bk1, bk2, bv);
  const Places16<D> pd(lane);
  const Places16<DV> pv(lane);
  TileRows r1(k1, bk1, D), r2(k2, bk2, D), r3(vv, bv, DV);
  r1.skip(t_begin);
  r2.skip(t_begin);
  r3.skip(t_begin);
  auto load = [&](int t, u32x4* stage) {
    const int rows = klen - t * kDiffTile;
    dma.issue(r1.next(rows), r2.next(rows), r3.next(rows), stage, wave);
  };

  auto tile = [&](int t, const u32x4* stage) {
    const int k0 = t * kDiffTile;
    if (k0 >= wave_max) return;
    constexpr int J1 = 2 * KD, J2 = 2 * J1, J3 = J2 + 2 * KV, J4 = J3 + 2 * ND, LA = C::LA;
    constexpr int B2 = kDiffTile * C::CD, B3 = 2 * B2;   // chunks before K_2 and V
    bf16x8 buf[J4];   // streamed operands, read LA of them ahead of their MFMAs
    auto rd = [&](int j) {
      if (j < J2) buf[j] = pd.rows(stage, j / J1 * B2, j % J1 / 2, j & 1);
      else if (j < J3) buf[j] = pv.rows(stage, B3, (j - J2) / 2, j & 1);
      else if (j < J4) buf[j] = pd.cols(stage, (j - J3) / ND * B2, (j - J3) % ND);
    };
    f32x4 s1[2], s2[2], dp[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) s1[x] = s2[x] = dp[x] = f32x4{0.f, 0.f, 0.f, 0.f};
    float e1[8], e2[8];
    const bool mask = k0 + kDiffTile > wave_min;
    auto hide = [&](f32x4 (&s)[2]) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        s[i >> 2][i & 3] = k0 + 16 * (i >> 2) + 4 * quad + (i & 3) < limit ? s[i >> 2][i & 3] : kNegInf;
    };
    diff_pin();
#pragma unroll
    for (int j = 0; j < LA; ++j) rd(j);
    diff_pin();
#pragma unroll
    for (int j = 0; j < J1; ++j) {
      rd(j + LA);
      s1[j & 1] = mfma16(buf[j], q1[j / 2], s1[j & 1]);
      diff_pin();
    }
    if (mask) hide(s1);
    diff_pin();
#pragma unroll
    for (int j = J1; j < J2; ++j) {
      rd(j + LA);
      s2[j & 1] = mfma16(buf[j], q2[(j - J1) / 2], s2[j & 1]);
#pragma unroll
      for (int i = 8 * (j - J1) / J1; i < 8 * (j - J1 + 1) / J1; ++i)
        e1[i] = exp2_fast(__builtin_fmaf(s1[i >> 2][i & 3], c, -ls1));
      diff_pin();
    }
    if (mask) hide(s2);
    diff_pin();
#pragma unroll
    for (int j = J2; j < J3; ++j) {
      rd(j + LA);
      dp[j & 1] = mfma16(buf[j], go[(j - J2) / 2], dp[j & 1]);
#pragma unroll
      for (int i = 8 * (j - J2) / (2 * KV); i < 8 * (j - J2 + 1) / (2 * KV); ++i)
        e2[i] = exp2_fast(__builtin_fmaf(s2[i >> 2][i & 3], c, -ls2));
      diff_pin();
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) e1[i] *= dp[i >> 2][i & 3] - d1;
    const bf16x8 a1 = pack8(e1);
    diff_pin();
    float dt = 0.f;
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int j = J3; j < J3 + ND; ++j) {
      rd(j + LA);
      g1[j - J3] = mfma16(a1, buf[j], g1[j - J3]);
#pragma unroll
      for (int i = 8 * (j - J3) / ND; i < 8 * (j - J3 + 1) / ND; ++i) {
        e2[i] *= dp[i >> 2][i & 3] - d2;
        dt += e2[i];
      }
      diff_pin();
    }
    const bf16x8 a2 = pack8(e2);
    diff_pin();
#pragma unroll
    for (int j = J3 + ND; j < J4; ++j) {
      rd(j + LA);
      g2[j - J3 - ND] = mfma16(a2, buf[j], g2[j - J3 - ND]);
      diff_pin();
    }
    __builtin_amdgcn_s_setprio(0);
    dl += (double)dt;
  };

  stream_tiles<C::STAGES, C::TR, C::STAGE, C::Dma::NCH>(st0, st1, st2, t_begin, t_end, load, tile);

  restore_rows(g1, g2, lift);
  const size_t rows = (size_t)bh * a.NQ;
  void *o1 = a.dq1, *o2 = a.dq2;
  bool as_bf16 = a.bf16_grads != 0;
  if (a.q_splits > 1) {
    const long long each = (long long)a.B * a.H * a.NQ * D;
    as_bf16 = false;
    if (o1) o1 = a.grad_part + (2 * (long long)blockIdx.y) * each;
    if (o2) o2 = a.grad_part + (2 * (long long)blockIdx.y + 1) * each;
  }
  if (o1) write_grad16(o1, as_bf16, g1, rows, rw, a.NQ, a.scale, lane);
  if (o2) write_grad16(o2, as_bf16, g2, rows, rw, a.NQ, -a.scale * lam, lane);
  if (a.dlam) {
    dl = __builtin_ldexp(dl, -lift) + (quad == 0 && blockIdx.y == 0 ? (double)d2 : 0.);   // D_2 once a row
    write_dlam_part(a.dlam_part + ((long long)bh * T + blk) * a.q_splits + blockIdx.y, red,
                    !ok ? 0. : (lane & 1) ? -dl : dl, tid);
  }
}

}  // namespace streamkl
