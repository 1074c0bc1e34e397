// Key-owned kernel of the differential-attention backward with 16 keys a wave.
//
// The same sums in the same order of a tile as diff_bwd_dkv_kernel, which has
// 32 keys a wave, on the 16x16x32 MFMA. Accumulators and resident rows take
// half the registers, so that two waves share a SIMD where 32 keys leave room
// for one; a streamed operand serves half the MFMA work, so that LDS delivers
// twice as much (47 and 50% of its cycles at d 64/128 and 128/128). One wave per SIMD issued its
// vector instructions and its MFMAs nearly one after the other (MFMAs busy
// 31 to 32% of the cycles, 37 and 43 now). dK dV with 32 and 16 keys a wave, us: 8 heads x
// 6007, d 128/128, 629 and 511; 32 heads x 4096 causal, 64/128, 364 and 342; 16 heads x
// 4096, 128/64, 398 and 357, 96/96, 359 and 339; 4 x 12 heads x 1021 ragged, 96/160, 112 and
// 97. Where 32 keys leave room for two waves as well, they are ahead: 64/64, 226 and
// 269, also with three or four waves of 16 keys.
//
// Workgroups of 64 keys, two on a CU, each at its own place in a tile: eight
// waves that meet at one barrier took 3 to 6% longer at 64/128.
//
// What bounds it: issue of two waves and LDS; waves wait 29% of the time.
//
// LDS: rows are swizzled by swz16 (diff_common.hpp), not as in the other
// kernels: here 32 lanes of a transpose read touch eight rows at one pair of
// chunks, not four rows at two, and 32 lanes of a row read two chunks.
#pragma once

#include "diff_bwd_16.hpp"

namespace streamkl {

// Where it runs: one wave per SIMD with 32 keys, and 256 registers suffice for 16.
template <int D, int DV>
constexpr bool kDiffKeys16 = DiffBwdCfg<D, DV>::WAVES_K == 1 && 2 * D + DV <= 384;

template <int D, int DV>
__global__ void __launch_bounds__(kThreads, 2) diff_bwd_dkv16_kernel(const DiffArgs a) {
  using C = Diff16Cfg<D, DV, kDiffStatsTile / 4>;
  constexpr int KD = D / 32, KV = DV / 32, ND = D / 16, NV = DV / 16;
  __shared__ u32x4 st0[C::TR * C::STAGE];
  __shared__ u32x4 st1[C::TR * C::STAGE];
  __shared__ u32x4 st2[C::STAGES == 3 ? C::TR * C::STAGE : 1];
  const int tid = threadIdx.x, lane = tid & 63, quad = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int T = (a.NK + C::ROWS - 1) / C::ROWS, G = a.H / a.HK;
  int bk, blk;
  if (a.causal) {
    causal_block(blockIdx.x, gridDim.x, T, 2 * kCus, bk, blk);
  } else {
    const int x = xcd_logical(blockIdx.x, gridDim.x);
    bk = x / T;
    blk = x - bk * T;
  }
  const int b = bk / a.HK, hk = bk - b * a.HK;
  const int qlen = clamp_len(a.q_len, b, a.NQ), klen = clamp_len(a.kv_len, b, a.NK);
  const int off = klen - qlen;
  const float c = a.scale * kLog2e;
  const int kb0 = blk * C::ROWS, kw = kb0 + 16 * wave, key = kw + (lane & 15);

  // row tiles that see a key of the block, for every head of the group
  const int t_all = (qlen + kDiffTile - 1) / kDiffTile;
  const int t_first = !a.causal ? 0 : min(max(kb0 - off, 0) / kDiffTile, t_all);
  const int per = kb0 < klen ? t_all - t_first : 0;
  int s_end = per * G, s_begin = 0;   // steps: one row tile of one head each
  if (a.k_splits > 1) {
    const int each = (s_end + a.k_splits - 1) / a.k_splits;
    s_begin = min(s_end, (int)blockIdx.y * each);
    s_end = min(s_end, s_begin + each);
  }
  const int g_begin = per ? s_begin / per : 0, t_begin = s_begin - g_begin * per;

  const bool ok = key < klen;
  const int first = !ok ? 0x7fffffff : a.causal ? key - off : 0;   // the first row that sees the lane's key
  bf16x8 k1[KD], k2[KD], vv[KV];
  auto row_of = [&](const DiffRows& x) {
    return x.p + (ok ? (long long)b * x.sb + (long long)hk * x.sh + (long long)key * x.sn : 0);
  };
  load_resident16(k1, row_of(a.k1), ok, quad);
  load_resident16(k2, row_of(a.k2), ok, quad);
  load_resident16(vv, row_of(a.v), ok, quad);
  wait_vmem();   // before the tile loop: a first use inside it would wait on every trip

  f32x4 g1[ND], g2[ND], gv[NV];
#pragma unroll
  for (int n = 0; n < ND; ++n) g1[n] = g2[n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int n = 0; n < NV; ++n) gv[n] = f32x4{0.f, 0.f, 0.f, 0.f};

  const uint32_t bq1 = (uint32_t)a.q1.sn * 2u, bq2 = (uint32_t)a.q2.sn * 2u, bo = (uint32_t)DV * 2u;
  const typename C::Dma dma(tid, bq1, bq2, bo);
  const Places16<D> pd(lane);
  const Places16<DV> pv(lane);
  const int ntq = (a.NQ + kDiffTile - 1) / kDiffTile;
  // step u: head hk G + u / per, row tile t_first + u % per. The loads run
  // ahead, so each side keeps its own place.
  int lg = g_begin, lt = t_begin;
  TileRows r1(nullptr, bq1, D), r2(nullptr, bq2, D), r3(nullptr, bo, DV);
  const float* ps = nullptr;
  auto begin_head = [&](int h, int t0) {
    const long long bh = (long long)b * a.H + h;
    r1.p = reinterpret_cast<const char*>(a.q1.p + (long long)b * a.q1.sb + (long long)h * a.q1.sh);
    r2.p = reinterpret_cast<const char*>(a.q2.p + (long long)b * a.q2.sb + (long long)h * a.q2.sh);
    r3.p = reinterpret_cast<const char*>(a.dout + bh * a.NQ * DV);
    r1.skip(t_first + t0);
    r2.skip(t_first + t0);
    r3.skip(t_first + t0);
    ps = a.stats + (bh * ntq + t_first + t0) * kDiffStatsTile;
  };
  begin_head(hk * G + (g_begin < G ? g_begin : 0), t_begin);
  auto load = [&](int, u32x4* stage) {
    const int rows = qlen - (t_first + lt) * kDiffTile;
    dma.issue(r1.next(rows), r2.next(rows), r3.next(rows), stage, wave);
#if defined(__HIP_DEVICE_COMPILE__)
    // every wave loads a quarter of the statistics: one instruction each, half of its lanes
    const rsrc_t rs = make_rsrc(ps, kDiffStatsTile * 4u);
    if (lane < 32)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void*)(reinterpret_cast<float*>(stage + C::Dma::CHUNKS) + 32 * wave),
                                               4, 4u * lane + 128u * wave, 0, 0, 0);
#endif
    ps += kDiffStatsTile;
    if (++lt == per) {
      lt = 0;
      if (++lg < G) begin_head(hk * G + lg, 0);
    }
  };

  int cg = g_begin, ct = t_begin;
  float nsign = a.lam[hk * G + (g_begin < G ? g_begin : 0)] < 0.f ? 1.f : -1.f;   // -sign(lam) of the current head
  auto products = [&](const u32x4* stage, int r0) {
    constexpr int J1 = 2 * KD, J2 = 2 * J1, J3 = J2 + 2 * KV, J4 = J3 + NV, J5 = J4 + 2 * ND, LA = C::LA;
    constexpr int B2 = kDiffTile * C::CD, B3 = 2 * B2;   // chunks before Q_2 and dO
    bf16x8 buf[J5];   // streamed operands, read LA of them ahead of their MFMAs
    auto rd = [&](int j) {
      if (j < J2) buf[j] = pd.rows(stage, j / J1 * B2, j % J1 / 2, j & 1);
      else if (j < J3) buf[j] = pv.rows(stage, B3, (j - J2) / 2, j & 1);
      else if (j < J4) buf[j] = pv.cols(stage, B3, j - J3);
      else if (j < J5) buf[j] = pd.cols(stage, (j - J4) / ND * B2, (j - J4) % ND);
    };
    // statistics of the lane's rows: block x of kind w at st[8 w + 4 x]
    const f32x4* st = reinterpret_cast<const f32x4*>(stage + C::Dma::CHUNKS) + quad;
    f32x4 s1[2], s2[2], dp[2], ga[2], gb[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) s1[x] = s2[x] = f32x4{0.f, 0.f, 0.f, 0.f};
    float e1[8], e2[8], p[8];
    const bool mask = (a.causal && kw + 15 > r0 + off) || kw + 16 > klen;
    auto hide = [&](f32x4 (&s)[2]) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        s[i >> 2][i & 3] = r0 + 16 * (i >> 2) + 4 * quad + (i & 3) >= first ? s[i >> 2][i & 3] : kNegInf;
      }
    };
    diff_pin();
#pragma unroll
    for (int j = 0; j < LA; ++j) rd(j);
    ga[0] = st[0];
    ga[1] = st[4];
    diff_pin();
#pragma unroll
    for (int j = 0; j < J1; ++j) {
      rd(j + LA);
      s1[j & 1] = mfma16(buf[j], k1[j / 2], s1[j & 1]);
      diff_pin();
    }
    gb[0] = st[8];
    gb[1] = st[12];
    if (mask) hide(s1);
    diff_pin();
#pragma unroll
    for (int j = J1; j < J2; ++j) {
      rd(j + LA);
      s2[j & 1] = mfma16(buf[j], k2[(j - J1) / 2], s2[j & 1]);
#pragma unroll
      for (int i = 8 * (j - J1) / J1; i < 8 * (j - J1 + 1) / J1; ++i)
        e1[i] = exp2_fast(__builtin_fmaf(s1[i >> 2][i & 3], c, -ga[i >> 2][i & 3]));   // P_1
      diff_pin();
    }
    dp[0] = st[16];   // -D_1
    dp[1] = st[20];
    if (mask) hide(s2);
    diff_pin();
#pragma unroll
    for (int j = J2; j < J3; ++j) {
      rd(j + LA);
      dp[j & 1] = mfma16(buf[j], vv[(j - J2) / 2], dp[j & 1]);
#pragma unroll
      for (int i = 8 * (j - J2) / (2 * KV); i < 8 * (j - J2 + 1) / (2 * KV); ++i) {
        e2[i] = exp2_fast(__builtin_fmaf(s2[i >> 2][i & 3], c, -gb[i >> 2][i & 3]));   // |lam| P_2
        p[i] = __builtin_fmaf(nsign, e2[i], e1[i]);
      }
      diff_pin();
    }
    const bf16x8 ap = pack8(p);
    ga[0] = st[24];
    ga[1] = st[28];
    diff_pin();
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int j = J3; j < J4; ++j) {
      rd(j + LA);
      gv[j - J3] = mfma16(ap, buf[j], gv[j - J3]);
#pragma unroll
      for (int i = 8 * (j - J3) / NV; i < 8 * (j - J3 + 1) / NV; ++i) {
        const float y = dp[i >> 2][i & 3];   // dP - D_1
        e1[i] *= y;
        e2[i] *= __builtin_fmaf(nsign, y, ga[i >> 2][i & 3]);
      }
      diff_pin();
    }
    const bf16x8 a1 = pack8(e1), a2 = pack8(e2);
    diff_pin();
#pragma unroll
    for (int j = J4; j < J5; ++j) {
      rd(j + LA);
      const int n = (j - J4) % ND;
      if (j - J4 < ND) g1[n] = mfma16(a1, buf[j], g1[n]);
      else g2[n] = mfma16(a2, buf[j], g2[n]);
      diff_pin();
    }
    __builtin_amdgcn_s_setprio(0);
  };
  auto tile = [&](int, const u32x4* stage) {
    const int r0 = (t_first + ct) * kDiffTile;
    const int rlast = min(r0 + kDiffTile, qlen) - 1;
    const bool active = kw < klen && (!a.causal || rlast + off >= kw);
    if (active) products(stage, r0);
    if (++ct == per) {
      ct = 0;
      if (++cg < G) nsign = a.lam[hk * G + cg] < 0.f ? 1.f : -1.f;
    }
  };

  stream_tiles<C::STAGES, C::TR, C::STAGE, C::Dma::NCH + 1>(st0, st1, st2, s_begin, s_end, load, tile);

  const size_t rows = (size_t)bk * a.NK;
  void *o1 = a.dk1, *o2 = a.dk2, *o3 = a.dv_out;
  bool as_bf16 = a.bf16_grads != 0;
  if (a.k_splits > 1) {
    const long long keys = (long long)a.B * a.HK * a.NK;
    float* part = a.grad_part + blockIdx.y * keys * (2 * D + DV);
    as_bf16 = false;
    if (o1) o1 = part;
    if (o2) o2 = part + keys * D;
    if (o3) o3 = part + keys * 2 * D;
  }
  if (o1) write_grad16(o1, as_bf16, g1, rows, kw, a.NK, a.scale, lane);
  if (o2) write_grad16(o2, as_bf16, g2, rows, kw, a.NK, a.scale, lane);
  if (o3) write_grad16(o3, as_bf16, gv, rows, kw, a.NK, 1.f, lane);
}

}  // namespace streamkl
