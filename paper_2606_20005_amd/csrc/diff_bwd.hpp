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
// Order of a tile, pinned: logits of map 1; logits of map 2 beside the
// exponentials of map 1; dP beside those of map 2; (dV beside the logit
// gradients;) dQ or dK. Streamed operands are read from LDS a few MFMAs ahead.
// Left to itself the compiler forms all products, then all vector work, and
// reads each operand right before its MFMA (d 64/128, 32 heads x 4096 causal:
// dQ 272 -> 257 us, dK dV 518 -> 392 in this order). Where two waves share a
// SIMD, raised priority in the gradient MFMAs lets the vector work of the other
// one fill their gaps (d 64/64, 16 heads x 4096: 208 -> 201, 249 -> 241).
//
// What bounds it: issue. At d 64/128 a tile of the key-owned kernel takes 32
// MFMAs (1024 cycles of the matrix pipe) and about 330 instructions, 184 of
// them vector ones, which one wave issued in 1850 cycles of 3200. So where 32
// keys a wave leave room for one wave per SIMD, diff_bwd_dkv16_kernel
// (diff_bwd_keys16.hpp) has 16 and room for two.
//
// The logit tile of the first contraction lies in the registers as the A
// operand of the second (its 16-row k-blocks are a permutation of the 32
// rows); the other operand comes from the streamed tile by transpose reads.
//
// Rounding: the logit gradients and P_1 - lam P_2 to bf16 as operands of the
// second contraction (each term is off by at most 2^-8 of itself), gradients
// once when they are written. D_t is formed from the bf16 outputs O and O_2, what
// a layer keeps anyway (in float32 they would be twice the bytes to save and to
// read): where a map is almost one key and dP - D cancels, that is the larger part
// of a gradient's error, 1% in norm for N(0,1) rows at scale 1, d 32, 0.2% at scale
// 1/sqrt(d).
//
// dlam can cancel to far below its terms P_2 dP, so it is held to what float32
// gives each of them:
// - sum_j P_2 dP = D_2 + sum_j P_2 (dP - D_2), as P_2 sums to 1: an error common
//   to the P_2 of a row (of its log-sum-exp) meets only what D_2 is off by. D_2
//   (from bf16 outputs) is rounded to 12 bits, so that dP - D_2 is exact: its
//   rounding would be the same for many keys of a row.
// - P_2 is formed times 2^n, n = log2 of the keys rounded down, which leaves its
//   exponent near 0 instead of near -n, where float32 has fewer bits for it.
// - Odd rows run with -dO, -D_1 and -D_2, and their results change sign at the
//   end: the matrix unit's sums fall short by about 2^-33 of their size,
//   whatever their sign (with -dO for dO throughout, dlam + dlam' was 2.0e-5 for
//   each of 8 heads x 6007, d 128/128), which adds up over rows of one sign.
// - The 16 (or 8) terms of a tile are added in float32, tiles, rows and blocks in
//   64 bits.
// Error relative to the root of the sum of the squared terms: 256 x 256, d 64/64,
// 1.5e-7; 64 rows x 8192 keys, 64/64, 1.2e-7; 6007 x 6007, 128/128, 2.3e-7. With
// P_2 dP in one float32 chain over a row's keys 3.9e-7, 7.3e-7 and 1.1e-6, in
// plain float32 1.9e-7, 1.9e-7 and 4.5e-7.
//
// Prepared statistics (diff_bwd_prep_kernel): for every head and 32-row tile
// 4 x 32 floats,
//   [0] LSE_1 log2 e                    [1] LSE_2 log2 e - log2 |lam|
//   [2] -D_1                            [3] sign(lam) (D_2 - D_1)
// so that 2^(c s_2 - [1]) is |lam| P_2 without a multiply, and dP - D_1 is what
// the product gives when its accumulators start from [2]; rows that do not
// exist or see nothing have +inf offsets (P = 0).
#pragma once

#include "diff_common.hpp"
#include "kl_bwd.hpp"

namespace streamkl {

constexpr int kDiffStatsTile = 4 * kDiffTile;   // floats per tile

// *p += v in LDS, where only this lane touches *p. Written out, since the
// compiler waits for every load into LDS in flight before a write to it that it
// knows of. Nothing comes back; LDS operations of a wave take effect in order.
__device__ __forceinline__ void lds_add_f64(double* p, double v) {
  typedef __attribute__((address_space(3))) double lds_f64;
  asm volatile("ds_add_f64 %0, %1" ::"v"((uint32_t)(uintptr_t)(lds_f64*)p), "v"(v) : "memory");
}

// x rounded to its leading 12 bits.
__device__ __forceinline__ float leading_bits(float x) {
  return __uint_as_float((__float_as_uint(x) + 0x800u) & 0xfffff000u);
}

// The rows of odd lanes with the other sign.
template <int K>
__device__ __forceinline__ void negate_odd_rows(bf16x8 (&op)[K], float& d1, float& d2, int lane) {
  const uint32_t sign = (lane & 1) ? 0x80008000u : 0u;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    u32x4 t = __builtin_bit_cast(u32x4, op[k]);
    t ^= sign;
    op[k] = __builtin_bit_cast(bf16x8, t);
  }
  d1 = (lane & 1) ? -d1 : d1;
  d2 = (lane & 1) ? -d2 : d2;
}

// The query gradients of a wave (element i of an accumulator is in a row of i's
// parity) as they are: signs of odd rows, 2^lift of map 2.
template <typename Acc, int N>
__device__ __forceinline__ void restore_rows(Acc (&g1)[N], Acc (&g2)[N], int lift) {
  const float f = __builtin_ldexpf(1.f, -lift);
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int i = 0; i < (int)(sizeof(Acc) / sizeof(float)); ++i) {
      g1[n][i] = (i & 1) ? -g1[n][i] : g1[n][i];
      g2[n][i] *= (i & 1) ? -f : f;
    }
}

// The sum over a workgroup of its lanes' parts of sum_j P_2 dP, to part[0].
__device__ __forceinline__ void write_dlam_part(double* part, double* red, double dl, int tid) {
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) dl += __shfl_xor(dl, x);
  if ((tid & 63) == 0) red[tid >> 6] = dl;
  __syncthreads();
  if (tid == 0) part[0] = (red[0] + red[1]) + (red[2] + red[3]);
}

template <int D, int DV, int PART = 3>
struct DiffBwdCfg {
  static constexpr int NW = 4, NT = 64 * NW, ROWS = 32 * NW;
  static constexpr int CD = lds_cols(D) / 8, CV = lds_cols(DV) / 8;   // chunks of a row in LDS
  static constexpr int STAGE = DiffDma<D, DV, NT>::CHUNKS;
  static constexpr int STATS = kDiffStatsTile / 4;   // chunks of prepared statistics behind a stage (dK, dV)
  // registers: gradients, resident rows, three logit tiles, about 64 for the rest
  static constexpr int REGS_Q = D + (2 * D + DV) / 4 + 48 + 64;
  static constexpr int REGS_K = (PART & 1 ? D + DV / 4 + 16 : 0) + (PART & 2 ? DV / 2 : 0) + D / 2 + DV / 16 + 28 + 64;
  // 256 registers leave room for two waves per SIMD. The estimate is tight: d 64/192 meets 256 and spills in the
  // query-owned kernel (190 us with one wave, 226 with two), as does dV alone at 128/192. Where WAVES_Q or WAVES_K is 1,
  // the kernels with 16 rows or keys a wave take over (diff_bwd_rows16.hpp, diff_bwd_keys16.hpp), but for the widest keys.
  static constexpr int WAVES_Q = REGS_Q <= 248 ? 2 : 1, WAVES_K = REGS_K <= 256 - (PART == 2 ? 8 : 0) ? 2 : 1;
  static constexpr int LA_Q = REGS_Q > 232 ? 2 : 3, LA_K = WAVES_K == 1 ? 4 : 2;   // operand reads in flight
  // Three stages where the workgroups that the registers leave room for have
  // room for them; two tiles a stage in the key-owned kernel with one wave per
  // SIMD, which nothing else occupies while it waits for the others (d 64/128,
  // 32 heads x 4096 causal: 414 -> 394 us together with the next item; no gain
  // in the query-owned kernel).
  static constexpr int ROOM = 158 * 1024;
  static constexpr int TILE_Q = STAGE * 16 * 2, TILE_K = (STAGE + STATS) * 16 * WAVES_K;
  static constexpr int TR_K = WAVES_K == 1 && 4 * TILE_K <= ROOM ? 2 : 1;
  static constexpr int STAGES_Q = 3 * TILE_Q <= ROOM ? 3 : 2, STAGES_K = 3 * TR_K * TILE_K <= ROOM ? 3 : 2;
  // dP's accumulators start from -D_1, which saves a subtraction an element;
  // with two waves per SIMD the registers that hold it early spill (d 64/64,
  // 16 heads x 4096: 259 -> 291 us).
  static constexpr bool START_D = WAVES_K == 1;
};

// ---------------------------------------------------------------------------
// dQ: workgroup = 128 query rows of one head, streams tiles [K_1 | K_2 | V].
// ---------------------------------------------------------------------------
template <int D, int DV>
__global__ void __launch_bounds__(kThreads, 2) diff_bwd_dq_kernel(const DiffArgs a) {
  using C = DiffBwdCfg<D, DV>;
  constexpr int KD = D / 16, KV = DV / 16, ND = D / 32;
  __shared__ u32x4 st0[C::STAGE];
  __shared__ u32x4 st1[C::STAGE];
  __shared__ u32x4 st2[C::STAGES_Q == 3 ? C::STAGE : 1];
  __shared__ double red[C::NW];
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
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
  const int r0 = blk * C::ROWS, rw = r0 + 32 * wave, row = rw + (lane & 31);
  int t_end = r0 < qlen ? (limit_of(min(r0 + C::ROWS, qlen) - 1) + kDiffTile - 1) / kDiffTile : 0, t_begin = 0;
  if (a.q_splits > 1) {
    const int each = (t_end + a.q_splits - 1) / a.q_splits;
    t_begin = min(t_end, (int)blockIdx.y * each);
    t_end = min(t_end, t_begin + each);
  }
  const int wave_min = limit_of(rw), wave_max = rw < qlen ? limit_of(min(rw + 32, qlen) - 1) : 0;

  const bool ok = row < qlen;
  const int limit = ok ? limit_of(row) : klen;
  bf16x8 q1[D / 16], q2[D / 16], go[DV / 16];
  auto row_of = [&](const DiffRows& x) {
    return x.p + (ok ? (long long)b * x.sb + (long long)h * x.sh + (long long)row * x.sn : 0);
  };
  load_row_operand<D>(q1, row_of(a.q1), ok, half);
  load_row_operand<D>(q2, row_of(a.q2), ok, half);
  const long long ri = (long long)bh * a.NQ + row;
  load_row_operand<DV>(go, a.dout + (ok ? ri * DV : 0), ok, half);
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

  f32x16 g1[D / 32], g2[D / 32];
#pragma unroll
  for (int n = 0; n < D / 32; ++n) {
    g1[n] = zero16();
    g2[n] = zero16();
  }
  // 2^lift times the sum of P_2 (dP - D_2) of every lane, in LDS: the two registers spill at d 64/128
  __shared__ double dl[C::NT];
  dl[tid] = 0.;

  const uint32_t bk1 = (uint32_t)a.k1.sn * 2u, bk2 = (uint32_t)a.k2.sn * 2u, bv = (uint32_t)a.v.sn * 2u;
  const uint16_t* k1 = a.k1.p + (long long)b * a.k1.sb + (long long)hk * a.k1.sh;
  const uint16_t* k2 = a.k2.p + (long long)b * a.k2.sb + (long long)hk * a.k2.sh;
  const uint16_t* vv = a.v.p + (long long)b * a.v.sb + (long long)hk * a.v.sh;
  const DiffDma<D, DV, C::NT> dma(tid, bk1, bk2, bv);
  const TrCols<D> tr(lane);
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
    constexpr int J1 = KD, J2 = J1 + KD, J3 = J2 + KV, J4 = J3 + 4 * ND, LA = C::LA_Q;
    bf16x8 buf[J4];   // streamed operands, read LA of them ahead of their MFMAs
    auto rd = [&](int j) {
      if (j < J2) buf[j] = lds_row8<C::CD>(stage + j / KD * kDiffTile * C::CD, lane & 31, 2 * (j % KD) + half);
      else if (j < J3) buf[j] = lds_row8<C::CV>(stage + 2 * kDiffTile * C::CD, lane & 31, 2 * (j - J2) + half);
      else if (j < J4)   // [k-block][map][columns]
        buf[j] = tr.read(stage, (j - J3) / ND % 2 * kDiffTile * C::CD * 16, (j - J3) % ND, (j - J3) / (2 * ND));
    };
    f32x16 s1 = zero16(), s2 = zero16(), dp = zero16();
    float e1[16], e2[16];
    const bool mask = k0 + kDiffTile > wave_min;
    auto hide = [&](f32x16& s) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = k0 + 8 * (i >> 2) + 4 * half + (i & 3) < limit ? s[i] : kNegInf;
    };
    diff_pin();
#pragma unroll
    for (int j = 0; j < LA; ++j) rd(j);
    diff_pin();
#pragma unroll
    for (int j = 0; j < J1; ++j) {
      rd(j + LA);
      s1 = mfma32(buf[j], q1[j], s1);
      diff_pin();
    }
    if (mask) hide(s1);
    diff_pin();
#pragma unroll
    for (int j = J1; j < J2; ++j) {
      rd(j + LA);
      s2 = mfma32(buf[j], q2[j - J1], s2);
#pragma unroll
      for (int i = 16 * (j - J1) / KD; i < 16 * (j - J1 + 1) / KD; ++i)
        e1[i] = exp2_fast(__builtin_fmaf(s1[i], c, -ls1));
      diff_pin();
    }
    if (mask) hide(s2);
    diff_pin();
#pragma unroll
    for (int j = J2; j < J3; ++j) {
      rd(j + LA);
      dp = mfma32(buf[j], go[j - J2], dp);
#pragma unroll
      for (int i = 16 * (j - J2) / KV; i < 16 * (j - J2 + 1) / KV; ++i)
        e2[i] = exp2_fast(__builtin_fmaf(s2[i], c, -ls2));
      diff_pin();
    }
    bf16x8 a1[2], a2[2];
    float dt = 0.f;
    auto grad = [&](int i) {
      e1[i] *= dp[i] - d1;
      e2[i] *= dp[i] - d2;
      dt += e2[i];
      if (i % 8 == 7) {
        a1[i / 8] = pack8(e1 + i - 7);
        a2[i / 8] = pack8(e2 + i - 7);
      }
    };
#pragma unroll
    for (int i = 0; i < 8; ++i) grad(i);
    diff_pin();
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int j = J3; j < J4; ++j) {
      rd(j + LA);
      const int x = j - J3, u = x / (2 * ND), n = x % ND;
      if (x / ND % 2 == 0) g1[n] = mfma32(a1[u], buf[j], g1[n]);
      else g2[n] = mfma32(a2[u], buf[j], g2[n]);
      if (u == 0) {
#pragma unroll
        for (int i = 8 * x / (2 * ND); i < 8 * (x + 1) / (2 * ND); ++i) grad(8 + i);
      }
      diff_pin();
    }
    __builtin_amdgcn_s_setprio(0);
    lds_add_f64(&dl[tid], (double)dt);
  };

  stream_tiles<C::STAGES_Q, 1, C::STAGE, DiffDma<D, DV, C::NT>::NCH>(st0, st1, st2, t_begin, t_end, load, tile);

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
  if (o1) write_grad<D>(o1, as_bf16, g1, rows, rw, a.NQ, a.scale, lane);
  if (o2) write_grad<D>(o2, as_bf16, g2, rows, rw, a.NQ, -a.scale * lam, lane);
  if (a.dlam) {
    const double part = __builtin_ldexp(dl[tid], -lift) + (half == 0 && blockIdx.y == 0 ? (double)d2 : 0.);   // D_2 once a row
    write_dlam_part(a.dlam_part + ((long long)bh * T + blk) * a.q_splits + blockIdx.y, red,
                    !ok ? 0. : (lane & 1) ? -part : part, tid);
  }
}

// ---------------------------------------------------------------------------
// dK, dV: workgroup = 128 keys of one key head, streams tiles [Q_1 | Q_2 | dO]
// of 32 rows, one query head of the group after the other, with their
// prepared statistics.
// ---------------------------------------------------------------------------
template <int D, int DV, int PART>
__global__ void __launch_bounds__(kThreads, (DiffBwdCfg<D, DV, PART>::WAVES_K)) diff_bwd_dkv_kernel(const DiffArgs a) {
  using C = DiffBwdCfg<D, DV, PART>;
  constexpr bool WANT_K = (PART & 1) != 0, WANT_V = (PART & 2) != 0;
  constexpr int KD = D / 16, KV = DV / 16, ND = D / 32, NV = DV / 32;
  __shared__ u32x4 st0[C::TR_K * (C::STAGE + C::STATS)];
  __shared__ u32x4 st1[C::TR_K * (C::STAGE + C::STATS)];
  __shared__ u32x4 st2[C::STAGES_K == 3 ? C::TR_K * (C::STAGE + C::STATS) : 1];
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
  const int per = kb0 < klen ? t_all - t_first : 0;
  int s_end = per * G, s_begin = 0;   // steps: one row tile of one head each
  if (a.k_splits > 1) {
    const int each = (s_end + a.k_splits - 1) / a.k_splits;
    s_begin = min(s_end, (int)blockIdx.y * each);
    s_end = min(s_end, s_begin + each);
  }
  const int g_begin = per ? s_begin / per : 0, t_begin = s_begin - g_begin * per;

  const bool ok = key < klen;
  bf16x8 k1[D / 16], k2[D / 16], vv[DV / 16];
  auto row_of = [&](const DiffRows& x) {
    return x.p + (ok ? (long long)b * x.sb + (long long)hk * x.sh + (long long)key * x.sn : 0);
  };
  load_row_operand<D>(k1, row_of(a.k1), ok, half);
  load_row_operand<D>(k2, row_of(a.k2), ok, half);
  if constexpr (WANT_K) load_row_operand<DV>(vv, row_of(a.v), ok, half);
  wait_vmem();   // before the tile loop: a first use inside it would wait on every trip

  f32x16 g1[D / 32], g2[D / 32], gv[DV / 32];
#pragma unroll
  for (int n = 0; n < D / 32; ++n) {
    g1[n] = zero16();
    g2[n] = zero16();
  }
#pragma unroll
  for (int n = 0; n < DV / 32; ++n) gv[n] = zero16();

  const uint32_t bq1 = (uint32_t)a.q1.sn * 2u, bq2 = (uint32_t)a.q2.sn * 2u, bo = (uint32_t)DV * 2u;
  const DiffDma<D, DV, C::NT> dma(tid, bq1, bq2, bo);
  const TrCols<D> trd(lane);
  const TrCols<DV> trv(lane);
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
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void*)(reinterpret_cast<float*>(stage + C::STAGE) + 32 * wave),
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
    constexpr int J1 = KD, J2 = J1 + KD, J3 = J2 + (WANT_K ? KV : 0), J4 = J3 + (WANT_V ? 2 * NV : 0);
    constexpr int J5 = J4 + (WANT_K ? 4 * ND : 0), LA = C::LA_K;
    bf16x8 buf[J5];   // streamed operands, read LA of them ahead of their MFMAs
    auto rd = [&](int j) {
      if (j < J2) buf[j] = lds_row8<C::CD>(stage + j / KD * kDiffTile * C::CD, lane & 31, 2 * (j % KD) + half);
      else if (j < J3) buf[j] = lds_row8<C::CV>(stage + 2 * kDiffTile * C::CD, lane & 31, 2 * (j - J2) + half);
      else if (j < J4) buf[j] = trv.read(stage, 2 * kDiffTile * C::CD * 16, (j - J3) % NV, (j - J3) / NV);
      else if (j < J5)   // [map][k-block][columns]
        buf[j] = trd.read(stage, (j - J4) / (2 * ND) * kDiffTile * C::CD * 16, (j - J4) % ND, (j - J4) / ND % 2);
    };
    const f32x4* st = reinterpret_cast<const f32x4*>(stage + C::STAGE);
    f32x4 ga[4], gb[4];   // statistics of four elements, read one such group ahead of their use
    auto rd_st = [&](f32x4 (&g)[4], int which, int i) {
      if (i < 16) g[i >> 2] = st[8 * which + 2 * (i >> 2) + half];
    };
    f32x16 s1 = zero16(), s2 = zero16(), dp;
    float e1[16], e2[16], p[16];
    const bool mask = (a.causal && kw + 31 > r0 + off) || kw + 32 > klen;
    auto hide = [&](f32x16& s) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const bool seen = ok && (!a.causal || key <= r0 + 8 * (i >> 2) + 4 * half + (i & 3) + off);
        s[i] = seen ? s[i] : kNegInf;
      }
    };
    diff_pin();
#pragma unroll
    for (int j = 0; j < LA; ++j) rd(j);
    diff_pin();
#pragma unroll
    for (int j = 0; j < J1; ++j) {
      rd(j + LA);
      s1 = mfma32(buf[j], k1[j], s1);
      diff_pin();
    }
    rd_st(ga, 0, 0);
    if (mask) hide(s1);
    diff_pin();
#pragma unroll
    for (int j = J1; j < J2; ++j) {
      rd(j + LA);
      s2 = mfma32(buf[j], k2[j - J1], s2);
#pragma unroll
      for (int i = 16 * (j - J1) / KD; i < 16 * (j - J1 + 1) / KD; ++i) {
        if (i % 4 == 0) rd_st(ga, 0, i + 4);
        e1[i] = exp2_fast(__builtin_fmaf(s1[i], c, -ga[i >> 2][i & 3]));   // P_1
      }
      diff_pin();
    }
    rd_st(gb, 1, 0);
    if constexpr (WANT_K && C::START_D) {
#pragma unroll
      for (int i = 0; i < 16; i += 4) rd_st(ga, 2, i);
#pragma unroll
      for (int i = 0; i < 16; ++i) dp[i] = ga[i >> 2][i & 3];
    } else {
      dp = zero16();
    }
    if (mask) hide(s2);
    diff_pin();
    bf16x8 ap[2];
    auto second = [&](int i) {
      if (i % 4 == 0) rd_st(gb, 1, i + 4);
      e2[i] = exp2_fast(__builtin_fmaf(s2[i], c, -gb[i >> 2][i & 3]));   // |lam| P_2
      if constexpr (WANT_V) {
        p[i] = __builtin_fmaf(nsign, e2[i], e1[i]);
        if (i % 8 == 7) ap[i / 8] = pack8(p + i - 7);
      }
    };
    if constexpr (!WANT_K) {
#pragma unroll
      for (int i = 0; i < 8; ++i) second(i);
      diff_pin();
    }
#pragma unroll
    for (int j = J2; j < J3; ++j) {
      rd(j + LA);
      dp = mfma32(buf[j], vv[j - J2], dp);
#pragma unroll
      for (int i = 16 * (j - J2) / KV; i < 16 * (j - J2 + 1) / KV; ++i) second(i);
      diff_pin();
    }
    bf16x8 a1[2], a2[2];
    auto grad = [&](int i) {
      if (i % 4 == 0) {
        rd_st(gb, 3, i + 4);
        if (!C::START_D) rd_st(ga, 2, i + 4);
      }
      const float y = C::START_D ? dp[i] : dp[i] + ga[i >> 2][i & 3];   // dP - D_1
      e1[i] *= y;
      e2[i] *= __builtin_fmaf(nsign, y, gb[i >> 2][i & 3]);
      if (i % 8 == 7) {
        a1[i / 8] = pack8(e1 + i - 7);
        a2[i / 8] = pack8(e2 + i - 7);
      }
    };
    if constexpr (WANT_K) {
      rd_st(gb, 3, 0);
      if (!C::START_D) rd_st(ga, 2, 0);
      diff_pin();
      if constexpr (!WANT_V) {
#pragma unroll
        for (int i = 0; i < 16; ++i) grad(i);
        diff_pin();
      }
    }
    if constexpr (C::WAVES_K == 2) __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int j = J3; j < J4; ++j) {
      rd(j + LA);
      const int x = j - J3;
      gv[x % NV] = mfma32(ap[x / NV], buf[j], gv[x % NV]);
      if constexpr (WANT_K) {
#pragma unroll
        for (int i = 16 * x / (2 * NV); i < 16 * (x + 1) / (2 * NV); ++i) grad(i);
      } else if (x < NV) {
#pragma unroll
        for (int i = 8 * x / NV; i < 8 * (x + 1) / NV; ++i) second(8 + i);
      }
      diff_pin();
    }
#pragma unroll
    for (int j = J4; j < J5; ++j) {
      rd(j + LA);
      const int x = j - J4, u = x / ND % 2, n = x % ND;
      if (x < 2 * ND) g1[n] = mfma32(a1[u], buf[j], g1[n]);
      else g2[n] = mfma32(a2[u], buf[j], g2[n]);
      diff_pin();
    }
    if constexpr (C::WAVES_K == 2) __builtin_amdgcn_s_setprio(0);
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

  stream_tiles<C::STAGES_K, C::TR_K, C::STAGE + C::STATS, DiffDma<D, DV, C::NT>::NCH + 1>(st0, st1, st2, s_begin, s_end, load, tile);

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
  if (WANT_K && o1) write_grad<D>(o1, as_bf16, g1, rows, kw, a.NK, a.scale, lane);
  if (WANT_K && o2) write_grad<D>(o2, as_bf16, g2, rows, kw, a.NK, a.scale, lane);
  if (WANT_V && o3) write_grad<DV>(o3, as_bf16, gv, rows, kw, a.NK, 1.f, lane);
}

}  // namespace streamkl
