// Forward kernel of differential attention.
//
// A workgroup owns a block of query rows of one (sequence, key head) and
// streams the key tiles of both maps and the value tile through LDS. The
// query rows of the G heads that share the key head are packed, row r = i G + g,
// so that a cache is read once per key head however few rows there are.
//
// Each wave works on ONE map: waves 2 w and 2 w + 1 hold the same 32 RB rows,
// the first of map 1, the second of map 2. A wave that held both maps for
// half as many rows would issue the same MFMAs but read each value operand
// from LDS for half as many rows: per 32 keys and 24 MFMAs of d 64, dv 128 it
// reads 12 KB this way and 16 KB the other way, and LDS delivers 128 bytes a
// clock to four SIMDs.
//
// Per tile: S^T = K Q^T on the 32x32x16 MFMA (A = key rows from LDS, B =
// resident query rows), so that a lane owns one row (l % 32) and 16 keys;
// p = 2^(c s - u), c = scale log2 e; P^T, rounded to bf16, is the B operand of
// O^T += V^T P^T as it lies in the registers (the 16 keys of a k-block in the
// order the accumulator has them), V^T comes from the row-major value tile by
// transpose reads. O^T again has the row in the lane, so that rescaling needs
// no exchange.
//
// The exponent reference u is kept as long as no logit rises more than
// kDiffSlack doublings above it: sums and products stay in the float32 range
// with any such reference and are exact relative to it, and a bf16 p has the
// same relative precision at any size. So the rescaling of O (DV / 2 multiplies
// a lane and block) runs about once per row, not once per tile.
//
// Rounding: P to bf16 (each term of O is off by at most 2^-8 of itself, the
// sum l keeps the float32 p), O to bf16 once at the end; everything else is
// float32.
//
// splits > 1: blockIdx.y takes a contiguous range of the key tiles and leaves
// unnormalised float32 sums and their reference in `part`; a second kernel
// joins them. part: [row][split][map] x dv floats, then [row][split][map] x 2
// (reference, sum), rows in output order (b, h, i).
#pragma once

#include "diff_common.hpp"

namespace streamkl {

constexpr float kDiffSlack = 64.f;

template <int D, int DV, int RB_, int NW_>
struct DiffFwdCfg {
  static constexpr int RB = RB_, NW = NW_, NT = 64 * NW_;
  static constexpr int GROUPS = NW / 2;               // pairs of waves
  static constexpr int ROWS = 32 * RB * GROUPS;       // query rows per workgroup
  static constexpr int STAGE = DiffDma<D, DV, NT>::CHUNKS;
  static constexpr int XCHG = GROUPS * 256;           // chunks of the exchange of one 32 x 32 block per pair
  // registers: accumulators, resident rows, logits, about 64 for the rest
  static constexpr int REGS = RB * (DV / 2 + D / 4 + 16) + 64;
  static constexpr int WAVES = REGS <= 256 ? 2 : 1;   // waves per SIMD
};

template <int D, int DV, int RB, int NW>
__global__ void __launch_bounds__(64 * NW, (DiffFwdCfg<D, DV, RB, NW>::WAVES))
diff_fwd_kernel(const DiffArgs a) {
  using C = DiffFwdCfg<D, DV, RB, NW>;
  constexpr int KS = D / 16, NB = DV / 32;
  __shared__ u32x4 st0[C::STAGE > C::XCHG ? C::STAGE : C::XCHG];
  __shared__ u32x4 st1[C::STAGE];
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), map = wave & 1, group = wave >> 1;
  const int G = a.H / a.HK, R = a.NQ * G, T = (R + C::ROWS - 1) / C::ROWS;
  int bh, blk;
  if (a.causal) {
    causal_block(blockIdx.x, gridDim.x, T, kCus * 4 * C::WAVES / NW, bh, blk);
    blk = T - 1 - blk;   // rank 0: the last rows, the longest
  } else {
    const int l = xcd_logical(blockIdx.x, gridDim.x);
    bh = l / T;
    blk = l - bh * T;
  }
  const int b = bh / a.HK, hk = bh - b * a.HK;
  const int qlen = clamp_len(a.q_len, b, a.NQ), klen = clamp_len(a.kv_len, b, a.NK);
  const int off = klen - qlen;   // row i stands at key off + i
  const float c = a.scale * kLog2e;

  // keys that the rows of the block and of this wave can see
  auto limit_of = [&](int i) { return a.causal ? min(max(off + i + 1, 0), klen) : klen; };
  const int rblk = blk * C::ROWS, rw = rblk + 32 * RB * group;
  const int ilast = min((min(rblk + C::ROWS, R) - 1) / G, qlen - 1);
  const int i0w = rw / G, i1w = min((min(rw + 32 * RB, R) - 1) / G, qlen - 1);
  int t_end = rblk / G < qlen ? (limit_of(ilast) + kDiffTile - 1) / kDiffTile : 0, t_begin = 0;
  if (a.splits > 1) {
    const int all = (klen + kDiffTile - 1) / kDiffTile, per = (all + a.splits - 1) / a.splits;
    t_begin = (int)blockIdx.y * per;
    t_end = min(t_end, t_begin + per);
  }
  const bool live = rw < R && i0w < qlen;   // some row of the wave exists
  const int wave_min = limit_of(i0w), wave_max = live ? limit_of(i1w) : 0;

  // resident rows
  int limit[RB], row_i[RB], row_h[RB];
  bool row_ok[RB];
  bf16x8 q[RB][KS];
  const DiffRows& qv = map ? a.q2 : a.q1;
#pragma unroll
  for (int x = 0; x < RB; ++x) {
    const int r = rw + 32 * x + (lane & 31);
    row_i[x] = r / G;
    row_h[x] = hk * G + (r - row_i[x] * G);
    row_ok[x] = r < R && row_i[x] < qlen;
    limit[x] = row_ok[x] ? limit_of(row_i[x]) : klen;   // rows that do not exist take part unmasked, nothing reads them
    const uint16_t* p = qv.p + (row_ok[x] ? (long long)b * qv.sb + (long long)row_h[x] * qv.sh +
                                                (long long)row_i[x] * qv.sn : 0);
    load_row_operand<D>(q[x], p, row_ok[x], half, a.d);
  }
  wait_vmem();   // before the tile loop: a first use inside it would wait on every trip

  f32x16 o[RB][NB];
  float m[RB], nu[RB], l[RB];   // raw maximum at the last rescaling, -u, the sum of this half-wave's keys
#pragma unroll
  for (int x = 0; x < RB; ++x) {
    m[x] = kNegInf;
    nu[x] = 0.f;
    l[x] = 0.f;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) o[x][nb] = zero16();
  }
  const float slack = kDiffSlack / c;

  const uint32_t bk1 = (uint32_t)a.k1.sn * 2u, bk2 = (uint32_t)a.k2.sn * 2u, bv = (uint32_t)a.v.sn * 2u;
  const uint16_t* k1 = a.k1.p + (long long)b * a.k1.sb + (long long)hk * a.k1.sh;
  const uint16_t* k2 = a.k2.p + (long long)b * a.k2.sb + (long long)hk * a.k2.sh;
  const uint16_t* vv = a.v.p + (long long)b * a.v.sb + (long long)hk * a.v.sh;
  const DiffDma<D, DV, C::NT> dma(tid, a.d, a.dv, bk1, bk2, bv);
  const TrCols<DV> tr(lane);
  auto load = [&](int t, u32x4* stage) {
    dma.issue(tile_rsrc(k1, t * kDiffTile, klen, bk1, a.d), tile_rsrc(k2, t * kDiffTile, klen, bk2, a.d),
              tile_rsrc(vv, t * kDiffTile, klen, bv, a.dv), stage, wave);
  };

  auto tile = [&](const u32x4* stage, int t) {
    const int k0 = t * kDiffTile;
    if (k0 >= wave_max) return;
    const u32x4* kt = stage + map * kDiffTile * (D / 8);
    f32x16 s[RB];
#pragma unroll
    for (int x = 0; x < RB; ++x) s[x] = zero16();
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const bf16x8 k = lds_row8<D / 8>(kt, lane & 31, 2 * ks + half);
#pragma unroll
      for (int x = 0; x < RB; ++x) s[x] = mfma32(k, q[x][ks], s[x]);
    }
    if (k0 + kDiffTile > wave_min) {
#pragma unroll
      for (int x = 0; x < RB; ++x)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[x][i] = k0 + 8 * (i >> 2) + 4 * half + (i & 3) < limit[x] ? s[x][i] : kNegInf;
    }
    float top[RB];
    bool rise = false;
#pragma unroll
    for (int x = 0; x < RB; ++x) {
      top[x] = s[x][0];
#pragma unroll
      for (int i = 1; i < 16; i += 2) top[x] = fmaxf(fmaxf(top[x], s[x][i]), s[x][i < 15 ? i + 1 : 15]);
      rise = rise || top[x] > m[x] + slack;
    }
    if (__builtin_amdgcn_ballot_w64(rise)) {
#pragma unroll
      for (int x = 0; x < RB; ++x) {
        const float both = fmaxf(top[x], __shfl_xor(top[x], 32));   // the two half-waves share a row's reference
        if (both > m[x] + slack) {
          const float f = m[x] == kNegInf ? 0.f : exp2_fast(c * (m[x] - both));
          m[x] = both;
          nu[x] = -c * both;
          l[x] *= f;
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) o[x][nb] *= f;
        }
      }
    }
    bf16x8 p[RB][2];
#pragma unroll
    for (int x = 0; x < RB; ++x) {
      float e[16], sum = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        e[i] = exp2_fast(__builtin_fmaf(s[x][i], c, nu[x]));
        sum += e[i];
      }
      l[x] += sum;
      p[x][0] = pack8(e);
      p[x][1] = pack8(e + 8);
    }
    constexpr int vbase = 2 * kDiffTile * (D / 8) * 16;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const bf16x8 v = tr.read(stage, vbase, nb, u);
#pragma unroll
        for (int x = 0; x < RB; ++x) o[x][nb] = mfma32(v, p[x][u], o[x][nb]);
      }
  };

  if (t_begin < t_end) load(t_begin, st0);
  wait_vmem();
  barrier_no_fence();
  auto step = [&](const u32x4* cur, u32x4* nxt, int t) {
    if (t + 1 < t_end) load(t + 1, nxt);
    tile(cur, t);
    wait_vmem();
    wait_lds();
    barrier_no_fence();
  };
  for (int t = t_begin; t < t_end; t += 2) {
    step(st0, st1, t);
    if (t + 1 < t_end) step(st1, st0, t + 1);
  }

#pragma unroll
  for (int x = 0; x < RB; ++x) l[x] += __shfl_xor(l[x], 32);

  auto out_row = [&](int x) { return ((long long)b * a.H + row_h[x]) * a.NQ + row_i[x]; };
  if (a.splits > 1) {
    const long long rows = (long long)a.B * a.H * a.NQ;
#pragma unroll
    for (int x = 0; x < RB; ++x) {
      if (!row_ok[x]) continue;
      const long long at = (out_row(x) * a.splits + blockIdx.y) * 2 + map;
      float* po = a.part + at * a.dv;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int qd = 0; qd < 4; ++qd) {
          const int col = 32 * nb + 8 * qd + 4 * half;
          if (col < a.dv)
            *reinterpret_cast<f32x4*>(po + col) =
                f32x4{o[x][nb][4 * qd], o[x][nb][4 * qd + 1], o[x][nb][4 * qd + 2], o[x][nb][4 * qd + 3]};
        }
      if (half == 0) {
        float* pm = a.part + rows * a.splits * 2 * a.dv + at * 2;
        pm[0] = m[x] == kNegInf ? kNegInf : -nu[x];
        pm[1] = l[x];
      }
    }
    return;
  }

  float f[RB];   // 1 / l, times lam for map 2 after out2 is written; 0 for rows that see nothing
#pragma unroll
  for (int x = 0; x < RB; ++x) f[x] = l[x] > 0.f || l[x] != l[x] ? 1.f / l[x] : 0.f;
  {
    float* lse = map ? a.lse2 : a.lse1;
    if (lse && half == 0) {
#pragma unroll
      for (int x = 0; x < RB; ++x)
        if (rw + 32 * x + (lane & 31) < R)
          lse[out_row(x)] = !row_ok[x] || m[x] == kNegInf ? kNegInf : (log2f(l[x]) - nu[x]) * kLn2;
    }
  }
  auto store4 = [&](uint16_t* dst, const float (&v)[4]) {
    bf16x4 r;
#pragma unroll
    for (int j = 0; j < 4; ++j) r[j] = (__bf16)v[j];
    *reinterpret_cast<bf16x4*>(dst) = r;
  };
  float lam[RB];
#pragma unroll
  for (int x = 0; x < RB; ++x) lam[x] = rw + 32 * x + (lane & 31) < R ? a.lam[row_h[x]] : 0.f;
#pragma unroll
  for (int x = 0; x < RB; ++x) {
    const bool in = rw + 32 * x + (lane & 31) < R;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      // the wave of map 2 hands its block to the wave of map 1, lane by lane
      f32x4* slot = reinterpret_cast<f32x4*>(st0) + group * 256 + lane;
      __syncthreads();
      if (map == 1) {
#pragma unroll
        for (int qd = 0; qd < 4; ++qd) {
          float v[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) v[j] = row_ok[x] ? o[x][nb][4 * qd + j] * f[x] : 0.f;
          slot[64 * qd] = f32x4{v[0], v[1], v[2], v[3]};
          const int col = 32 * nb + 8 * qd + 4 * half;
          if (a.out2 && in && col < a.dv) store4(a.out2 + out_row(x) * a.dv + col, v);
        }
      }
      __syncthreads();
      if (map == 0) {
#pragma unroll
        for (int qd = 0; qd < 4; ++qd) {
          const f32x4 o2 = slot[64 * qd];
          float v[4];
#pragma unroll
          for (int j = 0; j < 4; ++j)
            v[j] = row_ok[x] ? __builtin_fmaf(-lam[x], o2[j], o[x][nb][4 * qd + j] * f[x]) : 0.f;
          const int col = 32 * nb + 8 * qd + 4 * half;
          if (in && col < a.dv) store4(a.out + out_row(x) * a.dv + col, v);
        }
      }
    }
  }
}

}  // namespace streamkl
