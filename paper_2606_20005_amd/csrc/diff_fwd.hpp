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
// Rounding: P to bf16 (each term of O is off by at most 2^-8 of itself), O to
// bf16 once at the end; everything else is float32. The sum l takes the
// float32 p, in chunks of kDiffChunk tiles (over 131072 keys the log-sum-exps are
// off by 3.3e-7, of which 2.7e-7 are the rounding of a value near 12; in one
// chain by 3.0e-6. Tiles added apart, in float32 or 64 bits, took 1.5 to 2% longer
// at d 128/256): with the rounded ones (two at a time by dot products, half of the
// additions) the log-sum-exps, and with them the recomputed probabilities of
// the backward pass, were off by up to 1e-3.
//
// splits > 1: blockIdx.y takes a contiguous range of the key tiles and leaves
// unnormalised float32 sums and their reference in `part`; a second kernel
// joins them. part: [row][split][map] x dv floats, then [row][split][map] x 2
// (reference, sum), rows in output order (b, h, i).
#pragma once

#include "diff_common.hpp"

namespace streamkl {

constexpr float kDiffSlack = 64.f;
constexpr int kDiffChunk = 16;   // tiles

template <int D, int DV, int RB_, int NW_>
struct DiffFwdCfg {
  static constexpr int RB = RB_, NW = NW_, NT = 64 * NW_;
  static constexpr int GROUPS = NW / 2;               // pairs of waves
  static constexpr int ROWS = 32 * RB * GROUPS;       // query rows per workgroup
  static constexpr int CD = lds_cols(D) / 8;           // chunks of a key row in LDS
  static constexpr int STAGE = DiffDma<D, DV, NT>::CHUNKS;
  static constexpr int XCHG = GROUPS * 256;           // chunks of the exchange of one 32 x 32 block per pair
  // registers: accumulators, resident rows, logits, about 64 for the rest
  static constexpr int REGS = RB * (DV / 2 + D / 4 + 16) + 60 + D / 16;
  static constexpr int WAVES = REGS <= 168 ? 3 : REGS <= 256 ? 2 : 1;   // waves per SIMD
  static constexpr int LA = WAVES == 1 ? 4 : REGS > 248 ? 2 : 3;   // operand reads in flight ahead of their MFMAs
  // three stages where the workgroups that the registers leave room for have room for them too
  static constexpr int LDS2 = (STAGE + (STAGE > XCHG ? STAGE : XCHG)) * 16;
  static constexpr int STAGES = (LDS2 + STAGE * 16) * (4 * WAVES / NW) <= 160 * 1024 ? 3 : 2;
  static constexpr int LDS = LDS2 + (STAGES - 2) * STAGE * 16;
};

template <int D, int DV, int RB, int NW>
__global__ void __launch_bounds__(64 * NW, (DiffFwdCfg<D, DV, RB, NW>::WAVES))
diff_fwd_kernel(const DiffArgs a) {
  using C = DiffFwdCfg<D, DV, RB, NW>;
  constexpr int KS = D / 16, NB = DV / 32;
  __shared__ u32x4 st0[C::STAGE > C::XCHG ? C::STAGE : C::XCHG];
  __shared__ u32x4 st1[C::STAGE];
  __shared__ u32x4 st2[C::STAGES == 3 ? C::STAGE : 1];
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

  // Packed row r of this lane in block x: query i of head h. Formed from `at`,
  // which the epilogue hides from the optimizer: kept through the loop, these
  // would take registers that it has none to spare of.
  struct Row {
    int i, h;
    bool in, ok;   // inside the tensor; and inside its sequence
  };
  auto row_of = [&](int x, int at) {
    const int r = rw + 32 * x + at, i = r / G;
    return Row{i, hk * G + (r - i * G), r < R, r < R && i < qlen};
  };
  int limit[RB];
  bf16x8 q[RB][KS];
  const DiffRows& qv = map ? a.q2 : a.q1;
#pragma unroll
  for (int x = 0; x < RB; ++x) {
    const Row w = row_of(x, lane & 31);
    limit[x] = w.ok ? limit_of(w.i) : klen;   // rows that do not exist take part unmasked, nothing reads them
    const uint16_t* p = qv.p + (w.ok ? (long long)b * qv.sb + (long long)w.h * qv.sh + (long long)w.i * qv.sn : 0);
    load_row_operand<D>(q[x], p, w.ok, half);
  }
  wait_vmem();   // before the tile loop: a first use inside it would wait on every trip

  f32x16 o[RB][NB];
  float m[RB], nu[RB];   // raw maximum at the last rescaling, -u
  float lc[RB], l[RB];   // the sum of this half-wave's keys since the last multiple of kDiffChunk tiles, and up to there
#pragma unroll
  for (int x = 0; x < RB; ++x) {
    m[x] = kNegInf;
    nu[x] = 0.f;
    lc[x] = 0.f;
    l[x] = 0.f;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) o[x][nb] = zero16();
  }
  const float slack = kDiffSlack / c;

  const uint32_t bk1 = (uint32_t)a.k1.sn * 2u, bk2 = (uint32_t)a.k2.sn * 2u, bv = (uint32_t)a.v.sn * 2u;
  const uint16_t* k1 = a.k1.p + (long long)b * a.k1.sb + (long long)hk * a.k1.sh;
  const uint16_t* k2 = a.k2.p + (long long)b * a.k2.sb + (long long)hk * a.k2.sh;
  const uint16_t* vv = a.v.p + (long long)b * a.v.sb + (long long)hk * a.v.sh;
  const DiffDma<D, DV, C::NT> dma(tid, bk1, bk2, bv);
  const TrCols<DV> tr(lane);
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
    const u32x4* kt = stage + map * kDiffTile * C::CD;
    constexpr int vbase = 2 * kDiffTile * C::CD * 16, NR = KS + 2 * NB, LA = C::LA;
    bf16x8 buf[NR];   // streamed operands: key chunks, then value blocks; read LA of them ahead of their MFMAs
    auto rd = [&](int j) {
      if (j < KS) buf[j] = lds_row8<C::CD>(kt, lane & 31, 2 * j + half);
      else if (j < NR) buf[j] = tr.read(stage, vbase, (j - KS) % NB, (j - KS) / NB);
    };
    f32x16 s[RB];
#pragma unroll
    for (int x = 0; x < RB; ++x) s[x] = zero16();
    diff_pin();
#pragma unroll
    for (int j = 0; j < LA; ++j) rd(j);
    diff_pin();
#pragma unroll
    for (int j = 0; j < KS; ++j) {
      rd(j + LA);
#pragma unroll
      for (int x = 0; x < RB; ++x) s[x] = mfma32(buf[j], q[x][j], s[x]);
      diff_pin();
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
          lc[x] *= f;
          l[x] *= f;
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) o[x][nb] *= f;
        }
      }
    }
    diff_pin();
    float e[RB][16];
    bf16x8 p[RB][2];
    auto prob = [&](int x, int i) {
      e[x][i] = exp2_fast(__builtin_fmaf(s[x][i], c, nu[x]));
      lc[x] += e[x][i];
      if (i % 8 == 7) p[x][i / 8] = pack8(e[x] + i - 7);
    };
#pragma unroll
    for (int x = 0; x < RB; ++x)
#pragma unroll
      for (int i = 0; i < 8; ++i) prob(x, i);
    diff_pin();
    // The second half of the exponentials beside the products of the first.
    // Raised priority: the products go out as soon as the matrix pipe takes
    // them, and the other wave of the SIMD does its vector work in between (5 to
    // 9% of the whole at d 64/64, 64/128 and 128/64; none where raised in the second
    // half alone).
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      rd(KS + nb + LA);
#pragma unroll
      for (int x = 0; x < RB; ++x) o[x][nb] = mfma32(buf[KS + nb], p[x][0], o[x][nb]);
#pragma unroll
      for (int y = 8 * RB * nb / NB; y < 8 * RB * (nb + 1) / NB; ++y) prob(y / 8, 8 + y % 8);
      diff_pin();
    }
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      rd(KS + NB + nb + LA);
#pragma unroll
      for (int x = 0; x < RB; ++x) o[x][nb] = mfma32(buf[KS + NB + nb], p[x][1], o[x][nb]);
      diff_pin();
    }
    __builtin_amdgcn_s_setprio(0);
    if (t % kDiffChunk == kDiffChunk - 1) {
#pragma unroll
      for (int x = 0; x < RB; ++x) {
        l[x] += lc[x];
        lc[x] = 0.f;
      }
    }
  };

  stream_tiles<C::STAGES, 1, C::STAGE, DiffDma<D, DV, C::NT>::NCH>(st0, st1, st2, t_begin, t_end, load, tile);

#pragma unroll
  for (int x = 0; x < RB; ++x) {
    l[x] += lc[x];
    l[x] += __shfl_xor(l[x], 32);
  }

  Row row[RB];
#pragma unroll
  for (int x = 0; x < RB; ++x) row[x] = row_of(x, opaque(lane) & 31);
  auto out_row = [&](int x) { return ((long long)b * a.H + row[x].h) * a.NQ + row[x].i; };
  if (a.splits > 1) {
    const long long rows = (long long)a.B * a.H * a.NQ;
#pragma unroll
    for (int x = 0; x < RB; ++x) {
      if (!row[x].ok) continue;
      const long long at = (out_row(x) * a.splits + blockIdx.y) * 2 + map;
      float* po = a.part + at * DV;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int qd = 0; qd < 4; ++qd) {
          const int col = 32 * nb + 8 * qd + 4 * half;
          *reinterpret_cast<f32x4*>(po + col) =
              f32x4{o[x][nb][4 * qd], o[x][nb][4 * qd + 1], o[x][nb][4 * qd + 2], o[x][nb][4 * qd + 3]};
        }
      if (half == 0) {
        float* pm = a.part + rows * a.splits * 2 * DV + at * 2;
        pm[0] = m[x] == kNegInf ? kNegInf : -nu[x];
        pm[1] = l[x];
      }
    }
    return;
  }

  float* lse = map ? a.lse2 : a.lse1;
  auto store4 = [&](uint16_t* dst, const float (&v)[4]) {
    bf16x4 r;
#pragma unroll
    for (int j = 0; j < 4; ++j) r[j] = (__bf16)v[j];
    *reinterpret_cast<bf16x4*>(dst) = r;
  };
#pragma unroll
  for (int x = 0; x < RB; ++x) {
    const bool in = row[x].in, ok = row[x].ok;
    const float f = l[x] > 0.f || l[x] != l[x] ? 1.f / l[x] : 0.f;   // 0 for rows that see nothing
    const float lam = in ? a.lam[row[x].h] : 0.f;
    if (lse && half == 0 && in)
      lse[out_row(x)] = !ok || l[x] == 0.f ? kNegInf : diff_lse(l[x], -nu[x]);
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
          for (int j = 0; j < 4; ++j) v[j] = ok ? o[x][nb][4 * qd + j] * f : 0.f;
          slot[64 * qd] = f32x4{v[0], v[1], v[2], v[3]};
          const int col = 32 * nb + 8 * qd + 4 * half;
          if (a.out2 && in) store4(a.out2 + out_row(x) * DV + col, v);
        }
      }
      __syncthreads();
      if (map == 0) {
#pragma unroll
        for (int qd = 0; qd < 4; ++qd) {
          const f32x4 o2 = slot[64 * qd];
          float v[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) v[j] = ok ? __builtin_fmaf(-lam, o2[j], o[x][nb][4 * qd + j] * f) : 0.f;
          const int col = 32 * nb + 8 * qd + 4 * half;
          if (in) store4(a.out + out_row(x) * DV + col, v);
        }
      }
    }
  }
}

}  // namespace streamkl
