// Pieces of the differential-attention backward kernels with 16 keys or rows a
// wave, on the 16x16x32 MFMA (diff_bwd_keys16.hpp, diff_bwd_rows16.hpp).
//
// A 16x16 result has index 4 quad + i of its first operand in register i and
// lane % 16 of the second in the lane (quad = lane / 16); a tile of 32 streamed
// rows gives two of them. A lane's eight values are, as they lie, one operand
// of an MFMA over the 32 rows, in the order 4 quad + 0..3, 16 + 4 quad + 0..3;
// transpose reads deliver the other operand in that order.
#pragma once

#include "diff_bwd.hpp"

namespace streamkl {

__device__ __forceinline__ f32x4 mfma16(const bf16x8& a, const bf16x8& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// LDS stages of a workgroup of four waves, two of them on a CU; tiles with EXTRA further chunks.
template <int D, int DV, int EXTRA>
struct Diff16Cfg {
  static constexpr int NT = kThreads, ROWS = 64;
  static constexpr int CD = lds_cols(D) / 8, CV = lds_cols(DV) / 8;
  using Dma = DiffDma<D, DV, NT, true>;
  static constexpr int STAGE = Dma::CHUNKS + EXTRA;
  static constexpr int ROOM = 79 * 1024, TILE = STAGE * 16;
  // two tiles a stage where they fit twice (keys, d 64/128: 423 us with one, 400 with two, eight waves), else three stages
  static constexpr int TR = 4 * TILE <= ROOM ? 2 : 1, STAGES = 3 * TR * TILE <= ROOM ? 3 : 2;
  static constexpr int LA = 3;   // operand reads in flight; four spill (keys, d 96/192) and gain nothing
};

// Places of a lane's operands in a matrix of D columns: the chunk of row
// lane % 16 and step ks, and the byte offset of the transpose read of 16
// columns. A second block of 16 rows lies a constant further. Hidden from the
// optimizer, which would form them anew for every read.
template <int D>
struct Places16 {
  static constexpr int CPR = lds_cols(D) / 8;
  int row[D / 32], col[D / 16];
  __device__ __forceinline__ explicit Places16(int lane) {
    const int quad = lane >> 4, l = lane & 15, r = 4 * quad + (l >> 2);
#pragma unroll
    for (int ks = 0; ks < D / 32; ++ks) row[ks] = opaque(l * CPR + ((4 * ks + quad) ^ swz16<CPR>(l)));
#pragma unroll
    for (int n = 0; n < D / 16; ++n)
      col[n] = opaque((r * CPR + ((2 * n + ((l >> 1) & 1)) ^ swz16<CPR>(r))) * 16 + (l & 1) * 8);
  }
  // operand of rows 16 x .. 16 x + 15, step ks; base: chunks before the matrix
  __device__ __forceinline__ bf16x8 rows(const u32x4* buf, int base, int ks, int x) const {
    return __builtin_bit_cast(bf16x8, buf[row[ks] + base + 16 * x * CPR]);
  }
  // operand of columns 16 n .. 16 n + 15 over all 32 rows
  __device__ __forceinline__ bf16x8 cols(const u32x4* buf, int base, int n) const {
    return cat8(lds_tr4_at(buf, col[n] + 16 * base), lds_tr4_at(buf, col[n] + 16 * base + 256 * CPR));
  }
};

// Resident row of lane % 16 as operands; zeros where it does not exist.
template <int K>
__device__ __forceinline__ void load_resident16(bf16x8 (&op)[K], const uint16_t* row, bool ok, int quad) {
  const u32x4* p = reinterpret_cast<const u32x4*>(row);
#pragma unroll
  for (int ks = 0; ks < K; ++ks) op[ks] = __builtin_bit_cast(bf16x8, ok ? p[4 * ks + quad] : u32x4{0u, 0u, 0u, 0u});
}

// Rows base + 4 quad + i, columns 16 n + lane % 16, times s; see write_grad in
// kl_bwd.hpp: adjacent lanes trade values, so that each stores a dword of bf16.
template <int NB>
__device__ __forceinline__ void write_grad16(void* out, bool bf16, const f32x4 (&acc)[NB], size_t rows, int base, int n_rows,
                                             float s, int lane) {
  const int quad = lane >> 4;
  if (bf16) {
    const bool odd = (lane & 1) != 0;
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
      const int row = base + 4 * quad + i + (lane & 1);
      uint32_t* o = reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(out) + (rows + row) * (16 * NB) + (lane & 14));
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        const float v0 = acc[n][i] * s, v1 = acc[n][i + 1] * s;
        const float got = __int_as_float(
            __builtin_amdgcn_update_dpp(0, __float_as_int(odd ? v0 : v1), 0xB1, 0xF, 0xF, true));
        const uint16_t lo = __builtin_bit_cast(uint16_t, (__bf16)(odd ? got : v0));
        const uint16_t hi = __builtin_bit_cast(uint16_t, (__bf16)(odd ? v1 : got));
        if (row < n_rows) o[8 * n] = (uint32_t)lo | ((uint32_t)hi << 16);
      }
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = base + 4 * quad + i;
    if (row < n_rows) {
      float* o = static_cast<float*>(out) + (rows + row) * (16 * NB) + (lane & 15);
#pragma unroll
      for (int n = 0; n < NB; ++n) o[16 * n] = acc[n][i] * s;
    }
  }
}

}  // namespace streamkl
