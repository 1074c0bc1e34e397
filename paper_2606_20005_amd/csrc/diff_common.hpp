// Shared parts of the differential-attention kernels: arguments, tile
// staging from strided rows, operand addressing.
//
//   S_t = s Q_t K_t^T (masked), P_t = softmax(S_t), O_t = P_t V,
//   O = O_1 - lam_h O_2,   t = 1, 2
//
// Query heads share keys and values in groups of G = H / HK consecutive
// heads. Sequence b has q_len[b] rows and kv_len[b] keys (all of them without
// lengths); row i of it sees the keys j < kv_len[b] and, under the causal
// mask, j <= kv_len[b] - q_len[b] + i.
#pragma once

#include "kl_common.hpp"

namespace streamkl {

constexpr int kDiffTile = 32;   // streamed rows per tile: one 32 x 32 MFMA block

// The kernels are built for every head dim (a multiple of 32). In LDS a row
// takes the next multiple of 64 columns, which the swizzles of kl_common.hpp
// need; the columns past its end are written as zeros and never read.
constexpr int lds_cols(int d) { return (d + 63) / 64 * 64; }

// Rows [batch, head, row] with element strides; see streamkl_rows.
struct DiffRows {
  const uint16_t* p;
  long long sb, sh, sn;
};

struct DiffArgs {
  DiffRows q1, k1, q2, k2, v;
  int B, H, HK, NQ, NK, d, dv;
  float scale;
  int causal;
  const float* lam;          // [H]
  const int *q_len, *kv_len; // [B] or null
  // forward
  uint16_t *out, *out2;      // [B, H, NQ, dv]; out2 (O_2) may be null
  float *lse1, *lse2;        // [B, H, NQ], may be null
  int splits;
  float* part;               // splits > 1: see diff_fwd.hpp
  // backward
  const uint16_t* dout;      // [B, H, NQ, dv]
  float* stats;              // prepared row statistics, see diff_bwd.hpp
  double* dlam_part;         // partial sums of dlam
  int q_splits, k_splits;    // ranges of the streamed axis in the query- and the key-owned kernel
  int row_blocks;            // of the query-owned kernel
  float* grad_part;          // their partial gradients where there is more than one
  void *dq1, *dk1, *dq2, *dk2, *dv_out;
  float* dlam;
  int bf16_grads;
  hipStream_t stream;
};

// Nothing moves across: the order of loads, MFMAs and vector work around it is the one written.
__device__ __forceinline__ void diff_pin() { __builtin_amdgcn_sched_barrier(0); }

__device__ __forceinline__ int clamp_len(const int* len, int b, int n) {
  return len ? min(max(len[b], 0), n) : n;
}

// Natural logarithm of 2^ref l, rounded once: the integer part of log2 l is added in 64 bits.
__device__ __forceinline__ float diff_lse(float l, float ref) {
  const double whole = (double)ref + (double)__builtin_amdgcn_frexp_expf(l);
  return (float)((whole + (double)log2f(__builtin_amdgcn_frexp_mantf(l))) * 0.69314718055994531);
}

// Byte offset, from the first row of a tile, of logical chunk c of row r, or
// kOutOfSlab for a chunk past the row's end.
__device__ __forceinline__ uint32_t row_chunk_offset(int r, int c, int creal, uint32_t row_bytes) {
  return c < creal ? (uint32_t)r * row_bytes + (uint32_t)c * 16u : kOutOfSlab;
}

// The rows of one head, tile after tile. The resource of a tile begins at its
// first row (a 64-bit address, so a head may span more than 4 GiB) and ends
// with the last row that exists: reads past it return zeros. A step costs a
// few scalar instructions: with the tile's address and extent formed anew
// every time, the kernels spent as many issue cycles on scalar as on vector
// instructions.
struct TileRows {
  const char* p;
  uint32_t row_bytes, full, last;   // bytes per row, of a whole tile up to the end of its last row, of a row's data
  __device__ __forceinline__ TileRows(const uint16_t* first, uint32_t rb, int dreal)
      : p(reinterpret_cast<const char*>(first)), row_bytes(rb), full((kDiffTile - 1) * rb + (uint32_t)dreal * 2u),
        last((uint32_t)dreal * 2u) {}
  __device__ __forceinline__ void skip(int tiles) { p += (long long)tiles * kDiffTile * row_bytes; }
  // the current tile, of which `rows` >= 1 rows exist; moves on to the next
  __device__ __forceinline__ rsrc_t next(int rows) {
    const rsrc_t r = make_rsrc(p, rows >= kDiffTile ? full : (uint32_t)(rows - 1) * row_bytes + last);
    p += (unsigned long long)(kDiffTile * row_bytes);
    return r;
  }
};

// Swizzle of a tile that is read as 16x16x32 operands: bijective in the 16
// rows of a row read, whose service groups of 16 lanes are rows 0-3 and 12-15
// at one chunk with rows 4-11 at the next (chunk c and c ^ 1), and the reverse;
// and distinct in all but the lowest bit for the eight rows that 32 lanes of a
// transpose read touch at one pair of chunks. With rows of 8 chunks two rows
// share the 16 slots. (Bank conflicts counted: none; 29% of the LDS cycles
// with a swizzle that ignores the service groups.)
template <int CPR>
__host__ __device__ constexpr int swz16(int r) {
  const int low = 2 * (((r >> 2) ^ (r >> 3)) & 1) + ((r >> 3) & 1);
  return CPR % 16 == 0 ? 4 * (r & 3) + low : 4 * ((r >> 1) & 1) + low;
}

// Staging of a tile of three matrices A, B (DA columns each) and C (DC
// columns), 32 rows each, by direct-to-LDS loads of NT threads: stage layout
// [A | B | C], every matrix in the swizzled layout of kl_common.hpp, or in
// that of swz16 (K16).
template <int DA, int DC, int NT, bool K16 = false>
struct DiffDma {
  static constexpr int CA = lds_cols(DA) / 8, CC = lds_cols(DC) / 8;
  static constexpr int CHUNKS = kDiffTile * (2 * CA + CC);
  static constexpr int NCH = CHUNKS / NT;
  // every load instruction of a wave (64 chunks) serves one matrix; which one is known at compile time unless the
  // instruction of the whole workgroup straddles two
  static constexpr bool WHOLE = (kDiffTile * CA) % NT == 0;
  static_assert(CHUNKS % NT == 0, "staging split");
  uint32_t voff[NCH];

  // which matrix chunk p of the stage belongs to
  __device__ __forceinline__ static constexpr int matrix(int p) {
    return p < kDiffTile * CA ? 0 : p < 2 * kDiffTile * CA ? 1 : 2;
  }

  __device__ __forceinline__ DiffDma(int tid, uint32_t ba, uint32_t bb, uint32_t bc) {
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int p = tid + NT * i, m = matrix(p);
      if (m < 2) {
        const int pp = p - m * kDiffTile * CA;
        const int r = pp / CA, c = (pp - r * CA) ^ (K16 ? swz16<CA>(r) : swz<CA>(r));
        voff[i] = row_chunk_offset(r, c, DA / 8, m == 0 ? ba : bb);
      } else {
        const int pp = p - 2 * kDiffTile * CA;
        const int r = pp / CC, c = (pp - r * CC) ^ (K16 ? swz16<CC>(r) : swz<CC>(r));
        voff[i] = row_chunk_offset(r, c, DC / 8, bc);
      }
    }
  }

  __device__ __forceinline__ void issue(rsrc_t ra, rsrc_t rb, rsrc_t rc, u32x4* stage, int wave) const {
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int m = matrix(NT * i + (WHOLE ? 0 : 64 * wave));
      const rsrc_t r = m == 0 ? ra : m == 1 ? rb : rc;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)(stage + NT * i + 64 * wave), 16, voff[i], 0, 0, 0);
    }
#endif
  }
};

// Streams tiles t0 .. t1 - 1 through STAGES (2 or 3) LDS stages of TR (1 or 2)
// tiles, CHUNKS chunks apart: while the tiles of one are worked on, the loads
// of the next one or two are in flight, and the workgroup meets once a stage.
// load(t, place) starts the loads of a tile, NLOAD instructions of this wave;
// tile(t, place) works on it. The stages are separate arrays, named
// explicitly, so that the compiler can tell reads of one from loads into
// another. With two, s2 is unused.
template <int STAGES, int TR, int CHUNKS, int NLOAD, typename Load, typename Tile>
__device__ __forceinline__ void stream_tiles(u32x4* s0, u32x4* s1, u32x4* s2, int t0, int t1, Load load, Tile tile) {
  static_assert((STAGES == 2 || STAGES == 3) && (TR == 1 || TR == 2), "two or three stages of one or two tiles");
  auto fill = [&](u32x4* s, int t) {
#pragma unroll
    for (int i = 0; i < TR; ++i)
      if (t + i < t1) load(t + i, s + i * CHUNKS);
  };
  // all loads but those of the stage that begins with tile t have landed
  auto wait_but = [&](int t) {
    if (STAGES == 3 && t + TR <= t1) wait_vmem_le<TR * NLOAD>();
    else if (STAGES == 3 && TR == 2 && t < t1) wait_vmem_le<NLOAD>();
    else wait_vmem();
  };
  fill(s0, t0);
  if (STAGES == 3) fill(s1, t0 + TR);
  wait_but(t0 + TR);
  barrier_no_fence();
  auto step = [&](u32x4* cur, u32x4* ahead, int t) {
    fill(ahead, t + (STAGES - 1) * TR);
#pragma unroll
    for (int i = 0; i < TR; ++i)
      if (i == 0 || t + i < t1) tile(t + i, cur + i * CHUNKS);
    wait_but(t + (STAGES - 1) * TR);
    wait_lds();
    barrier_no_fence();
  };
  for (int t = t0; t < t1; t += STAGES * TR) {
    step(s0, STAGES == 3 ? s2 : s1, t);
    if (t + TR < t1) step(s1, s0, t + TR);
    if constexpr (STAGES == 3) {
      if (t + 2 * TR < t1) step(s2, s1, t + 2 * TR);
    }
  }
}

// Byte offsets within a matrix of D columns of the transpose reads that
// deliver, for 16-row block s, the 32 columns 32 nb + l % 32 of rows
// 4 half + 0..3 (h = 0) and 8 + 4 half + 0..3 (h = 1): offset(nb, h) + 256 CPR s.
// Computed once and hidden from the optimizer (see TrOffsets in kl_bwd.hpp).
template <int D>
struct TrCols {
  static constexpr int CPR = lds_cols(D) / 8, NB = D / 32;
  int o[NB][2];
  __device__ __forceinline__ explicit TrCols(int lane) {
    const int half = lane >> 5;
    const int row = 4 * half + ((lane & 15) >> 2);
    const int col = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const int e = 32 * nb + col;
        o[nb][h] = opaque(chunk_slot<CPR>(row + 8 * h, e >> 3) * 16 + ((e >> 2) & 1) * 8);
      }
  }
  // base: byte offset of the matrix in buf
  __device__ __forceinline__ bf16x8 read(const void* buf, int base, int nb, int s) const {
    return cat8(lds_tr4_at(buf, o[nb][0] + base + 256 * CPR * s), lds_tr4_at(buf, o[nb][1] + base + 256 * CPR * s));
  }
};

// 16-byte chunks 2 ks + half of a row as MFMA operands; zeros where the row
// does not exist.
template <int D>
__device__ __forceinline__ void load_row_operand(bf16x8 (&op)[D / 16], const uint16_t* row, bool ok, int half) {
  const u32x4* p = reinterpret_cast<const u32x4*>(row);
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks)
    op[ks] = __builtin_bit_cast(bf16x8, ok ? p[2 * ks + half] : u32x4{0u, 0u, 0u, 0u});
}

}  // namespace streamkl
