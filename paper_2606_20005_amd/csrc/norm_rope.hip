// Norms of queries and keys per head with the position rotation in the same
// pass (streamkl_qk_norm_rope_fwd, streamkl_qk_norm_rope_bwd): kernels,
// argument checks and launches.
//
// With x one head of one token (d values), w the learned weight and (c, s)
// the cosine and sine of the token's position for a rotated pair (a, b),
//   r = 1 / sqrt(mean_j x_j^2 + eps),   n_j = x_j r w_j,
//   y_a = n_a c - n_b s,                y_b = n_b c + n_a s,
// and y_j = n_j for the columns that are not rotated. Backward:
//   g_a = dy_a c + dy_b s,              g_b = dy_b c - dy_a s,
//   dw_j = sum_rows g_j x_j r,          h_j = g_j w_j,
//   dx_j = r (h_j - x_j r^2 mean_i(h_i x_i)).
// All of it is float32; y and dx are rounded once, when they are written.
//
// Bound: HBM. A value is read once and written once (twice read in the
// backward), with about 10 (35) operations between. The layout follows from
// that: a lane holds one 16-byte chunk of a bf16 row (8 values), TPR lanes a
// row, and a wave 64 / TPR consecutive tokens of one head, so that the
// head-major side (y, dy) moves in runs of 64 / TPR rows and the token-major
// side (x, dx) in whole rows. A wave keeps its tokens and walks over heads:
// the products of weights with cosines and sines are formed once per token
// and serve all of them. The partner of a rotated value lies rot/2 columns
// away, in a chunk of another lane of the row; it comes by one cross-lane
// read per dword.
#include <cmath>
#include <cstdint>

#include "kl_common.hpp"
#include "streamkl.h"

namespace streamkl {
namespace {

typedef unsigned int u32;
typedef u32 u32x2 __attribute__((ext_vector_type(2)));

constexpr int kRotNone = 0, kRotHalf = 1, kRotPairs = 2;
constexpr int kWaves = kThreads / 64;

// One of the two tensors of a call (queries or keys).
struct NrSide {
  const void* x;               // [B, N, H, d], element strides below
  long long sb, sn, sh;
  const float* w;              // [d] or null (ones)
  const void* pos;             // [N] or [B, N] (pos_sb = N) positions, or null: start + n
  long long pos_sb;
  int start;
  void* y;                     // forward: [B, H copies, N, d] bf16
  const void* dy;              // backward: the same layout, bf16 or float32
  void* dx;                    // backward: [B, N, H, d] contiguous, the type of x
  float* part;                 // backward: [blocks][d] partial sums of dw, or null
  int N, H, copies;
  int tokens;                  // B N
  int heads_per_item, chunks;  // an item is 64 / TPR tokens x heads_per_item heads; chunks per token group
  int items, blocks;
};

struct NrArgs {
  NrSide q, k;
  const float* table;          // [n_pos][rot]: cosines of the rot/2 pairs, then their sines
  int n_pos, rot, d, pos64;
  float eps;
};

template <typename T>
struct Raw;                    // 8 values as they lie in memory
template <>
struct Raw<__bf16> { u32x4 v[1]; };
template <>
struct Raw<_Float16> { u32x4 v[1]; };
template <>
struct Raw<float> { u32x4 v[2]; };

template <typename T>
__device__ __forceinline__ Raw<T> load8(const T* p) {
  Raw<T> r;
#pragma unroll
  for (int i = 0; i < (int)(sizeof(r.v) / 16); ++i) r.v[i] = reinterpret_cast<const u32x4*>(p)[i];
  return r;
}

template <typename T>
__device__ __forceinline__ void unpack8(const Raw<T>& r, float (&f)[8]) {
  typedef T T8 __attribute__((ext_vector_type(8)));
  const T8 t = __builtin_bit_cast(T8, r.v);
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = (float)t[e];
}

template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&f)[8]) {
  typedef T T8 __attribute__((ext_vector_type(8)));
  T8 t;
#pragma unroll
  for (int e = 0; e < 8; ++e) t[e] = (T)f[e];
  Raw<T> r;
  __builtin_memcpy(&r, &t, sizeof(r));
#pragma unroll
  for (int i = 0; i < (int)(sizeof(r.v) / 16); ++i) reinterpret_cast<u32x4*>(p)[i] = r.v[i];
}

// The raw chunk of lane `src` of this row.
template <typename T>
__device__ __forceinline__ Raw<T> from_lane(const Raw<T>& r, int src) {
  Raw<T> o;
#pragma unroll
  for (int i = 0; i < (int)(sizeof(r.v) / 16); ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) o.v[i][j] = (u32)__builtin_amdgcn_ds_bpermute(4 * src, (int)r.v[i][j]);
  return o;
}

template <int TPR>
__device__ __forceinline__ float row_sum(float v) {
#pragma unroll
  for (int m = 1; m < TPR; m <<= 1) v += __shfl_xor(v, m);
  return v;
}

// What a lane knows of its token and chunk, the same for every head.
template <int TPR, int ROT>
struct Place {
  int c, b, n, src;            // chunk, sequence, token, lane of the partner chunk
  bool live;                   // the token exists and the chunk lies inside the row
  bool known;                  // its position is in the table, or nothing is rotated
  float co[8], si[8];          // of the own columns; si is 0 and co 1 where nothing is rotated

  __device__ __forceinline__ Place(const NrArgs& a, const NrSide& s, int group, int lane) {
    constexpr int RPW = 64 / TPR;
    c = lane & (TPR - 1);
    const int t = group * RPW + lane / TPR;
    const bool token = t < s.tokens;
    b = token ? t / s.N : 0;
    n = token ? t - b * s.N : 0;
    live = token && 8 * c < a.d;
    src = lane;
    known = true;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      co[e] = 1.f;
      si[e] = 0.f;
    }
    if constexpr (ROT != kRotNone) {
      const bool turned = 8 * c < a.rot;
      const int half = a.rot >> 1;   // a multiple of 8
      if (ROT == kRotHalf && turned) src = 8 * c < half ? lane + half / 8 : lane - half / 8;
      long long p = s.start + n;
      if (token && s.pos) {
        const long long i = (long long)b * s.pos_sb + n;
        p = a.pos64 ? static_cast<const long long*>(s.pos)[i] : static_cast<const int*>(s.pos)[i];
      }
      // a position outside the table: NaN in the rotated columns, nothing is read
      known = p >= 0 && p < a.n_pos;
      if (live && turned) {
        const float* row = a.table + (known ? p : 0) * a.rot;
        if constexpr (ROT == kRotHalf) {
          const bool low = 8 * c < half;
          const float* q = row + (low ? 8 * c : 8 * c - half);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const f32x4 cc = reinterpret_cast<const f32x4*>(q)[i], ss = reinterpret_cast<const f32x4*>(q + half)[i];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              co[4 * i + j] = known ? cc[j] : __builtin_nanf("");
              si[4 * i + j] = low ? -ss[j] : ss[j];
            }
          }
        } else {
          const f32x4 cc = *reinterpret_cast<const f32x4*>(row + 4 * c);
          const f32x4 ss = *reinterpret_cast<const f32x4*>(row + half + 4 * c);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            co[2 * j] = co[2 * j + 1] = known ? cc[j] : __builtin_nanf("");
            si[2 * j] = -ss[j];
            si[2 * j + 1] = ss[j];
          }
        }
      }
    }
  }
};

__device__ __forceinline__ void load_weight(const float* w, int c, bool live, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const f32x4 v = w && live ? reinterpret_cast<const f32x4*>(w + 8 * c)[i] : f32x4{1.f, 1.f, 1.f, 1.f};
#pragma unroll
    for (int j = 0; j < 4; ++j) f[4 * i + j] = v[j];
  }
}

// The values that those of this lane are rotated with, from their raw chunk.
template <typename T, int ROT>
__device__ __forceinline__ void partner8(const Raw<T>& raw, const float (&x)[8], int src, float (&xp)[8]) {
  if constexpr (ROT == kRotHalf) {
    unpack8<T>(from_lane<T>(raw, src), xp);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) xp[e] = x[e ^ 1];
  }
}

template <typename T, int TPR, int ROT>
__global__ void __launch_bounds__(kThreads) norm_rope_fwd_kernel(const NrArgs a) {
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int block = (int)(blockIdx.y * gridDim.x + blockIdx.x);
  const bool keys = block >= a.q.blocks;
  const NrSide& s = keys ? a.k : a.q;
  const int item = (block - (keys ? a.q.blocks : 0)) * kWaves + wave;
  if (item >= s.items) return;
  const int group = item / s.chunks, h0 = (item - group * s.chunks) * s.heads_per_item;
  const int h1 = min(h0 + s.heads_per_item, s.H);
  const Place<TPR, ROT> at(a, s, group, lane);
  float own[8], other[8];   // factors of the own and of the partner's values, r apart
  {
    float w[8], wp[8];
    load_weight(s.w, at.c, at.live, w);
    if constexpr (ROT == kRotHalf) {
      load_weight(s.w, at.src & (TPR - 1), at.live, wp);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) wp[e] = w[e ^ 1];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      own[e] = w[e] * at.co[e];
      other[e] = wp[e] * at.si[e];
    }
  }
  const float rd = 1.f / (float)a.d;
  const T* px = static_cast<const T*>(s.x) + (long long)at.b * s.sb + (long long)at.n * s.sn + 8 * at.c;
  __bf16* py = static_cast<__bf16*>(s.y) + 8 * at.c;
  const long long hstride = (long long)s.N * a.d;
  py += (long long)at.b * s.H * s.copies * hstride + (long long)at.n * a.d;
  Raw<T> next = {};
  if (at.live && h0 < h1) next = load8<T>(px + h0 * s.sh);
  for (int h = h0; h < h1; ++h) {
    const Raw<T> raw = next;
    if (at.live && h + 1 < h1) next = load8<T>(px + (h + 1) * s.sh);
    float x[8], ss = 0.f;
    unpack8<T>(raw, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = __builtin_fmaf(x[e], x[e], ss);
    ss = row_sum<TPR>(ss);
    const float r = 1.f / sqrtf(__builtin_fmaf(ss, rd, a.eps));
    float y[8];
    if constexpr (ROT != kRotNone) {
      float xp[8];
      partner8<T, ROT>(raw, x, at.src, xp);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = r * __builtin_fmaf(xp[e], other[e], x[e] * own[e]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = r * (x[e] * own[e]);
    }
    if (at.live) {
      for (int g = 0; g < s.copies; ++g) store8<__bf16>(py + ((long long)h * s.copies + g) * hstride, y);
    }
  }
}

// The gradients. Blocks walk over items with a fixed stride and add up dw in
// registers; each leaves one partial row of dw, summed in a fixed order by
// norm_rope_dw_kernel: the results are reproducible bit for bit.
template <typename T, typename TG, int TPR, int ROT>
__global__ void __launch_bounds__(kThreads) norm_rope_bwd_kernel(const NrArgs a) {
  __shared__ float red[kWaves][TPR * 8];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool keys = (int)blockIdx.x >= a.q.blocks;
  const NrSide& s = keys ? a.k : a.q;
  const int blk = (int)blockIdx.x - (keys ? a.q.blocks : 0);
  const float rd = 1.f / (float)a.d;
  const long long hstride = (long long)s.N * a.d;
  const int c = lane & (TPR - 1);
  float w[8], dw[8];
  load_weight(s.w, c, 8 * c < a.d, w);
#pragma unroll
  for (int e = 0; e < 8; ++e) dw[e] = 0.f;
  for (int item = blk * kWaves + wave; item < s.items; item += s.blocks * kWaves) {
    const int group = item / s.chunks, h0 = (item - group * s.chunks) * s.heads_per_item;
    const int h1 = min(h0 + s.heads_per_item, s.H);
    const Place<TPR, ROT> at(a, s, group, lane);
    const bool strange = ROT != kRotNone && __builtin_amdgcn_ballot_w64(!at.known) != 0;
    const T* px = static_cast<const T*>(s.x) + (long long)at.b * s.sb + (long long)at.n * s.sn + 8 * at.c;
    const TG* pg = static_cast<const TG*>(s.dy) + 8 * at.c;
    pg += (long long)at.b * s.H * s.copies * hstride + (long long)at.n * a.d;
    T* pd = static_cast<T*>(s.dx) + ((long long)at.b * s.N + at.n) * s.H * a.d + 8 * at.c;
    Raw<T> xnext = {};
    Raw<TG> gnext = {};
    if (at.live && h0 < h1) {
      xnext = load8<T>(px + h0 * s.sh);
      gnext = load8<TG>(pg + (long long)h0 * s.copies * hstride);
    }
    for (int h = h0; h < h1; ++h) {
      const Raw<T> xraw = xnext;
      Raw<TG> graw = gnext;
      if (at.live && h + 1 < h1) {
        xnext = load8<T>(px + (h + 1) * s.sh);
        gnext = load8<TG>(pg + (long long)(h + 1) * s.copies * hstride);
      }
      float x[8], g[8], gp[8];
      unpack8<T>(xraw, x);
      unpack8<TG>(graw, g);
      if (s.copies > 1) {   // a shared head's gradient is the sum over its copies
        for (int j = 1; j < s.copies; ++j) {
          float more[8];
          Raw<TG> m = {};
          if (at.live) m = load8<TG>(pg + ((long long)h * s.copies + j) * hstride);
          unpack8<TG>(m, more);
#pragma unroll
          for (int e = 0; e < 8; ++e) g[e] += more[e];
        }
        if constexpr (ROT == kRotHalf) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            gp[e] = __int_as_float(__builtin_amdgcn_ds_bpermute(4 * at.src, __float_as_int(g[e])));
        }
      } else if constexpr (ROT == kRotHalf) {
        unpack8<TG>(from_lane<TG>(graw, at.src), gp);
      }
      if constexpr (ROT != kRotNone) {
        if constexpr (ROT == kRotPairs) {
#pragma unroll
          for (int e = 0; e < 8; ++e) gp[e] = g[e ^ 1];
        }
        // the transposed rotation: the sine changes its sign
        float turned[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) turned[e] = __builtin_fmaf(-at.si[e], gp[e], at.co[e] * g[e]);
        if (strange) {   // a row outside the table that the loss does not reach (padding): no gradient, not 0 times NaN
#pragma unroll
          for (int e = 0; e < 8; ++e) turned[e] = !at.known && g[e] == 0.f && gp[e] == 0.f ? 0.f : turned[e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) g[e] = turned[e];
      }
      float ss = 0.f, hx = 0.f, hh[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        hh[e] = g[e] * w[e];
        ss = __builtin_fmaf(x[e], x[e], ss);
        hx = __builtin_fmaf(hh[e], x[e], hx);
      }
      ss = row_sum<TPR>(ss);
      hx = row_sum<TPR>(hx);
      const float r = 1.f / sqrtf(__builtin_fmaf(ss, rd, a.eps));
      const float m = r * r * (hx * rd);
      float o[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        dw[e] = __builtin_fmaf(g[e] * x[e], r, dw[e]);
        o[e] = r * __builtin_fmaf(-m, x[e], hh[e]);
      }
      if (at.live) store8<T>(pd + (long long)h * a.d, o);
    }
  }
  if (s.part == nullptr) return;
  // lanes of a wave that hold the same columns, then the waves. Lanes past
  // the row held zeros throughout.
#pragma unroll
  for (int e = 0; e < 8; ++e) {
#pragma unroll
    for (int m = TPR; m < 64; m <<= 1) dw[e] += __shfl_xor(dw[e], m);
  }
  if (lane < TPR) {
#pragma unroll
    for (int e = 0; e < 8; ++e) red[wave][8 * lane + e] = dw[e];
  }
  __syncthreads();
  for (int j = threadIdx.x; j < a.d; j += kThreads) {
    float v = red[0][j];
#pragma unroll
    for (int i = 1; i < kWaves; ++i) v += red[i][j];
    s.part[(long long)blk * a.d + j] = v;
  }
}

constexpr int kDwCols = 16, kDwThreads = 1024, kDwRows = kDwThreads / kDwCols;

__global__ void __launch_bounds__(kDwThreads)
norm_rope_dw_kernel(const float* __restrict__ pq, int nq, float* __restrict__ dwq, const float* __restrict__ pk, int nk,
                    float* __restrict__ dwk, int d) {
  __shared__ float red[kDwRows][kDwCols];
  const bool keys = blockIdx.y == 1;
  const float* p = keys ? pk : pq;
  float* out = keys ? dwk : dwq;
  if (!out) return;
  const int rows = keys ? nk : nq;
  const int col = blockIdx.x * kDwCols + threadIdx.x % kDwCols, r0 = threadIdx.x / kDwCols;
  // eight loads in flight: one after the other, 2048 partial rows took 11 us
  float v = 0.f;
  for (int r = r0; r < rows; r += 8 * kDwRows) {
    float x[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) x[u] = r + u * kDwRows < rows ? p[(long long)(r + u * kDwRows) * d + col] : 0.f;
#pragma unroll
    for (int u = 0; u < 8; ++u) v += x[u];
  }
  red[r0][threadIdx.x % kDwCols] = v;
  __syncthreads();
  if (threadIdx.x < kDwCols) {
    float t = 0.f;
    for (int i = 0; i < kDwRows; ++i) t += red[i][threadIdx.x];
    out[col] = t;
  }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------

int lanes_per_row(int d) { return d <= 32 ? 4 : d <= 64 ? 8 : d <= 128 ? 16 : 32; }

// Heads that a wave walks over with the factors of its tokens: as many as
// leave the chip 16 waves a CU, at most 8.
void plan(NrSide& s, int d, int most_blocks) {
  const int rpw = 64 / lanes_per_row(d);
  const int groups = (int)((s.tokens + rpw - 1LL) / rpw);
  int hpi = 1;
  while (hpi < 8 && hpi < s.H && (long long)groups * ((s.H + 2LL * hpi - 1) / (2 * hpi)) >= 16LL * kCus) hpi *= 2;
  s.heads_per_item = hpi;
  s.chunks = (int)((hpi - 1LL + s.H) / hpi);
  s.items = groups * s.chunks;
  s.blocks = (int)((s.items + kWaves - 1LL) / kWaves);
  if (most_blocks > 0 && s.blocks > most_blocks) s.blocks = most_blocks;
}

// Blocks of the backward per tensor: 8 of 256 threads a CU are what is
// resident, and each leaves one partial row of dw.
constexpr int kBwdBlocks = 8 * kCus;

bool aligned_to(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// Heads of tokens are counted in 31 bits, with room for a stride past the end.
bool countable(int B, int N, int H) {
  constexpr long long most = 0x7fff0000LL;
  const long long tokens = (long long)B * N;
  return tokens <= most && tokens * H <= most;
}

int elem_size(int dtype) { return dtype == STREAMKL_F32 ? 4 : 2; }

// One side: extents, strides, positions, the tensor it writes. `present`: the
// side has rows.
int check_side(const streamkl_rows* x, int B, int N, int H, int copies, int dtype, const float* w, const void* pos,
               int pos64, const void* y, bool* present) {
  *present = x != nullptr && B != 0 && N != 0 && H != 0;
  if (!x) return STREAMKL_OK;
  if (N < 0 || H < 0 || copies < 1) return STREAMKL_ERR_INVALID_ARG;
  if (!countable(B, N, H) || (long long)H * copies > 0x7fff0000LL) return STREAMKL_ERR_UNSUPPORTED;
  if (!*present) return STREAMKL_OK;
  const int per16 = 16 / elem_size(dtype);
  if (!x->data || !aligned_to(x->data, 16)) return STREAMKL_ERR_INVALID_ARG;
  if (x->sb % per16 || x->sh % per16 || x->sn % per16) return STREAMKL_ERR_INVALID_ARG;
  if (x->sb < 0 || x->sh < 0 || x->sn < 0) return STREAMKL_ERR_INVALID_ARG;
  if (w && !aligned_to(w, 16)) return STREAMKL_ERR_INVALID_ARG;
  if (pos && !aligned_to(pos, pos64 ? 8 : 4)) return STREAMKL_ERR_INVALID_ARG;
  if (!y || !aligned_to(y, 16)) return STREAMKL_ERR_INVALID_ARG;
  return STREAMKL_OK;
}

int check_call(int B, int d, int dtype, float eps, const float* table, int n_pos, int rot, int interleaved, int pos64) {
  if (B < 0 || n_pos < 0) return STREAMKL_ERR_INVALID_ARG;
  if (dtype != STREAMKL_BF16 && dtype != STREAMKL_F16 && dtype != STREAMKL_F32) return STREAMKL_ERR_INVALID_ARG;
  if (!(std::isfinite(eps) && eps > 0.f)) return STREAMKL_ERR_INVALID_ARG;
  if ((interleaved != 0 && interleaved != 1) || (pos64 != 0 && pos64 != 1)) return STREAMKL_ERR_INVALID_ARG;
  if (d < 32 || d > 256 || d % 32 != 0) return STREAMKL_ERR_UNSUPPORTED;
  if (rot < 0 || rot > d) return STREAMKL_ERR_INVALID_ARG;
  if (rot % 16 != 0) return STREAMKL_ERR_UNSUPPORTED;
  if (rot > 0 && (n_pos < 1 || !table || !aligned_to(table, 16))) return STREAMKL_ERR_INVALID_ARG;
  return STREAMKL_OK;
}

// The places that rows without positions stand at, all of them in the table:
// keys at 0 .. N_K - 1, queries at the last N_Q of these (without keys, at
// 0 .. N_Q - 1).
int check_places(bool has_q, bool has_k, bool keys_given, bool queries_given, int N_Q, int N_K, const void* q_pos,
                 const void* k_pos, int rot, int n_pos) {
  if (rot == 0) return STREAMKL_OK;
  if (keys_given && queries_given && !q_pos && N_Q > N_K) return STREAMKL_ERR_INVALID_ARG;   // places before the first
  if (has_k && !k_pos && N_K > n_pos) return STREAMKL_ERR_INVALID_ARG;
  if (has_q && !q_pos && (keys_given ? N_K : N_Q) > n_pos) return STREAMKL_ERR_INVALID_ARG;
  return STREAMKL_OK;
}

NrSide make_side(const streamkl_rows* x, bool present, int B, int N, int H, int copies, const float* w, const void* pos,
                 int pos_shared, int start, int d, int most_blocks) {
  NrSide s = {};
  if (!present) return s;
  s.x = x->data;
  s.sb = x->sb;
  s.sn = x->sn;
  s.sh = x->sh;
  s.w = w;
  s.pos = pos;
  s.pos_sb = pos_shared ? 0 : N;
  s.start = start;
  s.N = N;
  s.H = H;
  s.copies = copies;
  s.tokens = B * N;
  plan(s, d, most_blocks);
  return s;
}

template <typename T, int TPR, int ROT>
void run_fwd(const NrArgs& a, hipStream_t st) {
  // an axis of the grid holds less than 2^32 threads
  const unsigned blocks = (unsigned)(a.q.blocks + a.k.blocks), x = blocks < 1u << 22 ? blocks : 1u << 22;
  norm_rope_fwd_kernel<T, TPR, ROT><<<dim3(x, (blocks + x - 1) / x), dim3(kThreads), 0, st>>>(a);
}

template <typename T, typename TG, int TPR, int ROT>
void run_bwd(const NrArgs& a, hipStream_t st) {
  norm_rope_bwd_kernel<T, TG, TPR, ROT><<<dim3((unsigned)(a.q.blocks + a.k.blocks)), dim3(kThreads), 0, st>>>(a);
}

// f(lanes per row, rotation) for compile-time values of both
template <typename F>
void by_shape(int d, int rot, int interleaved, F f) {
  auto by_rot = [&](auto tpr) {
    if (rot == 0)
      f(tpr, std::integral_constant<int, kRotNone>{});
    else if (interleaved)
      f(tpr, std::integral_constant<int, kRotPairs>{});
    else
      f(tpr, std::integral_constant<int, kRotHalf>{});
  };
  switch (lanes_per_row(d)) {
    case 4: return by_rot(std::integral_constant<int, 4>{});
    case 8: return by_rot(std::integral_constant<int, 8>{});
    case 16: return by_rot(std::integral_constant<int, 16>{});
    default: return by_rot(std::integral_constant<int, 32>{});
  }
}

template <typename T>
void by_shape_fwd(const NrArgs& a, int interleaved, hipStream_t st) {
  by_shape(a.d, a.rot, interleaved, [&](auto tpr, auto rot) { run_fwd<T, tpr.value, rot.value>(a, st); });
}

template <typename T, typename TG>
void by_shape_bwd(const NrArgs& a, int interleaved, hipStream_t st) {
  by_shape(a.d, a.rot, interleaved, [&](auto tpr, auto rot) { run_bwd<T, TG, tpr.value, rot.value>(a, st); });
}

}  // namespace
}  // namespace streamkl

using namespace streamkl;

extern "C" int streamkl_qk_norm_rope_fwd(const streamkl_rows* q, const streamkl_rows* k, int B, int H, int HK, int N_Q,
                                         int N_K, int d, int dtype, const float* wq, const float* wk, float eps,
                                         const float* table, int n_pos, int rot, int interleaved, const void* q_pos,
                                         const void* k_pos, int pos64, int q_pos_shared, int k_pos_shared, int k_copies,
                                         void* yq, void* yk, hipStream_t stream) {
  int st = check_call(B, d, dtype, eps, table, n_pos, rot, interleaved, pos64);
  bool has_q = false, has_k = false;
  if (st == STREAMKL_OK) st = check_side(q, B, N_Q, H, 1, dtype, wq, q_pos, pos64, yq, &has_q);
  if (st == STREAMKL_OK) st = check_side(k, B, N_K, HK, k_copies, dtype, wk, k_pos, pos64, yk, &has_k);
  if (st == STREAMKL_OK) st = check_places(has_q, has_k, k, q, N_Q, N_K, q_pos, k_pos, rot, n_pos);
  if (st != STREAMKL_OK) return st;
  if (!has_q && !has_k) return STREAMKL_OK;
  NrArgs a = {};
  // without positions the queries are the last N_Q of the N_K places
  a.q = make_side(q, has_q, B, N_Q, H, 1, wq, q_pos, q_pos_shared, k ? N_K - N_Q : 0, d, 0);
  a.k = make_side(k, has_k, B, N_K, HK, k_copies, wk, k_pos, k_pos_shared, 0, d, 0);
  a.q.y = yq;
  a.k.y = yk;
  a.table = table;
  a.n_pos = n_pos;
  a.rot = rot;
  a.d = d;
  a.pos64 = pos64;
  a.eps = eps;
  if (dtype == STREAMKL_F32)
    by_shape_fwd<float>(a, interleaved, stream);
  else if (dtype == STREAMKL_F16)
    by_shape_fwd<_Float16>(a, interleaved, stream);
  else
    by_shape_fwd<__bf16>(a, interleaved, stream);
  return hipGetLastError() == hipSuccess ? STREAMKL_OK : STREAMKL_ERR_HIP;
}

extern "C" size_t streamkl_qk_norm_rope_bwd_workspace_bytes(int B, int H, int HK, int N_Q, int N_K, int d) {
  if (B < 0 || H < 0 || HK < 0 || N_Q < 0 || N_K < 0 || d < 32 || d > 256 || d % 32 != 0) return 0;
  if (!countable(B, N_Q, H) || !countable(B, N_K, HK)) return 0;
  NrSide q = {}, k = {};
  q.tokens = B * N_Q;
  q.H = H;
  k.tokens = B * N_K;
  k.H = HK;
  if (q.H) plan(q, d, kBwdBlocks);
  if (k.H) plan(k, d, kBwdBlocks);
  return (size_t)(q.blocks + k.blocks) * (size_t)d * sizeof(float);
}

extern "C" int streamkl_qk_norm_rope_bwd(const streamkl_rows* q, const streamkl_rows* k, int B, int H, int HK, int N_Q,
                                         int N_K, int d, int dtype, const float* wq, const float* wk, float eps,
                                         const float* table, int n_pos, int rot, int interleaved, const void* q_pos,
                                         const void* k_pos, int pos64, int q_pos_shared, int k_pos_shared, int k_copies,
                                         const void* dyq, const void* dyk, int dy_dtype, void* workspace,
                                         size_t workspace_bytes, void* dxq, void* dxk, float* dwq, float* dwk,
                                         hipStream_t stream) {
  int st = check_call(B, d, dtype, eps, table, n_pos, rot, interleaved, pos64);
  bool has_q = false, has_k = false;
  if (st == STREAMKL_OK && dy_dtype != STREAMKL_BF16 && dy_dtype != STREAMKL_F32) st = STREAMKL_ERR_INVALID_ARG;
  if (st == STREAMKL_OK) st = check_side(q, B, N_Q, H, 1, dtype, wq, q_pos, pos64, dxq, &has_q);
  if (st == STREAMKL_OK) st = check_side(k, B, N_K, HK, k_copies, dtype, wk, k_pos, pos64, dxk, &has_k);
  if (st == STREAMKL_OK) st = check_places(has_q, has_k, k, q, N_Q, N_K, q_pos, k_pos, rot, n_pos);
  if (st != STREAMKL_OK) return st;
  if ((has_q && (!dyq || !aligned_to(dyq, 16))) || (has_k && (!dyk || !aligned_to(dyk, 16))))
    return STREAMKL_ERR_INVALID_ARG;
  if ((dwq && !aligned_to(dwq, 4)) || (dwk && !aligned_to(dwk, 4))) return STREAMKL_ERR_INVALID_ARG;
  if ((dwq && !q) || (dwk && !k)) return STREAMKL_ERR_INVALID_ARG;
  if (!has_q && !has_k && !dwq && !dwk) return STREAMKL_OK;
  NrArgs a = {};
  a.q = make_side(q, has_q, B, N_Q, H, 1, wq, q_pos, q_pos_shared, k ? N_K - N_Q : 0, d, kBwdBlocks);
  a.k = make_side(k, has_k, B, N_K, HK, k_copies, wk, k_pos, k_pos_shared, 0, d, kBwdBlocks);
  const size_t need = (size_t)((dwq ? a.q.blocks : 0) + (dwk ? a.k.blocks : 0)) * d * sizeof(float);
  if (need && (!workspace || !aligned_to(workspace, 4) || workspace_bytes < need)) return STREAMKL_ERR_INVALID_ARG;
  float* part = static_cast<float*>(workspace);
  a.q.dy = dyq;
  a.q.dx = dxq;
  a.q.part = dwq ? part : nullptr;
  a.k.dy = dyk;
  a.k.dx = dxk;
  a.k.part = dwk ? part + (dwq ? (size_t)a.q.blocks * d : 0) : nullptr;
  a.table = table;
  a.n_pos = n_pos;
  a.rot = rot;
  a.d = d;
  a.pos64 = pos64;
  a.eps = eps;
  const bool g32 = dy_dtype == STREAMKL_F32;
  if (has_q || has_k) {
    if (dtype == STREAMKL_F32)
      g32 ? by_shape_bwd<float, float>(a, interleaved, stream) : by_shape_bwd<float, __bf16>(a, interleaved, stream);
    else if (dtype == STREAMKL_F16)
      g32 ? by_shape_bwd<_Float16, float>(a, interleaved, stream)
          : by_shape_bwd<_Float16, __bf16>(a, interleaved, stream);
    else
      g32 ? by_shape_bwd<__bf16, float>(a, interleaved, stream) : by_shape_bwd<__bf16, __bf16>(a, interleaved, stream);
    if (hipGetLastError() != hipSuccess) return STREAMKL_ERR_HIP;
  }
  if (dwq || dwk) {   // with no rows the sums are empty: zeros
    norm_rope_dw_kernel<<<dim3((unsigned)(d / kDwCols), 2), dim3(kDwThreads), 0, stream>>>(
        a.q.part, a.q.blocks, dwq, a.k.part, a.k.blocks, dwk, d);
    if (hipGetLastError() != hipSuccess) return STREAMKL_ERR_HIP;
  }
  return STREAMKL_OK;
}
