// Rows of logits as the kernels of logit_logprobs.hip and logit_distill.hip
// read them: 16-byte chunks, the running sums of a softmax, and how a
// workgroup joins them.
//
// A row is V logits x at any element address (rows of an odd vocabulary begin
// anywhere). It is read in aligned 16-byte chunks of EPC elements: chunk 0 is
// the one that holds the first element, `ph` places into it. Chunks that lie
// wholly in the row are loaded as they are, the two that may not be element by
// element, so that nothing outside the row is read; places outside it hold
// -inf, which adds nothing to any sum.
//
// Sums. With c = s log2(e) in float32, every lane keeps a reference r, one of
// its logits, and
//     l = sum 2^((x - r) c),      a = sum 2^((x - r) c) (x - r) c.
// The sums are exact for any reference, so it is moved only when an exponent
// passes kRise, which after the first turns is rare; a small one, since the
// error of an exponent grows with it. The difference comes first: it is exact, or nearly so, for
// the logits that matter, and does not overflow for a row of the type's lowest
// values (which is uniform). A logit of -inf has the power 0; for a its
// exponent is taken as kFloor, where the power is 0 as well.
#pragma once

#include <cmath>
#include <cstdint>
#include <type_traits>

#include "kl_common.hpp"
#include "logit_launch.hpp"
#include "streamkl.h"

namespace streamkl {

typedef unsigned int u32;
typedef unsigned long long u64;

constexpr float kRise = 4.f;
constexpr float kFloor = -1000.f;
constexpr float kNoRef = -3.402823466e38f;   // reference of a lane that has seen nothing but -inf, or only this value

// v_max_f32, v_max3_f32 without the instructions that quiet signalling NaN (a NaN loses against a number). The compiler does
// not see vector instructions in these: what it inserts waits for between two of its own must not follow one or precede it.
// So their operands come from no transcendental instruction, and their results go into no cross-lane operand of another.
__device__ __forceinline__ float vmax(float a, float b) {
  float r;
  asm("v_max_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}
__device__ __forceinline__ float vmax3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

// max of a lane's value and that of lane l ^ 1, l ^ 2. A cross-lane operand may be read two wait states after a vector
// instruction has written it; s_nop 1 is these two.
__device__ __forceinline__ float vmax_xor1(float v) {
  float r;
  asm("s_nop 1\n\tv_max_f32_dpp %0, %1, %1 quad_perm:[1,0,3,2] row_mask:0xf bank_mask:0xf" : "=v"(r) : "v"(v));
  return r;
}
__device__ __forceinline__ float vmax_xor2(float v) {
  float r;
  asm("s_nop 1\n\tv_max_f32_dpp %0, %1, %1 quad_perm:[2,3,0,1] row_mask:0xf bank_mask:0xf" : "=v"(r) : "v"(v));
  return r;
}

// Elements of a type and of the chunks it comes in.
template <typename T>
struct Elem;
template <>
struct Elem<__bf16> {
  static constexpr u32 kNegInfBits = 0xFF80;
};
template <>
struct Elem<_Float16> {
  static constexpr u32 kNegInfBits = 0xFC00;
};
template <>
struct Elem<float> {
  static constexpr u32 kNegInfBits = 0xFF800000;
};
template <typename T>
constexpr int kEpc = 16 / (int)sizeof(T);         // elements of a chunk

template <typename T>
__device__ __forceinline__ void unpack(const u32x4& raw, float (&f)[kEpc<T>]) {
  typedef T TN __attribute__((ext_vector_type(kEpc<T>)));
  const TN t = __builtin_bit_cast(TN, raw);
#pragma unroll
  for (int e = 0; e < kEpc<T>; ++e) f[e] = (float)t[e];
}

template <typename T>
__device__ __forceinline__ u32x4 pack(const float (&f)[kEpc<T>]) {
  typedef T TN __attribute__((ext_vector_type(kEpc<T>)));
  TN t;
#pragma unroll
  for (int e = 0; e < kEpc<T>; ++e) t[e] = (T)f[e];
  return __builtin_bit_cast(u32x4, t);
}

template <int N>
__device__ __forceinline__ float max_all(const float (&m)[N]) {
  float t = m[0];
#pragma unroll
  for (int i = 1; i + 1 < N; i += 2) t = vmax3(t, m[i], m[i + 1]);
  return N % 2 ? t : vmax(t, m[N - 1]);
}

template <typename T>
__device__ __forceinline__ float max_of(const float (&f)[kEpc<T>]) {
  if constexpr (kEpc<T> == 8)
    return vmax3(vmax3(f[0], f[1], f[2]), vmax3(f[3], f[4], f[5]), vmax(f[6], f[7]));
  else
    return vmax(vmax3(f[0], f[1], f[2]), f[3]);
}

// One row.
template <typename T>
struct Row {
  const T* row;          // its first element
  const u32x4* chunk;    // the chunk that holds it
  int V, ph, chunks;     // elements, places of chunk 0 before the first one, chunks that hold elements

  __device__ __forceinline__ Row(const LogitRows& a, int r) {
    const int b = r / a.N;
    row = static_cast<const T*>(a.x) + b * a.sb + (r - b * a.N) * a.sn;
    ph = (int)(reinterpret_cast<uintptr_t>(row) & 15) / (int)sizeof(T);
    chunk = reinterpret_cast<const u32x4*>(row - ph);   // no cast from a number: its loads would be flat ones
    V = a.V;
    chunks = (ph + V + kEpc<T> - 1) / kEpc<T>;
  }
  __device__ __forceinline__ bool whole(int c) const { return c * kEpc<T> >= ph && (c + 1) * kEpc<T> <= ph + V; }
  // chunks c .. c + n - 1 lie wholly in the row
  __device__ __forceinline__ bool whole(int c, int n) const {
    return c * kEpc<T> >= ph && (long long)(c + n) * kEpc<T> <= ph + V;
  }
  // any chunk, -inf in the places outside the row and from chunk `end` on
  __device__ __forceinline__ u32x4 load(int c, int end) const {
    if (c < end && whole(c)) return chunk[c];
    typedef T TN __attribute__((ext_vector_type(kEpc<T>)));
    u32x4 raw;
    const u32 fill = sizeof(T) == 4 ? Elem<T>::kNegInfBits : Elem<T>::kNegInfBits * 0x10001u;
#pragma unroll
    for (int i = 0; i < 4; ++i) raw[i] = fill;
    if (c >= end) return raw;
    TN t = __builtin_bit_cast(TN, raw);
#pragma unroll
    for (int e = 0; e < kEpc<T>; ++e) {
      const int j = c * kEpc<T> + e - ph;
      if (j >= 0 && j < V) t[e] = row[j];
    }
    return __builtin_bit_cast(u32x4, t);
  }
};

template <int N_>
struct Turn {
  static constexpr int N = N_;
  u32x4 raw[N];
};

// Chunks c0 .. c1 - 1 in turns of UNROLL per thread: f(chunk of this thread, Turn), the chunks of a turn THREADS apart, their
// loads in flight together. With ONES a last turn that is at most half full goes one chunk after the other (of 100003 logits
// by 512 threads it is the seventh, a tenth full, and the sums are bound by vector instructions: 148 -> 143 us for 4094
// rows). All threads of a wave call f.
template <typename T, int THREADS, int UNROLL, bool ONES, typename F>
__device__ __forceinline__ void each_turn(const Row<T>& row, int c0, int c1, F f) {
  const int tid = threadIdx.x;
  for (int b = c0; b < c1; b += THREADS * UNROLL) {
    Turn<UNROLL> t;
    if (b + THREADS * UNROLL <= c1 && row.whole(b, THREADS * UNROLL)) {
#pragma unroll
      for (int j = 0; j < UNROLL; ++j) t.raw[j] = row.chunk[b + j * THREADS + tid];
      f(b + tid, t);
    } else {
#pragma unroll
      for (int j = 0; j < UNROLL; ++j) t.raw[j] = row.load(b + j * THREADS + tid, c1);
      if (ONES && c1 - b <= THREADS * UNROLL / 2) {
#pragma unroll
        for (int j = 0; j < UNROLL / 2; ++j)
          if (b + j * THREADS < c1) f(b + j * THREADS + tid, Turn<1>{{t.raw[j]}});
      } else {
        f(b + tid, t);
      }
    }
  }
}

typedef u32x4 u32x4_any __attribute__((aligned(2), may_alias));   // a chunk at the address of any element

// Gradients go past the caches, which are left to the logits that are read again.
template <typename T>
__device__ __forceinline__ void store_chunk(T* to, const u32x4& v) {
  __builtin_nontemporal_store(v, reinterpret_cast<u32x4_any*>(to));
}

// The places of a chunk of `row` in a row of gradients of any alignment (its elements begin at `to`).
template <typename T>
__device__ __forceinline__ void store(const Row<T>& row, T* to, int c, const float (&f)[kEpc<T>]) {
  to += (long long)c * kEpc<T> - row.ph;
  if (row.whole(c)) {
    store_chunk(to, pack<T>(f));
  } else {
#pragma unroll
    for (int e = 0; e < kEpc<T>; ++e) {
      const int j = c * kEpc<T> + e - row.ph;
      if (j >= 0 && j < row.V) to[e] = (T)f[e];
    }
  }
}

// Running sums of a lane (or, after joining, of a workgroup).
struct Sums {
  float r, l, a;

  __device__ __forceinline__ Sums() : r(kNoRef), l(0.f), a(0.f) {}

  __device__ __forceinline__ void move(float m, float c) {
    const float d = vmax((r - m) * c, kFloor), w = exp2_fast(d);
    a = w * __builtin_fmaf(l, d, a);
    l *= w;
    r = m;
  }
  // The largest logit of some that are to come: the reference is moved to it if it is more than `rise` above.
  __device__ __forceinline__ void expect(float mx, float c, float rise) {
    const bool up = mx > r + rise;
    if (__any(up)) {
      if (up) move(mx, c);
    }
  }
  // The terms of a turn's logits. They are added among themselves first, in four chains: one chain of a row's terms would be
  // off by the roundings of V / THREADS additions (entropies 1.2e-7 instead of 6e-8 at 128000 logits and 512 threads; with
  // references moved at 24 doublings 1.2e-6).
  template <bool ENTROPY, int N, int E>
  __device__ __forceinline__ void add(const float (&f)[N][E], float c) {
    float ls[4] = {}, as[4] = {};
#pragma unroll
    for (int i = 0; i < N * E; ++i) {
      const float u = (f[i / E][i % E] - r) * c, e = exp2_fast(u);
      ls[i % 4] += e;
      if constexpr (ENTROPY) as[i % 4] = __builtin_fmaf(e, vmax(u, kFloor), as[i % 4]);   // a NaN stays in e
    }
    l += (ls[0] + ls[1]) + (ls[2] + ls[3]);
    if constexpr (ENTROPY) a += (as[0] + as[1]) + (as[2] + as[3]);
  }
};

__device__ __forceinline__ float first_lane(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, v)));
}

// The sums of the first WIDTH lanes of a wave, those of other WIDTH lanes being the same where WIDTH < 64, in every lane. It
// is the first lane's result: those of the others may be off by a rounding, where a product is fused into one addend.
template <int WIDTH>
__device__ __forceinline__ Sums lanes_join(Sums s, float c) {
  float m = s.r;
#pragma unroll
  for (int i = 1; i < WIDTH; i <<= 1) m = fmaxf(m, __shfl_xor(m, i));
  s.move(m, c);
#pragma unroll
  for (int i = 1; i < WIDTH; i <<= 1) {
    s.l += __shfl_xor(s.l, i);
    s.a += __shfl_xor(s.a, i);
  }
  s.r = first_lane(s.r);
  s.l = first_lane(s.l);
  s.a = first_lane(s.a);
  return s;
}

// The sums of a workgroup, in every thread. `red` holds 3 * THREADS / 64 floats and may be written again after the next
// barrier.
template <int THREADS>
__device__ __forceinline__ Sums block_join(Sums s, float c, float* red) {
  constexpr int W = THREADS / 64;
  static_assert(W > 1 && (W & (W - 1)) == 0, "");
  s = lanes_join<64>(s, c);
  const int w = threadIdx.x / 64;
  if (threadIdx.x % 64 == 0) {
    red[3 * w] = s.r;
    red[3 * w + 1] = s.l;
    red[3 * w + 2] = s.a;
  }
  __syncthreads();
  const int o = threadIdx.x % W;
  s.r = red[3 * o];
  s.l = red[3 * o + 1];
  s.a = red[3 * o + 2];
  return lanes_join<W>(s, c);
}

// log v for v > 0, off by about 2^-25: the logarithm of a number near 1, and the exponent in 64 bits.
__device__ __forceinline__ double log_of(double v) {
  int e;
  double m = frexp(v, &e);
  if (m < 0.70710678118654752) {
    m *= 2.0;
    --e;
  }
  return (double)e * 0.69314718055994530942 + (double)logf((float)m);
}

// exp(s x - lse) = 2^((x - at) c) f: what a log-sum-exp is for a kernel that forms probabilities, given as its float32
// value and what the rounding left off, both moderate (|lse| < 2^24).
struct Exponent {
  float at, f;
  __device__ __forceinline__ Exponent(float lse, float err, float scale) {
    at = (float)((double)lse / (double)scale);
    f = (float)exp(((double)scale * (double)at - (double)lse) - (double)err);   // the product is exact
  }
};

// A row of the grid: workgroup i of rows x parts, of which row r and part s.
__device__ __forceinline__ bool grid_place(long long rows, int parts, int* r, int* s) {
  const long long i = (long long)blockIdx.y * gridDim.x + blockIdx.x;
  if (i >= rows * parts) return false;
  *r = (int)(i / parts);
  *s = (int)(i - (long long)*r * parts);
  return true;
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------

// f(element) with a value of the type
template <typename F>
inline void by_type(int dtype, F f) {
  if (dtype == STREAMKL_F32)
    f(float{});
  else if (dtype == STREAMKL_F16)
    f(_Float16{});
  else
    f(__bf16{});
}

}  // namespace streamkl
