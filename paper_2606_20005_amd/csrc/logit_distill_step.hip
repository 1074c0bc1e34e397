// Loss and gradient of a distillation step in one kernel
// (streamkl_topk_distill_step); logit_distill.hpp has the mathematics.
//
// The upstream gradients are known beforehand, so a workgroup that has the sums
// of a row can write its gradient at once, and it still holds (much of) the
// row: a thread keeps HELD chunks of 16 bytes in registers. Chunks beyond that
// are read again out of the cache, the last ones first. So a logit is read from
// memory once and its gradient written, where a forward and a backward pass
// read it twice: two thirds of the bytes. Bound: HBM.
//
// A CU holds two workgroups of 512 threads, 8192 chunks each, so that one reads
// while the other finishes its row or writes. At 8192 x 128000 bf16, 64 entries
// (4.2 GB, 807 us at the rate of a large copy): 812 us; in two passes 1279 us.
// Where it took 828 us: one workgroup of 1024 threads that holds the whole row
// 1024 us; four of 256 960 us; 512 threads of 8 chunks 873 us; gradients kept
// in the caches 932 us; the chunks read again first to last 868 us. At 8192 x 262144 (three quarters
// read again, 1652 us) 1813 us.
//
// All loads of a row are issued before its list is read; the teacher's side is
// formed by one wave while they are on their way. Whole chunks only are held;
// the elements of the one or two that are not (rows begin anywhere) are one
// each in the first threads.
//
// The gradient of a listed logit is written by the thread that has written its
// chunk, after it: a wave's stores to one place arrive in order, so no barrier
// has to wait for them. Every thread finds its entries in a chained list in LDS.
#include "logit_distill.hpp"

namespace streamkl {
namespace {

constexpr int kTurn = 2;   // chunks that are summed at once

struct Upshot {
  float at, w;   // gradients outside the list: w 2^((x - at) c)
  int zero;      // no gradient
};

template <typename T, int THREADS, int HELD, bool REST, int WAVES>
__global__ void __launch_bounds__(THREADS, WAVES)
distill_step_kernel(DistillArgs a) {
  constexpr int E = kEpc<T>;
  __shared__ float red[3 * THREADS / 64];
  __shared__ List list;
  __shared__ Upshot up;
  __shared__ int head[THREADS];        // a thread's last entry, -1: none; the one before it in next
  __shared__ int next[kMostList];
  extern __shared__ u32 marks[];       // REST: a byte per chunk, a bit per listed logit
  int r, s;
  if (!grid_place((long long)a.rows.B * a.rows.N, 1, &r, &s)) return;
  const Row<T> row(a.rows, r);
  const int tid = threadIdx.x, V = row.V, ph = row.ph;
  // whole chunks c0 .. c1 - 1, elements before and behind them
  const int before = ph ? min(V, E - ph) : 0, c0 = ph ? 1 : 0, c1 = max(c0, (ph + V) / E);
  const int behind = max(before, c1 * E - ph);
  const int mine = tid < E ? (tid < before ? tid : -1) : tid < 2 * E && behind + tid - E < V ? behind + tid - E : -1;
  u32x4 held[HELD];
  if (c0 < c1) {
#pragma unroll
    for (int j = 0; j < HELD; ++j) held[j] = row.chunk[min(c0 + j * THREADS + tid, c1 - 1)];
  } else {
#pragma unroll
    for (int j = 0; j < HELD; ++j) held[j] = u32x4{0, 0, 0, 0};
  }
  float edge = mine >= 0 ? (float)row.row[mine] : kNegInf;
  if (tid == 0) list.some = list.bad = list.twice = 0;
  head[tid] = -1;
  if constexpr (REST)
    for (int i = tid; 4 * i < row.chunks; i += THREADS) marks[i] = 0;
  __syncthreads();
  read_list<T, THREADS>(a, r, row.row, list, [&](int k, int id) {
    const int at = id + ph, ch = at / E;
    if (REST) atomicOr(&marks[ch / 4], 1u << (8 * (ch % 4) + at % E));
    const int owner = id < before ? id : id >= behind ? E + id - behind : (ch - c0) % THREADS;
    next[k] = atomicExch(&head[owner], k);
  });
  __syncthreads();
  T* const dx = static_cast<T*>(a.dx) + (r / a.rows.N) * a.dsb + (r % a.rows.N) * a.dsn;
  if (list.some) {
    if (tid < 64) teacher_side(a, list);
    const unsigned char* const mark = reinterpret_cast<const unsigned char*>(marks);
    const float c = a.s2 * kLog2e, rise = kRise / c;
    Sums sums;
    // kTurn chunks of this thread, the first one ch, the others THREADS apart; those from c1 on are none
    auto sum = [&](int ch, const u32x4(&raw)[kTurn], bool all) {
      float f[kTurn][E], mx[kTurn];
#pragma unroll
      for (int j = 0; j < kTurn; ++j) {
        const bool there = all || ch + j * THREADS < c1;
        unpack<T>(raw[j], f[j]);
        if constexpr (REST) {
          leave_out(f[j], there ? mark[ch + j * THREADS] : (1u << E) - 1);
        } else if (!all) {
#pragma unroll
          for (int e = 0; e < E; ++e) f[j][e] = there ? f[j][e] : kNegInf;
        }
        mx[j] = max_of<T>(f[j]);
      }
      sums.expect(max_all(mx), c, rise);
      sums.template add<false>(f, c);
    };
#pragma unroll
    for (int j = 0; j < HELD; j += kTurn) {
      const int first = c0 + j * THREADS;
      if (first < c1) {
        const u32x4 raw[kTurn] = {held[j], held[j + 1]};
        sum(first + tid, raw, first + kTurn * THREADS <= c1);
      }
    }
    constexpr int ahead = 4;   // turns whose loads are in flight
    for (int first = c0 + HELD * THREADS; first < c1; first += ahead * kTurn * THREADS) {
      u32x4 raw[ahead][kTurn];
#pragma unroll
      for (int j = 0; j < ahead * kTurn; ++j) raw[j / kTurn][j % kTurn] = row.chunk[min(first + j * THREADS + tid, c1 - 1)];
#pragma unroll
      for (int h = 0; h < ahead; ++h) {
        const int at = first + h * kTurn * THREADS;
        if (at < c1) sum(at + tid, raw[h], at + kTurn * THREADS <= c1);
      }
    }
    {
      const int at = mine + ph;
      const bool listed = REST && mine >= 0 && (mark[at / E] >> (at % E)) & 1;
      const float f[1][1] = {{listed ? kNegInf : edge}};
      sums.expect(f[0][0], c, rise);
      sums.template add<false>(f, c);
    }
    sums = block_join<THREADS>(sums, c, red);
    if (tid < 64) {
      float loss;
      const DistillStats st = finish_row(a, sums, list, &loss);
      const float g = upstream(a, r);
      listed_gradients(a, st, g, list);
      if (tid == 0) {
        a.loss[r] = loss;
        a.stats[r] = st;
        up = Upshot{st.r, (float)((double)a.s2 * (double)g * st.rest), g == 0.f || st.lse == (double)kNegInf};
      }
    }
    __syncthreads();
    if (!up.zero) {
      const float at = up.at, w = up.w;
      auto put = [&](int ch, const u32x4& raw) {
        float f[E];
        unpack<T>(raw, f);
#pragma unroll
        for (int i = 0; i < E; ++i) f[i] = exp2_fast((f[i] - at) * c) * w;
        if (ch < c1) store_chunk(dx + ((long long)ch * E - ph), pack<T>(f));
      };
      // the chunks that were read last first: they are in the nearest cache
      constexpr int back = 8;
      const int held_to = c0 + HELD * THREADS, turns = (c1 - held_to + back * THREADS - 1) / (back * THREADS);
      for (int t = turns - 1; t >= 0; --t) {
        const int first = held_to + t * back * THREADS;
        u32x4 raw[back];
#pragma unroll
        for (int j = back - 1; j >= 0; --j) raw[j] = row.chunk[min(first + j * THREADS + tid, c1 - 1)];
#pragma unroll
        for (int j = back - 1; j >= 0; --j) put(first + j * THREADS + tid, raw[j]);
      }
#pragma unroll
      for (int j = 0; j < HELD; ++j)
        if (c0 + j * THREADS < c1) put(c0 + j * THREADS + tid, held[j]);
      if (mine >= 0) dx[mine] = (T)(exp2_fast((edge - at) * c) * w);
      for (int k = head[tid]; k >= 0; k = next[k]) dx[list.id[k]] = (T)list.value[k];
      return;
    }
  } else if (tid == 0) {
    a.loss[r] = 0.f;
    a.stats[r] = DistillStats{0.f, 0.f, (double)kNegInf, 0.0, 0.0};
  }
  for (int ch = c0 + tid; ch < c1; ch += THREADS)
    store_chunk(dx + ((long long)ch * E - ph), u32x4{0, 0, 0, 0});
  if (mine >= 0) dx[mine] = (T)0.f;
}

template <typename T, int THREADS, int HELD>
void run(const DistillArgs& a) {
  // waves a SIMD that the registers held leave room for
  constexpr int waves = HELD <= 4 ? 6 : 4;
  const long long rows = (long long)a.rows.B * a.rows.N;
  if (a.rest)
    distill_step_kernel<T, THREADS, HELD, true, waves>
        <<<logit_grid(rows), dim3(THREADS), (size_t)(chunks_of(a.rows.V, a.rows.dtype == STREAMKL_F32) + 3) / 4 * 4, a.stream>>>(a);
  else
    distill_step_kernel<T, THREADS, HELD, false, waves><<<logit_grid(rows), dim3(THREADS), 0, a.stream>>>(a);
}

}  // namespace

hipError_t launch_distill_step(const DistillArgs& a) {
  const int chunks = chunks_of(a.rows.V, a.rows.dtype == STREAMKL_F32);
  by_type(a.rows.dtype, [&](auto t) {
    using T = decltype(t);
    if (chunks <= 1024)
      run<T, 256, 4>(a);
    else if (chunks <= 4096)
      run<T, 256, 16>(a);
    else
      run<T, 512, 16>(a);
  });
  return hipGetLastError();
}

}  // namespace streamkl
