// C ABI of differential attention: argument checks and dispatch. Every check
// happens before anything is enqueued.
#include <cmath>
#include <cstdint>

#include "diff_launch.hpp"
#include "streamkl.h"

namespace streamkl {
namespace {

// From the runtime key dim to the unit that serves it.
DiffFwdShape diff_fwd_shape(int d, int dv, long long rows) {
  return diff_by_key_dim(d, [&](auto kd) { return diff_fwd_shape_of<kd.value>(dv, rows); });
}
hipError_t launch_diff_fwd(const DiffArgs& a) {
  return diff_by_key_dim(a.d, [&](auto kd) { return launch_diff_fwd_of<kd.value>(a); });
}
int diff_bwd_dq_waves(int d, int dv) {
  return diff_by_key_dim(d, [&](auto kd) { return diff_bwd_dq_waves_of<kd.value>(dv); });
}
int diff_bwd_dq_rows(int d, int dv) {
  return diff_by_key_dim(d, [&](auto kd) { return diff_bwd_dq_rows_of<kd.value>(dv); });
}
int diff_bwd_dkv_waves(int d, int dv) {
  return diff_by_key_dim(d, [&](auto kd) { return diff_bwd_dkv_waves_of<kd.value>(dv); });
}
hipError_t launch_diff_bwd_dq(const DiffArgs& a) {
  return diff_by_key_dim(a.d, [&](auto kd) { return launch_diff_bwd_dq_of<kd.value>(a); });
}
hipError_t launch_diff_bwd_dkv(const DiffArgs& a) {
  return diff_by_key_dim(a.d, [&](auto kd) { return launch_diff_bwd_dkv_of<kd.value>(a); });
}

}  // namespace
}  // namespace streamkl

namespace {

using streamkl::DiffArgs;
using streamkl::DiffRows;

constexpr long long kMaxInt = 0x7fffffffLL, kMaxBlocks = (1LL << 24) - 1;

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// Rows of one input; `used`: it has elements that a kernel may read.
int check_rows(const streamkl_rows* x, bool used) {
  if (!x) return STREAMKL_ERR_INVALID_ARG;
  if (!used) return STREAMKL_OK;
  if (!x->data || !aligned(x->data, 16)) return STREAMKL_ERR_INVALID_ARG;
  if (x->sb < 0 || x->sh < 0 || x->sn < 0 || x->sb % 8 || x->sh % 8 || x->sn % 8) return STREAMKL_ERR_INVALID_ARG;
  // a tile of 32 rows is addressed with 31-bit byte offsets
  if (x->sn >= 1LL << 25) return STREAMKL_ERR_UNSUPPORTED;
  return STREAMKL_OK;
}

int check_extents(int B, int H, int HK, int N_Q, int N_K, int d, int dv) {
  if (B < 0 || H < 0 || HK < 0 || N_Q < 0 || N_K < 0) return STREAMKL_ERR_INVALID_ARG;
  if (H > 0 && (HK == 0 || H % HK != 0)) return STREAMKL_ERR_INVALID_ARG;
  if (H == 0 && HK != 0) return STREAMKL_ERR_INVALID_ARG;
  if (!streamkl::diff_dims(d, dv)) return STREAMKL_ERR_UNSUPPORTED;
  const long long bh = (long long)B * H;
  // rows and 128-row blocks are counted in 31 bits
  if (bh > kMaxInt || (H && (long long)N_Q * (H / HK) > kMaxInt - 256) || (bh && N_Q > (kMaxInt - 256) / bh))
    return STREAMKL_ERR_UNSUPPORTED;
  if (N_K > kMaxInt - 256) return STREAMKL_ERR_UNSUPPORTED;
  // and an axis of a grid holds less than 2^32 threads, 256 a tile of 32 rows or a block of 64 keys
  if (bh * ((N_Q + 31LL) / 32) > kMaxBlocks || (long long)B * HK * ((N_K + 63LL) / 64) > kMaxBlocks)
    return STREAMKL_ERR_UNSUPPORTED;
  return STREAMKL_OK;
}

bool scale_ok(float s) { return std::isfinite(s) && s >= 0x1p-64f && s <= 0x1p64f; }

DiffRows rows_of(const streamkl_rows* x) {
  return DiffRows{static_cast<const uint16_t*>(x->data), x->sb, x->sh, x->sn};
}

int check_inputs(const streamkl_rows* q1, const streamkl_rows* k1, const streamkl_rows* q2, const streamkl_rows* k2,
                 const streamkl_rows* v, int B, int H, int HK, int N_Q, int N_K, int d, int dv, float scale, int causal,
                 const float* lam, const int* q_len, const int* kv_len, hipStream_t stream, DiffArgs* a) {
  if (causal != 0 && causal != 1) return STREAMKL_ERR_INVALID_ARG;
  int st = check_extents(B, H, HK, N_Q, N_K, d, dv);
  if (st != STREAMKL_OK) return st;
  if (!scale_ok(scale)) return STREAMKL_ERR_INVALID_ARG;
  const bool rows = (long long)B * H * N_Q != 0, keys = (long long)B * HK * N_K != 0;
  const streamkl_rows* in[] = {q1, q2, k1, k2, v};
  for (int i = 0; i < 5; ++i) {
    st = check_rows(in[i], i < 2 ? rows : keys);
    if (st != STREAMKL_OK) return st;
  }
  if (H > 0 && (!lam || !aligned(lam, 4))) return STREAMKL_ERR_INVALID_ARG;
  if ((q_len && !aligned(q_len, 4)) || (kv_len && !aligned(kv_len, 4))) return STREAMKL_ERR_INVALID_ARG;
  *a = DiffArgs{};
  a->q1 = rows_of(q1);
  a->k1 = rows_of(k1);
  a->q2 = rows_of(q2);
  a->k2 = rows_of(k2);
  a->v = rows_of(v);
  a->B = B;
  a->H = H;
  a->HK = HK;
  a->NQ = N_Q;
  a->NK = N_K;
  a->d = d;
  a->dv = dv;
  a->scale = scale;
  a->causal = causal;
  a->lam = lam;
  a->q_len = q_len;
  a->kv_len = kv_len;
  a->splits = 1;
  a->stream = stream;
  return STREAMKL_OK;
}

// Share of the pairs that the mask leaves.
double visible_share(int N_Q, int N_K, int causal) {
  return !causal ? 1.0 : N_Q <= N_K ? 1.0 - 0.5 * N_Q / N_K : 0.5 * N_K / N_Q;
}

// Ranges of the streamed axis in the backward kernels. A kernel's blocks own
// 128 rows (keys) and walk over all keys (rows) of their head; where that
// leaves the chip unevenly filled, the walk is cut into ranges whose partial
// float32 gradients a further kernel adds up. The number of ranges is the one
// with the least estimated time: rounds of resident workgroups times steps,
// about 0.042 us an MFMA and resident wave of a SIMD, and the partials written and
// read back at 4 TB/s. The estimate is that of the kernels with 32 rows (keys) a
// wave (measured 0.038 to 0.048 us); where those with 16 run, with half of the rows
// a block and two workgroups a CU, it only ranks the counts. Measured, us, with
// the statistics and the joins, one range, the choice and the best of 1, 2, 3, 4,
// 6, 8, 16 and 32: dQ of 16 heads x 64 rows against 65536 keys, d 128/128, 1591,
// 172 and 163; dK dV of 4 x 12 heads x 1021 ragged rows on 4 key heads, d 96/160
// causal, 110, 91 and 83; both of 8 heads x 6007, d 128/128, 404, 405 and 404, 522,
// 510 and 509; of 6 heads x 3001 causal, 96/96, 83, 67 and 65, 103, 80 and 79; of 4
// heads x 3001 causal on 2 key heads, 128/256, 100, 76 and 65, 526, 165 and 142.
struct GradSplits {
  int q, k;
  size_t part_floats;
};

int grad_splits(long long blocks, int waves, long long steps, double share, int mfmas, double bytes) {
  const double slots = 256.0 * waves, us = 0.042 * mfmas * waves;
  int best = 1;
  double least = 0;
  for (int s = 1; s <= streamkl::kDiffMaxGradSplits; ++s) {
    if (s > 1 && steps < 4LL * s) break;
    const double rounds = (double)blocks * s / slots, each = (double)steps / s;
    const double filled = rounds > 8 ? rounds * each : std::ceil(rounds) * each, even = share * rounds * each;
    // causal blocks are handed out longest first; a part of the longest is left over
    double t = (share > 0.75 ? filled : (even > each ? even : each) + 0.15 * each) * us;
    if (s > 1) t += (s + 1) * bytes / 4e6 + 8.0;
    if (s == 1 || t < 0.95 * least) {
      best = s;
      least = t;
    }
  }
  return best;
}

GradSplits bwd_splits(int B, int H, int HK, int N_Q, int N_K, int d, int dv, int causal) {
  GradSplits g = {1, 1, 0};
  if ((long long)B * H * N_Q == 0 || (long long)B * HK * N_K == 0) return g;
  const long long q_floats = 2LL * B * H * N_Q * d, k_floats = (long long)B * HK * N_K * (2 * d + dv);
  g.q = grad_splits((long long)B * H * streamkl::diff_row_blocks(N_Q), streamkl::diff_bwd_dq_waves(d, dv),
                    (N_K + 31LL) / 32, visible_share(N_Q, N_K, causal), d / 4 + dv / 16, 4.0 * q_floats);
  g.k = grad_splits((long long)B * HK * streamkl::diff_row_blocks(N_K), streamkl::diff_bwd_dkv_waves(d, dv),
                    (long long)(H / HK) * ((N_Q + 31LL) / 32), visible_share(N_Q, N_K, causal), d / 4 + dv / 8, 4.0 * k_floats);
  const long long q_part = g.q > 1 ? g.q * q_floats : 0, k_part = g.k > 1 ? g.k * k_floats : 0;
  g.part_floats = (size_t)(q_part > k_part ? q_part : k_part);
  return g;
}

int hip_status(hipError_t e) { return e == hipSuccess ? STREAMKL_OK : STREAMKL_ERR_HIP; }

}  // namespace

// The split count with the least estimated time. A workgroup takes 0.07 us for
// an MFMA of a tile where two share a CU, 0.045 alone (measured 0.065 to 0.08
// and 0.04 to 0.05 over the head dims); a grid of up to two workgroups per CU
// takes as long as its longest range, a larger one as many rounds, causal ones
// (longest block first) their share of the pairs. Keys and values come at 5.5
// TB/s from 512 workgroups on; the float32 partials are written and read back
// at 4 TB/s by a second launch.
extern "C" int streamkl_diff_fwd_split_count(int B, int H, int HK, int N_Q, int N_K, int d, int dv, int causal) {
  if (check_extents(B, H, HK, N_Q, N_K, d, dv) != STREAMKL_OK) return 0;
  if ((long long)B * H * N_Q == 0) return 1;
  const long long R = (long long)N_Q * (H / HK);
  const streamkl::DiffFwdShape w = streamkl::diff_fwd_shape(d, dv, R);
  const long long base = (long long)B * HK * ((R + w.rows - 1) / w.rows), tiles = (N_K + 31LL) / 32;
  const double partials = 16.0 * B * H * (double)N_Q * (dv + 2);
  const double bytes = 2.0 * B * HK * (double)N_K * (2 * d + dv);
  const double share = visible_share(N_Q, N_K, causal);
  const double slots = 2.0 * streamkl::kCus;
  int best = 1;
  double least = 0;
  for (long long s = 1; s <= streamkl::kDiffMaxSplits && (s == 1 || (s * 4 <= tiles && base * s <= 4 * slots)); ++s) {
    const double wgs = (double)base * s, even = share * wgs / slots;
    // a last round of at most one workgroup per CU runs at 0.045 / 0.07
    const double whole = std::floor(wgs / slots), left = wgs - whole * slots;
    const double filled = whole + (left == 0 ? 0.0 : left <= 0.5 * slots ? 0.64 : 1.0);
    const double rounds = wgs <= slots || even < 1 ? 1 : causal || wgs > 4 * slots ? even : filled;
    const double work = rounds * tiles / s * w.mfmas * (wgs > 0.5 * slots ? 0.07 : 0.045);
    const double mem = bytes / 5.5e6 * (wgs < slots ? slots / wgs : 1.0);
    const double t = (work > mem ? work : mem) + (s > 1 ? partials * s / 4e6 + 6.0 : 0.0);
    if (s == 1 || t < 0.95 * least) {
      best = (int)s;
      least = t;
    }
  }
  return best;
}

extern "C" size_t streamkl_diff_fwd_workspace_bytes(int B, int H, int N_Q, int dv, int splits) {
  if (B < 0 || H < 0 || N_Q < 0 || dv < 0 || splits <= 1 || splits > streamkl::kDiffMaxSplits) return 0;
  return (size_t)B * H * N_Q * splits * 2 * (dv + 2) * sizeof(float);
}

extern "C" int streamkl_diff_fwd(const streamkl_rows* q1, const streamkl_rows* k1, const streamkl_rows* q2,
                                 const streamkl_rows* k2, const streamkl_rows* v, int B, int H, int HK, int N_Q,
                                 int N_K, int d, int dv, float scale, int causal, const float* lam, const int* q_len,
                                 const int* kv_len, int splits, void* workspace, size_t workspace_bytes, void* out,
                                 void* out2, float* lse1, float* lse2, hipStream_t stream) {
  DiffArgs a;
  const int st = check_inputs(q1, k1, q2, k2, v, B, H, HK, N_Q, N_K, d, dv, scale, causal, lam, q_len, kv_len, stream,
                              &a);
  if (st != STREAMKL_OK) return st;
  if (splits < 1) return STREAMKL_ERR_INVALID_ARG;
  if (splits > streamkl::kDiffMaxSplits || (splits > 1 && (long long)B * H * N_Q > kMaxBlocks)) return STREAMKL_ERR_UNSUPPORTED;
  if ((long long)B * H * N_Q == 0) return STREAMKL_OK;
  if (splits > 1 && (!workspace || !aligned(workspace, 16) ||
                     workspace_bytes < streamkl_diff_fwd_workspace_bytes(B, H, N_Q, dv, splits)))
    return STREAMKL_ERR_INVALID_ARG;
  if (!out || !aligned(out, 16) || (out2 && !aligned(out2, 16))) return STREAMKL_ERR_INVALID_ARG;
  if ((lse1 && !aligned(lse1, 4)) || (lse2 && !aligned(lse2, 4))) return STREAMKL_ERR_INVALID_ARG;
  a.splits = splits;
  a.part = static_cast<float*>(workspace);
  a.out = static_cast<uint16_t*>(out);
  a.out2 = static_cast<uint16_t*>(out2);
  a.lse1 = lse1;
  a.lse2 = lse2;
  hipError_t e = streamkl::launch_diff_fwd(a);
  if (e == hipSuccess && splits > 1) e = streamkl::launch_diff_merge(a);
  return hip_status(e);
}

extern "C" size_t streamkl_diff_bwd_workspace_bytes(int B, int H, int HK, int N_Q, int N_K, int d, int dv, int causal) {
  if (check_extents(B, H, HK, N_Q, N_K, d, dv) != STREAMKL_OK) return 0;
  const GradSplits g = bwd_splits(B, H, HK, N_Q, N_K, d, dv, causal);
  return (streamkl::diff_bwd_stats_floats(B, H, N_Q) + streamkl::diff_bwd_dlam_floats(B, H, N_Q, g.q) + g.part_floats) *
         sizeof(float);
}

extern "C" int streamkl_diff_bwd(const streamkl_rows* q1, const streamkl_rows* k1, const streamkl_rows* q2,
                                 const streamkl_rows* k2, const streamkl_rows* v, int B, int H, int HK, int N_Q,
                                 int N_K, int d, int dv, float scale, int causal, const float* lam, const int* q_len,
                                 const int* kv_len, const void* dout, const void* out, const void* out2,
                                 const float* lse1, const float* lse2, void* workspace, size_t workspace_bytes,
                                 void* dq1, void* dk1, void* dq2, void* dk2, void* dvalues, float* dlam,
                                 int bf16_grads, hipStream_t stream) {
  DiffArgs a;
  const int st = check_inputs(q1, k1, q2, k2, v, B, H, HK, N_Q, N_K, d, dv, scale, causal, lam, q_len, kv_len, stream,
                              &a);
  if (st != STREAMKL_OK) return st;
  if (bf16_grads != 0 && bf16_grads != 1) return STREAMKL_ERR_INVALID_ARG;
  if (!dq1 && !dk1 && !dq2 && !dk2 && !dvalues && !dlam) return STREAMKL_ERR_INVALID_ARG;
  const bool rows = (long long)B * H * N_Q != 0, keys = (long long)B * HK * N_K != 0;
  const bool of_rows = dq1 || dq2 || dlam, of_keys = dk1 || dk2 || dvalues;
  const void* f32[] = {lse1, lse2, dlam, dq1, dk1, dq2, dk2, dvalues};
  for (const void* p : f32)
    if (p && !aligned(p, 4)) return STREAMKL_ERR_INVALID_ARG;
  if (rows) {
    if (!dout || !out || !out2 || !lse1 || !lse2) return STREAMKL_ERR_INVALID_ARG;
    if (!aligned(dout, 16) || !aligned(out, 16) || !aligned(out2, 16)) return STREAMKL_ERR_INVALID_ARG;
    if (!workspace || !aligned(workspace, 16) || 
        workspace_bytes < streamkl_diff_bwd_workspace_bytes(B, H, HK, N_Q, N_K, d, dv, causal))
      return STREAMKL_ERR_INVALID_ARG;
  }
  a.dout = static_cast<const uint16_t*>(dout);
  a.out = static_cast<uint16_t*>(const_cast<void*>(out));     // read only here
  a.out2 = static_cast<uint16_t*>(const_cast<void*>(out2));
  a.lse1 = const_cast<float*>(lse1);
  a.lse2 = const_cast<float*>(lse2);
  a.stats = static_cast<float*>(workspace);
  const GradSplits g = bwd_splits(B, H, HK, N_Q, N_K, d, dv, causal);
  a.q_splits = g.q;
  a.k_splits = g.k;
  const int rows_each = streamkl::diff_bwd_dq_rows(d, dv);
  a.row_blocks = (int)(((long long)N_Q + rows_each - 1) / rows_each);
  if (a.stats) {
    float* part = a.stats + streamkl::diff_bwd_stats_floats(B, H, N_Q);   // whole tiles of statistics: 16-byte aligned
    a.dlam_part = reinterpret_cast<double*>(part);
    a.grad_part = part + streamkl::diff_bwd_dlam_floats(B, H, N_Q, g.q);
  }
  a.dq1 = dq1;
  a.dk1 = dk1;
  a.dq2 = dq2;
  a.dk2 = dk2;
  a.dv_out = dvalues;
  a.dlam = dlam;
  a.bf16_grads = bf16_grads;
  hipError_t e = hipSuccess;
  if (rows) e = streamkl::launch_diff_bwd_prep(a);
  if (e == hipSuccess && keys && of_keys) e = streamkl::launch_diff_bwd_dkv(a);   // without rows: zeros
  if (e == hipSuccess && keys && of_keys && g.k > 1) e = streamkl::launch_diff_bwd_join_k(a);
  if (e == hipSuccess && rows && of_rows) e = streamkl::launch_diff_bwd_dq(a);
  if (e == hipSuccess && rows && of_rows && g.q > 1) e = streamkl::launch_diff_bwd_join_q(a);
  if (e == hipSuccess && dlam && H > 0) e = streamkl::launch_diff_bwd_dlam(a);
  return hip_status(e);
}
