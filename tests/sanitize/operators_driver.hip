// Host-only driver for the sanitizer test of the operators' C ABI
// (tests/test_operators_sanitizers.py). Built together with diff_api.hip and
// norm_rope.hip, all with AddressSanitizer and UndefinedBehaviorSanitizer on
// the host side; the launchers of differential attention are replaced by
// stubs. Checked is that refusals reach no launcher and that the arithmetic of
// extents, sizes and grids stays defined at any extents.
#include <climits>
#include <cstdio>

#include "diff_launch.hpp"
#include "streamkl.h"

namespace streamkl {
static int g_launches = 0;
static hipError_t stub() {
  ++g_launches;
  return hipSuccess;
}
#define KEY_DIM(D)                                                                             \
  template <>                                                                                  \
  DiffFwdShape diff_fwd_shape_of<D>(int, long long rows) { return {rows <= 32 ? 32 : 128, 24}; } \
  template <>                                                                                  \
  hipError_t launch_diff_fwd_of<D>(const DiffArgs&) { return stub(); }                         \
  template <>                                                                                  \
  int diff_bwd_dq_waves_of<D>(int) { return 2; }                                               \
  template <>                                                                                  \
  int diff_bwd_dq_rows_of<D>(int) { return 64; }                                               \
  template <>                                                                                  \
  int diff_bwd_dkv_waves_of<D>(int) { return 1; }                                              \
  template <>                                                                                  \
  hipError_t launch_diff_bwd_dq_of<D>(const DiffArgs&) { return stub(); }                      \
  template <>                                                                                  \
  hipError_t launch_diff_bwd_dkv_of<D>(const DiffArgs&) { return stub(); }
KEY_DIM(32)
KEY_DIM(64)
KEY_DIM(96)
KEY_DIM(128)
hipError_t launch_diff_merge(const DiffArgs&) { return stub(); }
size_t diff_bwd_stats_floats(int B, int H, int NQ) { return (size_t)B * H * ((NQ + 31LL) / 32) * 128; }
size_t diff_bwd_dlam_floats(int B, int H, int NQ, int s) { return (size_t)B * H * diff_row_blocks(NQ) * s; }
hipError_t launch_diff_bwd_prep(const DiffArgs&) { return stub(); }
hipError_t launch_diff_bwd_join_q(const DiffArgs&) { return stub(); }
hipError_t launch_diff_bwd_join_k(const DiffArgs&) { return stub(); }
hipError_t launch_diff_bwd_dlam(const DiffArgs&) { return stub(); }
}  // namespace streamkl

static int g_failures = 0;

static void fail(const char* what, int line) {
  ++g_failures;
  std::fprintf(stderr, "FAIL line %d: %s\n", line, what);
}
#define CHECK(x) \
  do {           \
    if (!(x)) fail(#x, __LINE__); \
  } while (0)

int main() {
  void* const p = reinterpret_cast<void*>(0x100000);
  float* const f = static_cast<float*>(p);
  const streamkl_rows ok = {p, 0, 512, 64}, far = {p, LLONG_MAX / 8 * 8, LLONG_MAX / 8 * 8, (1LL << 25) - 8};
  const int ext[] = {-1, 0, 1, 2, 31, 32, 33, 127, 1000, 65535, 1 << 20, INT_MAX / 128, INT_MAX - 1, INT_MAX, INT_MIN};
  const size_t huge = ~(size_t)0;
  int calls = 0;
  for (int B : ext)
    for (int H : ext)
      for (int N : ext) {
        for (int HK : {H, 1, 0})
          for (int M : {N, 1, INT_MAX, 4096}) {
            for (int causal : {0, 1}) {
              ++calls;
              const int s = streamkl_diff_fwd_split_count(B, H, HK, N, M, 64, 128, causal);
              CHECK(s >= 0 && s <= 256);
              (void)streamkl_diff_fwd_workspace_bytes(B, H, N, 128, s);
              (void)streamkl_diff_bwd_workspace_bytes(B, H, HK, N, M, 64, 128, causal);
              const streamkl_rows* r = (calls & 1) ? &ok : &far;
              int before = streamkl::g_launches;
              int st = streamkl_diff_fwd(r, r, r, r, r, B, H, HK, N, M, 64, 128, 0.125f, causal, f, nullptr, nullptr,
                                         s < 1 ? 1 : s, p, huge, p, p, f, f, nullptr);
              CHECK(st == STREAMKL_OK || st == STREAMKL_ERR_INVALID_ARG || st == STREAMKL_ERR_UNSUPPORTED);
              if (st != STREAMKL_OK || B == 0 || H == 0 || N == 0) CHECK(streamkl::g_launches == before);
              if (st == STREAMKL_OK && B > 0 && H > 0 && N > 0) CHECK(streamkl::g_launches == before + (s > 1 ? 2 : 1));
              before = streamkl::g_launches;
              st = streamkl_diff_bwd(r, r, r, r, r, B, H, HK, N, M, 64, 128, 0.125f, causal, f, nullptr, nullptr, p, p, p,
                                     f, f, p, huge, p, p, p, p, p, f, 1, nullptr);
              CHECK(st == STREAMKL_OK || st == STREAMKL_ERR_INVALID_ARG || st == STREAMKL_ERR_UNSUPPORTED);
              if (st != STREAMKL_OK) CHECK(streamkl::g_launches == before);
            }
            (void)streamkl_qk_norm_rope_bwd_workspace_bytes(B, H, HK, N, M, 128);
            // refused before any launch: a workspace that is too small, a table that is missing
            const int st = streamkl_qk_norm_rope_bwd(&ok, &ok, B, H, HK, N, M, 64, STREAMKL_BF16, f, f, 1e-6f, nullptr, 8,
                                                     64, 0, nullptr, nullptr, 0, 0, 0, INT_MAX, p, p, STREAMKL_F32, p, 0,
                                                     p, p, f, f, nullptr);
            CHECK(st == STREAMKL_ERR_INVALID_ARG || st == STREAMKL_ERR_UNSUPPORTED);
            const int st2 = streamkl_qk_norm_rope_fwd(&far, &ok, B, H, HK, N, M, 64, STREAMKL_F32, f, f, 1e-6f, f, 8, 64,
                                                      0, nullptr, nullptr, 0, 0, 0, 0, p, p, nullptr);
            CHECK(st2 == STREAMKL_ERR_INVALID_ARG || st2 == STREAMKL_ERR_UNSUPPORTED);
          }
      }
  std::printf("%d calls, %d failures\n", calls, g_failures);
  return g_failures != 0;
}
