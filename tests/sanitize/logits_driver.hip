// Host-only driver for the sanitizer test of the C ABI of the operators on
// logits (tests/test_logits_sanitizers.py). Built together with logit_api.hip,
// both with AddressSanitizer and UndefinedBehaviorSanitizer on the host side;
// the launchers are replaced by stubs that check what the kernels count on.
#include <climits>
#include <cstdio>

#include "logit_launch.hpp"
#include "streamkl.h"

static int g_failures = 0;

static void fail(const char* what, int line) {
  ++g_failures;
  std::fprintf(stderr, "FAIL line %d: %s\n", line, what);
}
#define CHECK(x) \
  do {           \
    if (!(x)) fail(#x, __LINE__); \
  } while (0)

namespace streamkl {
static int g_launches = 0;

static bool f32(const LogitRows& r) { return r.dtype == STREAMKL_F32; }

// Parts of whole groups that cover a row of any alignment, on a grid of two axes that hold less than 2^32 threads each.
static void check_plan(const LogitRows& r, const LogitPlan& p, int most_parts) {
  ++g_launches;
  const long long rows = (long long)r.B * r.N, chunks = chunks_of(r.V, f32(r));
  CHECK(p.parts >= 1 && p.parts <= most_parts && p.chunks >= 4 && p.chunks % 4 == 0);
  CHECK((long long)p.parts * p.chunks >= chunks && (long long)(p.parts - 1) * p.chunks < chunks);
  CHECK(p.threads == 256 || p.threads == 512);
  const dim3 g = logit_grid(rows * p.parts);
  CHECK((long long)g.x * g.y >= rows * p.parts && (long long)g.x * 1024 < 1LL << 32 && g.y <= 1u << 16);
}

hipError_t launch_logprob(const LogprobArgs& a) {
  check_plan(a.rows, a.plan, kMostParts);
  if (a.top) CHECK((long long)a.plan.chunks * (f32(a.rows) ? 4 : 8) <= (long long)kMostGroups * kGroup);
  return hipSuccess;
}
hipError_t launch_logprob_grad(const LogprobGradArgs& a) {
  check_plan(a.rows, a.plan, 256);
  return hipSuccess;
}
hipError_t launch_distill(const DistillArgs& a) {
  check_plan(a.rows, a.plan, kMostParts);
  if (a.rest) CHECK(a.plan.chunks <= kMostMarks);
  return hipSuccess;
}
hipError_t launch_distill_grad(const DistillArgs& a) {
  check_plan(a.rows, a.plan, 256);
  return hipSuccess;
}
hipError_t launch_distill_step(const DistillArgs& a) {
  ++g_launches;
  CHECK(chunks_of(a.rows.V, f32(a.rows)) <= kMostMarks);
  return hipSuccess;
}
hipError_t launch_weighted_sum(const float*, const float*, float, long long, float*, hipStream_t) {
  ++g_launches;
  return hipSuccess;
}
}  // namespace streamkl

int main() {
  void* const p = reinterpret_cast<void*>(0x100000);
  float* const f = static_cast<float*>(p);
  const int ext[] = {-1, 0, 1, 2, 31, 127, 128, 129, 1000, 65535, 1 << 20, INT_MAX / 128, INT_MAX - 1, INT_MAX, INT_MIN};
  const int vocab[] = {-1, 0, 1, 7, 8, 1000, 50257, 131072, 262144, 270337, 4194303, 1 << 22, (1 << 22) + 1, INT_MAX, INT_MIN};
  const long long strides[] = {0, 1, 999, 1LL << 22, 1LL << 33, 1LL << 59, LLONG_MAX, -1, LLONG_MIN};
  const size_t huge = ~(size_t)0;
  int calls = 0;
  for (int B : ext)
    for (int N : ext)
      for (int V : vocab)
        for (int dtype : {0, 1, 2}) {
          const long long sb = strides[calls % 9], sn = strides[calls / 9 % 9];
          const streamkl_logits x = {p, sb, sn, B, N, V, dtype};
          for (int top : {0, 1, 128}) {
            ++calls;
            (void)streamkl_token_logprobs_workspace_bytes(B, N, V, dtype, top);
            int before = streamkl::g_launches;
            int st = streamkl_token_logprobs_fwd(&x, p, 0, 1.f, top, p, huge, f, f, f, f, f, static_cast<int*>(p), nullptr);
            CHECK(st == STREAMKL_OK || st == STREAMKL_ERR_INVALID_ARG || st == STREAMKL_ERR_UNSUPPORTED);
            CHECK(streamkl::g_launches == before + (st == STREAMKL_OK && B > 0 && N > 0));
            before = streamkl::g_launches;
            st = streamkl_token_logprobs_bwd(&x, p, 1, 1.f, f, f, f, f, f, f, p, sb, sn, nullptr);
            CHECK(st == STREAMKL_OK || st == STREAMKL_ERR_INVALID_ARG || st == STREAMKL_ERR_UNSUPPORTED);
            CHECK(streamkl::g_launches == before + (st == STREAMKL_OK && B > 0 && N > 0));
          }
          for (int rest : {0, 1}) {
            ++calls;
            const streamkl_teacher_list t = {p, p, 128, calls & 1, 2, rest, 1.f};
            (void)streamkl_topk_distill_workspace_bytes(B, N, V, dtype, rest);
            const int before = streamkl::g_launches;
            const int a = streamkl_topk_distill_fwd(&x, &t, 1.f, rest, p, huge, f, p, nullptr);
            const int b = streamkl_topk_distill_bwd(&x, &t, 1.f, rest, p, f, 1.f, f, rest, p, sb, sn, nullptr);
            const int between = streamkl::g_launches;
            const int c = streamkl_topk_distill_step(&x, &t, 1.f, rest, p, huge, f, 1.f, f, p, p, sb, sn, nullptr);
            const bool some = B > 0 && N > 0;
            CHECK(between == before + (some && a == STREAMKL_OK) + (some && b == STREAMKL_OK));
            CHECK(some && c == STREAMKL_OK ? streamkl::g_launches > between : streamkl::g_launches == between);
            CHECK((c == STREAMKL_OK) == (a == STREAMKL_OK && b == STREAMKL_OK));
          }
        }
  std::printf("%d calls, %d failures\n", calls, g_failures);
  return g_failures != 0;
}
