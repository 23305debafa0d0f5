// Host-side driver for the AddressSanitizer / UndefinedBehaviorSanitizer build of
// the entry points over rows of logits (rp_logits.hip). Built and run by
// tests/test_sanitize_rows.py, without a GPU: launches, and what the rest of the
// library gives these calls, are stand-ins here that record what they are given.
// Device addresses are fake and never read.
#include <hip/hip_runtime_api.h>

#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <limits>
#include <string>

#include "rp.h"
#include "rp_internal.h"

namespace {

std::string g_error;
int g_launches = 0;
size_t g_need = 0;
rp::LogitArgs g_rows{};

hipError_t launched(const rp::LogitArgs& l) {
  ++g_launches;
  g_rows = l;
  return hipSuccess;
}

}  // namespace

namespace rp {

void clear_error() { g_error.clear(); }
rp_status set_error(rp_status st, const char* text) {
  g_error = text;
  return st;
}
rp_status device_cus(int* cus) {
  *cus = 256;
  return RP_OK;
}
size_t sample_workspace(int, int, int) { return g_need; }
hipError_t launch_sample(const SampleArgs& a, int, hipStream_t) { return launched(a.logits); }
hipError_t launch_logprobs(const LogprobArgs& a, int, hipStream_t) { return launched(a.logits); }
hipError_t launch_policy(const PolicyArgs& a, int, hipStream_t) { return launched(a.logits); }
hipError_t launch_distill(const DistillArgs& a, int, hipStream_t) { return launched(a.logits); }

}  // namespace rp

namespace {

int g_fail = 0;
#define EXPECT(cond)                                                                                             \
  do {                                                                                                           \
    if (!(cond)) {                                                                                               \
      std::fprintf(stderr, "FAILED %s:%d: %s (last error: %s)\n", __FILE__, __LINE__, #cond, g_error.c_str());   \
      ++g_fail;                                                                                                  \
    }                                                                                                            \
  } while (0)

void* at(uint64_t address) { return reinterpret_cast<void*>(static_cast<uintptr_t>(address)); }
float* const F = static_cast<float*>(at(0x10000000));
int32_t* const I = static_cast<int32_t*>(at(0x10000000));
constexpr uint64_t kRows = 0x7f0000000000, kGrad = 0x7e0000000000;

rp_logits rows(int32_t n = 4, int32_t vocab = 100, int64_t stride = 104, int dtype = RP_LOGITS_BF16, uint64_t data = kRows) {
  return {at(data), n, vocab, stride, static_cast<rp_logits_dtype>(dtype)};
}
rp_policy_batch batch() { return {I, F, F, F, I, 3, F, 1.0, 0.2, 0.2, 0.1, 0.0}; }
rp_teacher teacher() { return {I, F, 8, RP_DISTILL_TAIL, F, 1.0}; }

rp_status sample(const rp_logits& l, const rp_sampling* how = nullptr) {
  return rp_sample_tokens(&l, how, F, I, F, F, at(4096), size_t(1) << 40, nullptr);
}
rp_status logprobs(const rp_logits& l, double t = 1.0) {
  return rp_token_logprobs(&l, I, t, F, F, at(4096), size_t(1) << 40, nullptr);
}
rp_status policy(const rp_logits& l, const rp_policy_batch& b, uint64_t grad = kGrad, int64_t stride = 104) {
  return rp_policy_loss(&l, &b, F, F, F, at(grad), stride, at(4096), size_t(1) << 40, nullptr);
}
rp_status distill(const rp_logits& l, const rp_teacher& t, uint64_t grad = kGrad, int64_t stride = 104) {
  return rp_distill_loss(&l, &t, F, at(grad), stride, at(4096), size_t(1) << 40, nullptr);
}

void every_call_reaches_its_launch() {
  const rp_logits l = rows();
  const rp_sampling how = {F, I, F, F};
  size_t bytes = 1;
  EXPECT(rp_logits_workspace_size(&l, &bytes) == RP_OK && bytes == 0);
  g_launches = 0;
  EXPECT(sample(l) == RP_OK && sample(l, &how) == RP_OK && logprobs(l) == RP_OK && policy(l, batch()) == RP_OK &&
         distill(l, teacher()) == RP_OK && policy(l, batch(), 0, 0) == RP_OK && distill(l, teacher(), 0, 0) == RP_OK);
  EXPECT(g_launches == 7 && g_rows.num_cus == 256 && g_rows.stride == 104);
}

void refusals_of_rows() {
  struct Case { rp_logits l; rp_status want; };
  const Case cases[] = {
      {rows(-1), RP_ERR_INVALID_ARG},
      {rows(4, 0), RP_ERR_INVALID_ARG},
      {rows(4, (1 << 20) + 1, 1 << 21), RP_ERR_UNSUPPORTED},
      {rows(4, 100, 99), RP_ERR_INVALID_ARG},
      {rows(4, 100, int64_t(1) << 31), RP_ERR_INVALID_ARG},
      {rows(4, 100, INT64_MIN), RP_ERR_INVALID_ARG},
      {rows(4, 100, 104, 3), RP_ERR_UNSUPPORTED},
      {rows(4, 100, 104, -1), RP_ERR_UNSUPPORTED},
      {rows(4, 100, 104, RP_LOGITS_F32, kRows + 2), RP_ERR_INVALID_ARG},
      {rows(4, 100, 104, RP_LOGITS_F16, kRows + 1), RP_ERR_INVALID_ARG},
      {rows(4, 100, 104, RP_LOGITS_F16, 0), RP_ERR_INVALID_ARG},
  };
  g_launches = 0;
  for (const Case& c : cases) {
    size_t bytes = 0;
    EXPECT(rp_logits_workspace_size(&c.l, &bytes) == c.want && !g_error.empty());
    EXPECT(sample(c.l) == c.want && logprobs(c.l) == c.want);
    EXPECT(policy(c.l, batch()) == c.want && distill(c.l, teacher()) == c.want);
  }
  EXPECT(rp_logits_workspace_size(nullptr, nullptr) == RP_ERR_INVALID_ARG);
  EXPECT(g_launches == 0);
}

void refusals_of_what_goes_with_rows() {
  const rp_logits l = rows();
  const double nan = std::nan(""), inf = std::numeric_limits<double>::infinity();
  g_launches = 0;
  for (double t : {0.0, -1.0, nan, inf, 1e-320, std::numeric_limits<double>::denorm_min()}) {
    rp_policy_batch b = batch();
    b.temperature = t;
    rp_teacher d = teacher();
    d.temperature = t;
    EXPECT(logprobs(l, t) == RP_ERR_INVALID_ARG && policy(l, b) == RP_ERR_INVALID_ARG &&
           distill(l, d) == RP_ERR_INVALID_ARG);
  }
  const auto refused = [&](auto&& change) {
    rp_policy_batch b = batch();
    change(b);
    return policy(l, b) == RP_ERR_INVALID_ARG && !g_error.empty();
  };
  EXPECT(refused([&](rp_policy_batch& b) { b.tokens = nullptr; }));
  EXPECT(refused([&](rp_policy_batch& b) { b.clip_low = nan; }));
  EXPECT(refused([&](rp_policy_batch& b) { b.kl_beta = inf; }));
  EXPECT(refused([&](rp_policy_batch& b) { b.num_advantages = INT32_MIN; }));
  EXPECT(refused([&](rp_policy_batch& b) { b.row_seq = nullptr; }));
  EXPECT(refused([&](rp_policy_batch& b) { b.ref_logprobs = nullptr; }));
  rp_teacher d = teacher();
  d.k = INT32_MAX;
  EXPECT(distill(l, d) == RP_ERR_UNSUPPORTED);
  d.k = INT32_MIN;
  EXPECT(distill(l, d) == RP_ERR_INVALID_ARG);
  d = teacher();
  d.kind = static_cast<rp_distill_kind>(7);
  EXPECT(distill(l, d) == RP_ERR_UNSUPPORTED);
  g_need = 1 << 20;
  EXPECT(rp_sample_tokens(&l, nullptr, F, I, F, F, nullptr, g_need, nullptr) == RP_ERR_WORKSPACE);
  EXPECT(rp_sample_tokens(&l, nullptr, F, I, F, F, at(4096), g_need - 1, nullptr) == RP_ERR_WORKSPACE);
  EXPECT(rp_sample_tokens(&l, nullptr, F, I, F, F, at(4100), g_need, nullptr) == RP_ERR_INVALID_ARG);
  g_need = 0;
  EXPECT(g_launches == 0);
}

// A gradient that overlaps the logits without being them, at every size that is accepted.
void overlaps() {
  const int32_t most = INT32_MAX;
  const int64_t far = INT32_MAX;
  struct Case { rp_logits l; uint64_t grad; int64_t stride; bool fine; };
  const Case cases[] = {
      {rows(), kRows, 104, true},
      {rows(), kRows, 105, false},
      {rows(1), kRows, 105, true},
      {rows(), kRows + 2, 104, false},
      {rows(), kRows - 2, 104, false},
      {rows(), kRows + (3 * 104 + 100) * 2 - 2, 104, false},
      {rows(), kRows + (3 * 104 + 100) * 2, 104, true},
      {rows(), kRows - (3 * 200 + 100) * 2 + 2, 200, false},
      {rows(), kRows - (3 * 200 + 100) * 2, 200, true},
      // Spans of nearly 2^64 bytes, and ends behind the last address.
      {rows(most, 1 << 20, far, RP_LOGITS_F32), kRows + 4096, far, false},
      {rows(most, 1 << 20, far, RP_LOGITS_F32), kRows - 4096, far, false},
      {rows(most, 1 << 20, far, RP_LOGITS_F32), kRows - 4096, 1 << 20, false},
      {rows(most, 1 << 20, far, RP_LOGITS_BF16), kRows + (uint64_t(1) << 62), far, false},
      {rows(most, 1 << 20, 1 << 20, RP_LOGITS_BF16, 0xFFFFFFFFFFFF0000), 0xFFFFFFFFFFFF0100, 1 << 20, false},
      {rows(most, 1 << 20, 1 << 20, RP_LOGITS_BF16, 0xFFFFFFFFFFFF0000), 0xFFFFFFFFFFFE0000, 1 << 20, false},
      {rows(most, 100, 100, RP_LOGITS_BF16), kRows + (uint64_t(1) << 40), 100, true},
  };
  for (const Case& c : cases) {
    g_launches = 0;
    const rp_status want = c.fine ? RP_OK : RP_ERR_INVALID_ARG;
    EXPECT(policy(c.l, batch(), c.grad, c.stride) == want);
    EXPECT(distill(c.l, teacher(), c.grad, c.stride) == want);
    EXPECT(g_launches == (c.fine ? 2 : 0));
  }
}

}  // namespace

int main() {
  every_call_reaches_its_launch();
  refusals_of_rows();
  refusals_of_what_goes_with_rows();
  overlaps();
  if (g_fail) {
    std::fprintf(stderr, "%d expectation(s) failed\n", g_fail);
    return 1;
  }
  std::printf("sanitize_rows: all expectations held\n");
  return 0;
}
