// C-ABI entry points over rows of logits: argument checks and launches.
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "rp.h"
#include "rp_internal.h"

namespace {

rp_status fail(rp_status st, const char* fmt, ...) {
  char text[256];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(text, sizeof(text), fmt, ap);
  va_end(ap);
  return rp::set_error(st, text);
}

rp_status done(hipError_t e, const char* what) {
  return e == hipSuccess ? RP_OK : fail(RP_ERR_HIP, "%s kernel launch: %s (%d)", what, hipGetErrorString(e), (int)e);
}

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// A NULL or misaligned array of 4-byte entries.
bool bad(const void* p) { return p == nullptr || !aligned(p, 4); }
bool bad_if_there(const void* p) { return !aligned(p, 4); }

struct Rows {
  rp::LogitArgs args;
  int dtype, bytes;
};

rp_status check_rows(const rp_logits* l, Rows* r) {
  if (l == nullptr) return fail(RP_ERR_INVALID_ARG, "logits is NULL");
  r->dtype = rp::enum_bits(l->dtype);
  if (r->dtype != RP_LOGITS_BF16 && r->dtype != RP_LOGITS_F16 && r->dtype != RP_LOGITS_F32)
    return fail(RP_ERR_UNSUPPORTED, "logits dtype %d unsupported", r->dtype);
  r->bytes = r->dtype == RP_LOGITS_F32 ? 4 : 2;
  if (l->num_rows < 0) return fail(RP_ERR_INVALID_ARG, "num_rows must be >= 0");
  if (l->vocab < 1) return fail(RP_ERR_INVALID_ARG, "vocab must be >= 1");
  if (l->vocab > rp::kMaxVocab)
    return fail(RP_ERR_UNSUPPORTED, "vocab %d above the limit %d", l->vocab, rp::kMaxVocab);
  if (l->row_stride < l->vocab || l->row_stride >= (1ll << 31))
    return fail(RP_ERR_INVALID_ARG, "row_stride %lld must be in [vocab, 2^31)", (long long)l->row_stride);
  if (l->num_rows > 0 && (l->data == nullptr || !aligned(l->data, r->bytes)))
    return fail(RP_ERR_INVALID_ARG, "logits data must be non-NULL and aligned to its elements");
  r->args = {l->data, l->num_rows, l->vocab, l->row_stride, 0};
  return RP_OK;
}

rp_status check_temperature(double t) {
  if (!(t > 0.0) || !std::isfinite(t) || !std::isfinite(1.0 / t) || !std::isfinite((float)(rp::kLog2e64 / t)))
    return fail(RP_ERR_INVALID_ARG, "temperature must be finite and > 0");
  return RP_OK;
}

// dlogits may be the logits themselves; other overlaps are refused.
rp_status check_gradient(const Rows& r, void* dlogits, int64_t stride) {
  if (dlogits == nullptr) return RP_OK;
  if (!aligned(dlogits, r.bytes)) return fail(RP_ERR_INVALID_ARG, "dlogits must be aligned to its elements");
  if (stride < r.args.vocab || stride >= (1ll << 31))
    return fail(RP_ERR_INVALID_ARG, "dlogits_stride %lld must be in [vocab, 2^31)", (long long)stride);
  if (dlogits == r.args.data) {
    if (stride != r.args.stride && r.args.rows > 1)
      return fail(RP_ERR_INVALID_ARG, "dlogits in the logits' place needs their stride");
    return RP_OK;
  }
  // Below 2^64 bytes at the largest sizes accepted; the end of either might pass the last address.
  const auto span = [&](int64_t s) {
    return ((uint64_t)(r.args.rows - 1) * (uint64_t)s + (uint64_t)r.args.vocab) * (uint64_t)r.bytes;
  };
  const uint64_t x = reinterpret_cast<uintptr_t>(r.args.data), g = reinterpret_cast<uintptr_t>(dlogits);
  if (g > x ? g - x < span(r.args.stride) : x - g < span(stride))
    return fail(RP_ERR_INVALID_ARG, "dlogits overlaps the logits without being them");
  return RP_OK;
}

rp_status check_workspace(size_t need, const void* workspace, size_t bytes) {
  if (need == 0) return RP_OK;
  if (workspace == nullptr || bytes < need)
    return fail(RP_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", workspace == nullptr ? 0 : bytes, need);
  if (!aligned(workspace, 256)) return fail(RP_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
  return RP_OK;
}

size_t workspace_need(const Rows& r) { return rp::sample_workspace(r.args.rows, r.args.vocab, r.dtype); }

}  // namespace

extern "C" {

rp_status rp_logits_workspace_size(const rp_logits* logits, size_t* bytes) {
  rp::clear_error();
  if (bytes == nullptr) return fail(RP_ERR_INVALID_ARG, "bytes is NULL");
  Rows r;
  const rp_status st = check_rows(logits, &r);
  if (st != RP_OK) return st;
  *bytes = workspace_need(r);
  return RP_OK;
}

rp_status rp_sample_tokens(const rp_logits* logits, const rp_sampling* sampling, const float* u, int32_t* tokens,
                           float* logprobs, float* kept_logprobs, void* workspace, size_t workspace_bytes,
                           hipStream_t stream) {
  rp::clear_error();
  Rows r;
  rp_status st = check_rows(logits, &r);
  if (st != RP_OK || r.args.rows == 0) return st;
  if (bad(u) || bad(tokens)) return fail(RP_ERR_INVALID_ARG, "u/tokens must be non-NULL and 4-byte aligned");
  if (bad_if_there(logprobs) || bad_if_there(kept_logprobs))
    return fail(RP_ERR_INVALID_ARG, "logprobs/kept_logprobs must be 4-byte aligned");
  rp::SampleArgs a{r.args, nullptr, nullptr, nullptr, nullptr, u, tokens, logprobs, kept_logprobs, workspace};
  if (sampling != nullptr) {
    a.temperature = sampling->temperature;
    a.top_k = sampling->top_k;
    a.top_p = sampling->top_p;
    a.min_p = sampling->min_p;
    if (bad_if_there(a.temperature) || bad_if_there(a.top_k) || bad_if_there(a.top_p) || bad_if_there(a.min_p))
      return fail(RP_ERR_INVALID_ARG, "temperature/top_k/top_p/min_p must be 4-byte aligned");
  }
  st = check_workspace(workspace_need(r), workspace, workspace_bytes);
  if (st == RP_OK) st = rp::device_cus(&r.args.num_cus);
  a.logits = r.args;
  return st == RP_OK ? done(rp::launch_sample(a, r.dtype, stream), "sampling") : st;
}

rp_status rp_token_logprobs(const rp_logits* logits, const int32_t* tokens, double temperature, float* logprobs,
                            float* entropy, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  rp::clear_error();
  Rows r;
  rp_status st = check_rows(logits, &r);
  if (st == RP_OK) st = check_temperature(temperature);
  if (st != RP_OK || r.args.rows == 0) return st;
  if (bad(tokens) || bad(logprobs) || bad_if_there(entropy))
    return fail(RP_ERR_INVALID_ARG, "tokens/logprobs must be non-NULL, and with entropy 4-byte aligned");
  st = check_workspace(workspace_need(r), workspace, workspace_bytes);
  if (st == RP_OK) st = rp::device_cus(&r.args.num_cus);
  const rp::LogprobArgs a{r.args, tokens, 1.0 / temperature, logprobs, entropy};
  return st == RP_OK ? done(rp::launch_logprobs(a, r.dtype, stream), "log-probabilities") : st;
}

rp_status rp_policy_loss(const rp_logits* logits, const rp_policy_batch* b, float* losses, float* logprobs,
                         float* entropy, void* dlogits, int64_t dlogits_stride, void* workspace,
                         size_t workspace_bytes, hipStream_t stream) {
  rp::clear_error();
  Rows r;
  rp_status st = check_rows(logits, &r);
  if (st != RP_OK) return st;
  if (b == nullptr) return fail(RP_ERR_INVALID_ARG, "batch is NULL");
  st = check_temperature(b->temperature);
  if (st != RP_OK) return st;
  if (!(b->clip_low >= 0.0) || !(b->clip_high >= 0.0))
    return fail(RP_ERR_INVALID_ARG, "clip_low and clip_high must be >= 0");
  if (!std::isfinite(b->kl_beta) || !std::isfinite(b->entropy_coef))
    return fail(RP_ERR_INVALID_ARG, "kl_beta and entropy_coef must be finite");
  if (b->num_advantages < 0 || (b->row_seq == nullptr && b->num_advantages < r.args.rows))
    return fail(RP_ERR_INVALID_ARG, "num_advantages %d for %d rows without row_seq", b->num_advantages, r.args.rows);
  if (r.args.rows == 0) return RP_OK;
  if (bad(b->tokens) || bad(b->old_logprobs) || (b->num_advantages > 0 && b->advantages == nullptr) || bad(losses))
    return fail(RP_ERR_INVALID_ARG, "tokens/old_logprobs/advantages/losses must be non-NULL and 4-byte aligned");
  if (b->kl_beta != 0.0 && b->ref_logprobs == nullptr)
    return fail(RP_ERR_INVALID_ARG, "kl_beta needs ref_logprobs");
  if (bad_if_there(b->ref_logprobs) || bad_if_there(b->advantages) || bad_if_there(b->row_seq) ||
      bad_if_there(b->weights) || bad_if_there(logprobs) || bad_if_there(entropy))
    return fail(RP_ERR_INVALID_ARG, "ref_logprobs/advantages/row_seq/weights/logprobs/entropy must be 4-byte aligned");
  st = check_gradient(r, dlogits, dlogits_stride);
  if (st == RP_OK) st = check_workspace(workspace_need(r), workspace, workspace_bytes);
  if (st == RP_OK) st = rp::device_cus(&r.args.num_cus);
  if (st != RP_OK) return st;
  const rp::PolicyArgs a{r.args, b->tokens, b->old_logprobs, b->kl_beta != 0.0 ? b->ref_logprobs : nullptr,
                         b->advantages, b->row_seq, b->num_advantages, b->weights, 1.0 / b->temperature, b->clip_low,
                         b->clip_high, b->kl_beta, b->entropy_coef, losses, logprobs, entropy, dlogits,
                         dlogits_stride};
  return done(rp::launch_policy(a, r.dtype, stream), "policy loss");
}

rp_status rp_distill_loss(const rp_logits* logits, const rp_teacher* t, float* losses, void* dlogits,
                          int64_t dlogits_stride, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  rp::clear_error();
  Rows r;
  rp_status st = check_rows(logits, &r);
  if (st != RP_OK) return st;
  if (t == nullptr) return fail(RP_ERR_INVALID_ARG, "teacher is NULL");
  st = check_temperature(t->temperature);
  if (st != RP_OK) return st;
  if (t->k < 1) return fail(RP_ERR_INVALID_ARG, "k must be >= 1");
  if (t->k > rp::kMaxListed) return fail(RP_ERR_UNSUPPORTED, "k %d above the limit %d", t->k, rp::kMaxListed);
  const int kind = rp::enum_bits(t->kind);
  if (kind != RP_DISTILL_TOPK && kind != RP_DISTILL_TAIL && kind != RP_DISTILL_REVERSE)
    return fail(RP_ERR_UNSUPPORTED, "kind %d unsupported", kind);
  if (r.args.rows == 0) return RP_OK;
  if (bad(t->ids) || bad(t->values) || bad(losses) || bad_if_there(t->weights))
    return fail(RP_ERR_INVALID_ARG, "ids/values/losses must be non-NULL, and with weights 4-byte aligned");
  st = check_gradient(r, dlogits, dlogits_stride);
  if (st == RP_OK) st = check_workspace(workspace_need(r), workspace, workspace_bytes);
  if (st == RP_OK) st = rp::device_cus(&r.args.num_cus);
  if (st != RP_OK) return st;
  const rp::DistillArgs a{r.args, t->ids, t->values, t->k, kind, t->weights, 1.0 / t->temperature, losses,
                          dlogits, dlogits_stride};
  return done(rp::launch_distill(a, r.dtype, stream), "distillation loss");
}

}  // extern "C"
