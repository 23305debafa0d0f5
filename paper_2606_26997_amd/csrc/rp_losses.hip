// Log-probabilities, the policy loss and distillation over rows of logits:
// one workgroup per row.
//
// With m = max x and c = log2(e) / T, e_i = 2^((x_i - m) c), S = sum e_i and
// p_i = e_i / S, so ln p_i = (x_i - m) / T - ln S and
//   H = ln S - ln 2 sum e_i d_i / S,  d_i = (x_i - m) c.
// A first pass over the row keeps a running m, S and sum e d per thread; what
// is one number per row is then computed in 64 bits; a second pass writes the
// gradient, which is e_i (alpha + beta d_i) but for the row's token, or the
// ids of the teacher's list, which are written behind a barrier.
#include "rp_rows.h"

namespace rp {
namespace {

constexpr int kThreads = 1024;

struct Stats {
  float m, s, t;  // largest logit, sum e, sum e d
};

// Twice the finite range below any d: keeps e d a product of numbers where d is -inf (e = 0).
constexpr float kLeast = -1e30f;

template <int N>
__device__ inline void add_values(Stats& a, const float (&x)[N], float c) {
  float top = a.m;
#pragma unroll
  for (int k = 0; k < N; ++k) top = fmaxf(top, x[k]);
  if (top > a.m) {
    if (a.s > 0.f) {
      const float shift = (a.m - top) * c, f = fast_exp2(shift);
      a.t = f * (a.t + shift * a.s);
      a.s *= f;
    }
    a.m = top;
  }
  const float base = a.m == -INFINITY ? 0.f : a.m;
  float s = 0.f, t = 0.f;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const float d = (x[k] - base) * c, e = fast_exp2(d);
    s += e;
    t += e * fmaxf(d, kLeast);
  }
  a.s += s;
  a.t += t;
}

// The row's m (0 for a row without a finite logit), S and sum e d in 64 bits,
// the same in every thread.
struct RowStats {
  float m;
  double s, t;
};
template <int NT>
__device__ inline RowStats join(const Stats& a, float c, float* lds_f, double* lds_d) {
  const float m = block_max<NT>(a.m, lds_f);
  const float base = m == -INFINITY ? 0.f : m;
  double s = (double)a.s, t = (double)a.t;
  if (a.m > -INFINITY) {
    const float shift = (a.m - base) * c, f = fast_exp2(shift);
    t = (double)f * (t + (double)fmaxf(shift, kLeast) * s);
    s *= (double)f;
  }
  RowStats r;
  r.m = base;
  r.s = block_sum<NT>(s, lds_d);
  r.t = block_sum<NT>(t, lds_d);
  return r;
}

template <int DT, int NT>
__device__ inline Stats row_stats(const void* row, int vocab, float c) {
  Stats a = {-INFINITY, 0.f, 0.f};
  for (int v = threadIdx.x; v * Elem<DT>::kPerVec < vocab; v += NT) {
    float x[Elem<DT>::kPerVec];
    unpack<DT>(load_vec<DT>(row, v, vocab), x);
    add_values(a, x, c);
  }
  return a;
}

// dlogits = e (alpha + beta d), zero where every logit is -inf.
template <int DT, int NT>
__device__ inline void write_gradient(const void* row, void* out, int vocab, float m, float c, float alpha, float beta) {
  for (int v = threadIdx.x; v * Elem<DT>::kPerVec < vocab; v += NT) {
    float x[Elem<DT>::kPerVec];
    unpack<DT>(load_vec<DT>(row, v, vocab), x);
#pragma unroll
    for (int k = 0; k < Elem<DT>::kPerVec; ++k) {
      const float d = (x[k] - m) * c;
      x[k] = fast_exp2(d) * (alpha + beta * fmaxf(d, kLeast));
    }
    store_vec<DT>(out, v, vocab, x);
  }
}
template <int DT, int NT>
__device__ inline void write_zeros(void* out, int vocab) {
  const float zero[Elem<DT>::kPerVec] = {};
  for (int v = threadIdx.x; v * Elem<DT>::kPerVec < vocab; v += NT) store_vec<DT>(out, v, vocab, zero);
}

template <int DT>
__device__ inline const void* row_of(const LogitArgs& l, int n) {
  return static_cast<const char*>(l.data) + (long long)n * l.stride * Elem<DT>::kBytes;
}
template <int DT>
__device__ inline void* grad_row(void* g, long long stride, int n) {
  return static_cast<char*>(g) + (long long)n * stride * Elem<DT>::kBytes;
}

struct Shared {
  float f[kThreads / 64];
  double d[kThreads / 64];
};

template <int DT>
__global__ __launch_bounds__(kThreads) void logprobs_kernel(const LogprobArgs a) {
  __shared__ Shared lds;
  const int n = blockIdx.x, V = a.logits.vocab;
  const void* row = row_of<DT>(a.logits, n);
  const int y = a.tokens[n];
  if ((unsigned)y >= (unsigned)V) {
    if (threadIdx.x == 0) {
      a.logprobs[n] = 0.f;
      if (a.entropy != nullptr) a.entropy[n] = 0.f;
    }
    return;
  }
  const float c = (float)(a.inv_t * kLog2e64);
  const RowStats r = join<kThreads>(row_stats<DT, kThreads>(row, V, c), c, lds.f, lds.d);
  if (threadIdx.x == 0) {
    const bool empty = r.s == 0.0;
    const double ln_s = log(r.s);
    a.logprobs[n] = empty ? -INFINITY : (float)(((double)Elem<DT>::get(row, y) - (double)r.m) * a.inv_t - ln_s);
    if (a.entropy != nullptr) a.entropy[n] = empty ? 0.f : (float)(ln_s - kLn2_64 * r.t / r.s);
  }
}

template <int DT>
__global__ __launch_bounds__(kThreads) void policy_kernel(const PolicyArgs a) {
  __shared__ Shared lds;
  __shared__ float factors[2];
  const int n = blockIdx.x, V = a.logits.vocab;
  const void* row = row_of<DT>(a.logits, n);
  void* out = a.dlogits != nullptr ? grad_row<DT>(a.dlogits, a.dstride, n) : nullptr;
  const int y = a.tokens[n];
  const int seq = a.row_seq != nullptr ? a.row_seq[n] : n;
  if ((unsigned)y >= (unsigned)V || (unsigned)seq >= (unsigned)a.num_advantages) {
    if (threadIdx.x == 0) {
      a.losses[n] = 0.f;
      if (a.logprobs != nullptr) a.logprobs[n] = 0.f;
      if (a.entropy != nullptr) a.entropy[n] = 0.f;
    }
    if (out != nullptr) write_zeros<DT, kThreads>(out, V);
    return;
  }
  const float c = (float)(a.inv_t * kLog2e64);
  const RowStats r = join<kThreads>(row_stats<DT, kThreads>(row, V, c), c, lds.f, lds.d);
  float at_token = 0.f;
  const bool empty = r.s == 0.0;
  const double w = a.weights != nullptr ? (double)a.weights[n] : 1.0;
  if (threadIdx.x == 0) {
    const double ln_s = log(r.s);
    const double z = ((double)Elem<DT>::get(row, y) - (double)r.m) * a.inv_t;
    const double lp = empty ? -INFINITY : z - ln_s;
    const double H = empty ? 0.0 : ln_s - kLn2_64 * r.t / r.s;
    const double A = (double)a.advantages[seq];
    const double ratio = exp(lp - (double)a.old_logprobs[n]);
    const double free_s = ratio * A, held = fmin(fmax(ratio, 1.0 - a.clip_low), 1.0 + a.clip_high) * A;
    // Written so that a NaN on either side stays one.
    const bool is_free = !(held < free_s);
    double loss = -(is_free ? free_s : held) - a.entropy_coef * H, g = is_free ? -free_s : 0.0;
    if (a.ref_logprobs != nullptr) {
      const double gap = (double)a.ref_logprobs[n] - lp, e = exp(gap);
      loss += a.kl_beta * (e - gap - 1.0);
      g += a.kl_beta * (1.0 - e);
    }
    const bool none = empty || w == 0.0;
    a.losses[n] = none ? 0.f : (float)(w * loss);
    if (a.logprobs != nullptr) a.logprobs[n] = (float)lp;
    if (a.entropy != nullptr) a.entropy[n] = (float)H;
    // d loss / d x_i = w / T (g ([i = y] - p_i) + b p_i (ln p_i + H)), ln p_i = d_i ln 2 - ln S.
    const double per = w * a.inv_t, b = a.entropy_coef, p = exp(lp);
    factors[0] = (float)(per * (b * (H - ln_s) - g) / r.s);
    factors[1] = (float)(per * b * kLn2_64 / r.s);
    at_token = (float)(per * (g * (1.0 - p) + (b != 0.0 && p > 0.0 ? b * p * (lp + H) : 0.0)));
  }
  if (out == nullptr) return;
  if (empty || w == 0.0) {
    write_zeros<DT, kThreads>(out, V);
    return;
  }
  __syncthreads();
  write_gradient<DT, kThreads>(row, out, V, r.m, c, factors[0], factors[1]);
  __syncthreads();
  if (threadIdx.x == 0) put_elem<DT>(out, y, at_token);
}

// The row's list in LDS: entry j < k counts where its id is in the vocabulary,
// is not listed before it and its value is above -inf.
struct List {
  int id[kMaxListed];
  float x[kMaxListed], value[kMaxListed];
  double grad[kMaxListed];
};

template <int DT>
__global__ __launch_bounds__(kThreads) void distill_kernel(const DistillArgs a) {
  __shared__ Shared lds;
  __shared__ List list;
  extern __shared__ uint32_t listed[];  // a bit per token of the vocabulary
  const int n = blockIdx.x, V = a.logits.vocab, K = a.k, tid = threadIdx.x;
  const void* row = row_of<DT>(a.logits, n);
  void* out = a.dlogits != nullptr ? grad_row<DT>(a.dlogits, a.dstride, n) : nullptr;
  const double w = a.weights != nullptr ? (double)a.weights[n] : 1.0;
  if (w == 0.0) {
    if (tid == 0) a.losses[n] = 0.f;
    if (out != nullptr) write_zeros<DT, kThreads>(out, V);
    return;
  }
  const float c = (float)(a.inv_t * kLog2e64);
  static_assert(kMaxListed <= kThreads, "an entry per thread");
  for (int i = tid; i < cdiv(V, 32); i += kThreads) listed[i] = 0;
  int id = -1;
  float value = -INFINITY;
  if (tid < K) {
    id = a.ids[(long long)n * K + tid];
    value = a.values[(long long)n * K + tid];
    if ((unsigned)id >= (unsigned)V || value == -INFINITY) id = -1;
    list.id[tid] = id;
  }
  __syncthreads();
  if (id >= 0) {
    for (int j = 0; j < tid; ++j)
      if (list.id[j] == id) id = -1;
  }
  const bool counts = id >= 0;
  if (counts) atomicOr(&listed[id / 32], 1u << (id % 32));
  const float x_id = counts ? Elem<DT>::get(row, id) : -INFINITY;
  __syncthreads();
  // Sums over the tokens outside the list; those of the list are added apart,
  // so that a small mass outside is no difference of large ones.
  Stats st = {-INFINITY, 0.f, 0.f};
  for (int v = tid; v * Elem<DT>::kPerVec < V; v += kThreads) {
    constexpr int E = Elem<DT>::kPerVec;
    float x[E];
    unpack<DT>(load_vec<DT>(row, v, V), x);
    const uint32_t hit = listed[v * E / 32] >> (v * E % 32) & ((1u << E) - 1);
#pragma unroll
    for (int k = 0; k < E; ++k)
      if (hit >> k & 1) x[k] = -INFINITY;
    add_values(st, x, c);
  }
  const float m = fmaxf(block_max<kThreads>(st.m, lds.f), block_max<kThreads>(x_id, lds.f));
  const bool finite = m > -INFINITY;
  const float base = finite ? m : 0.f;
  const double so = block_sum<kThreads>(
      st.m > -INFINITY ? (double)st.s * (double)fast_exp2((st.m - base) * c) : (double)st.s, lds.d);
  const double zi = counts ? ((double)x_id - (double)base) * a.inv_t : -INFINITY, ei = counts ? exp(zi) : 0.0;
  const double s = so + block_sum<kThreads>(ei, lds.d);
  const bool empty = s == 0.0;
  const double ln_s = log(s), lq = zi - ln_s, q = ei / s;
  const double s1 = counts ? 1.0 : 0.0;
  double others = 1.0, mine = 0.0, loss;
  if (a.kind == RP_DISTILL_TOPK) {
    const double t = counts ? (double)value * a.inv_t : -INFINITY;
    const float tm = block_max<kThreads>(counts ? value : -INFINITY, lds.f);
    const double ts = counts ? t - (double)tm * a.inv_t : -INFINITY;
    const double total = block_sum<kThreads>(counts ? exp(ts) : 0.0, lds.d);
    const double lp = ts - log(total), P = counts ? exp(lp) : 0.0;
    loss = block_sum<kThreads>(P > 0.0 ? P * (lp - lq) : 0.0, lds.d);
    mine = q - P;
    if (total == 0.0) others = 0.0;  // an empty list teaches nothing
  } else {
    const double lp = (double)value, P = counts ? exp(lp) : 0.0;
    const double sum = block_sum<kThreads>(P, lds.d), rest = fmax(1.0 - sum, 0x1p-24), qo = so / s;
    const bool outside = !(qo == 0.0);  // a NaN stays
    const double gap = log(qo) - log(rest);
    if (a.kind == RP_DISTILL_TAIL) {
      loss = block_sum<kThreads>(P > 0.0 ? P * (lp - lq) : 0.0, lds.d) - (outside ? rest * gap : 0.0);
      const double whole = sum + (outside ? rest : 0.0);
      others = outside ? whole - rest / qo : 0.0;
      mine = whole * q - P;
    } else {
      loss = block_sum<kThreads>(counts && !(q == 0.0) ? q * (lq - lp) : 0.0, lds.d) + (outside ? qo * gap : 0.0);
      others = outside ? gap - loss : 0.0;
      mine = counts && !(q == 0.0) ? q * (lq - lp - loss) : 0.0;
    }
  }
  (void)s1;
  if (tid == 0) a.losses[n] = empty ? 0.f : (float)(w * loss);
  if (out == nullptr) return;
  if (empty) {
    write_zeros<DT, kThreads>(out, V);
    return;
  }
  const double per = w * a.inv_t;
  write_gradient<DT, kThreads>(row, out, V, base, c, (float)(per * others / s), 0.f);
  __syncthreads();
  if (counts) put_elem<DT>(out, id, (float)(per * mine));
}

}  // namespace

#define RP_BY_DTYPE(call)                       \
  switch (dtype) {                              \
    case RP_LOGITS_BF16: call(RP_LOGITS_BF16); break; \
    case RP_LOGITS_F16: call(RP_LOGITS_F16); break;   \
    default: call(RP_LOGITS_F32); break;        \
  }

hipError_t launch_logprobs(const LogprobArgs& a, int dtype, hipStream_t stream) {
#define CALL(DT) logprobs_kernel<DT><<<dim3(a.logits.rows), dim3(kThreads), 0, stream>>>(a)
  RP_BY_DTYPE(CALL)
#undef CALL
  return hipGetLastError();
}

hipError_t launch_policy(const PolicyArgs& a, int dtype, hipStream_t stream) {
#define CALL(DT) policy_kernel<DT><<<dim3(a.logits.rows), dim3(kThreads), 0, stream>>>(a)
  RP_BY_DTYPE(CALL)
#undef CALL
  return hipGetLastError();
}

hipError_t launch_distill(const DistillArgs& a, int dtype, hipStream_t stream) {
  const size_t bits = (size_t)cdiv(a.logits.vocab, 32) * 4;
#define CALL(DT) distill_kernel<DT><<<dim3(a.logits.rows), dim3(kThreads), bits, stream>>>(a)
  RP_BY_DTYPE(CALL)
#undef CALL
  return hipGetLastError();
}

}  // namespace rp
