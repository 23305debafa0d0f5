// Log-probabilities, the policy loss and distillation over rows of logits.
//
// With m = max x and c = log2(e) / T, d_i = (x_i - m) c, e_i = 2^d_i, S = sum e_i
// and p_i = e_i / S: ln p_i = d_i ln 2 - ln S, and
//   H = ln S - ln 2 sum e_i d_i / S.
// One pass over a row keeps a running m, S and sum e d per thread; what is one
// number per row is computed in 64 bits; the gradient is e_i (alpha + beta d_i)
// but for the row's token, or the ids of the teacher's list.
//
// A team of W waves has a row. The first NV vectors of 16 bytes of every thread
// stay in registers between the sums and the gradient; the others are read again,
// from the caches.
#include "rp_rows.h"

namespace rp {
namespace {

// Below any finite d, so that e d is a product of numbers where d is -inf (e = 0).
constexpr float kLeast = -1e30f;
// References r and maxima times c stay below this in magnitude, or the row is
// summed again without products that overflow (row_sums).
constexpr float kMostRef = 1e36f;

// log2(e) / T in fp32, above 0 however large T is: c times -inf has to be -inf.
__device__ inline float scale_of(double inv_t) { return fmaxf((float)(inv_t * kLog2e64), 0x1p-149f); }

// d = (x - max) c. Where c is below 1 by half the difference, which is as exact and does
// not pass fp32's range: at T = 1e38 logits of 3e38 and -3e38 both count.
struct Below {
  float half, half_max, c;
  __device__ inline Below(float max, float scale)
      : half(scale < 1.f ? 0.5f : 1.f), half_max(max * half), c(scale < 1.f ? scale * 2.f : scale) {}
  __device__ inline float operator()(float x) const { return fmaf(x, half, -half_max) * c; }
};

// A thread's sums relative to 2^r: of e and e d over the vector with its largest
// logit (group, group_t) and over all others (rest, rest_t). They are apart so
// that the one vector can be summed again in 64 bits (join): in a row in which
// one token has nearly all the mass, what matters is the rest, and fp32 sums
// with the largest term would lose it. r moves only when a term would pass 2^8.
struct Stats {
  float r = -kMostRef, top = -3.402823466e38f;
  float rest = 0.f, rest_t = 0.f, group = 0.f, group_t = 0.f;
  int at = -1;
};

// The vector units' work counts beside the read: an exponential a logit takes a wave 8
// cycles, its other instructions 2 each. With a reference that moved with every maximum,
// and so differences x - m, log-probabilities of 8192 rows of 151936 bf16 logits took
// 470 us; 437 this way (12 instructions a logit).
template <int E>
__device__ inline void add_values(Stats& a, int v, const float (&x)[E], float c) {
  float top = x[0];
#pragma unroll
  for (int k = 1; k < E; ++k) top = fmaxf(top, x[k]);
  if (fmaf(top, c, -a.r) > kLazyMax) {
    const float r = fminf(fmaxf(top * c, -kMostRef), kMostRef);
    const float shift = a.r - r, f = fast_exp2(shift);
    a.rest_t = f * (a.rest_t + shift * a.rest);
    a.group_t = f * (a.group_t + shift * a.group);
    a.rest *= f;
    a.group *= f;
    a.r = r;
  }
  const bool more = top > a.top;
  a.top = fmaxf(a.top, top);
  a.at = more ? v : a.at;
  float s = 0.f, t = 0.f;
#pragma unroll
  for (int k = 0; k < E; ++k) {
    const float d = fmaf(x[k], c, -a.r), e = fast_exp2(d);
    s += e;
    t = fmaf(e, fmaxf(d, kLeast), t);
  }
  a.rest += more ? a.group : s;
  a.rest_t += more ? a.group_t : t;
  a.group = more ? s : a.group;
  a.group_t = more ? t : a.group_t;
}

// A thread's sums (of e, of e d) relative to the row's maximum. reload(v, x) gives
// the vector v again.
template <int E, class Reload>
__device__ inline void join(const Stats& a, float max, float c, double& s, double& t, const Reload& reload) {
  const float shift = fmaxf(fmaf(-max, c, a.r), kLeast);
  const double f = (double)fast_exp2(shift);
  if (a.at < 0 || a.top < max) {
    s = f * (double)(a.rest + a.group);
    t = f * ((double)(a.rest_t + a.group_t) + (double)shift * (double)(a.rest + a.group));
    return;
  }
  s = f * (double)a.rest;
  t = f * ((double)a.rest_t + (double)shift * (double)a.rest);
  float x[E];
  reload(a.at, x);
  const Below below(max, c);
#pragma unroll
  for (int k = 0; k < E; ++k) {
    const float d = below(x[k]), e = fast_exp2(d);
    s += (double)e;
    t += (double)e * (double)fmaxf(d, kLeast);
  }
}

// Reductions over a team of W waves; every use of a slot is followed by a
// barrier before its next one.
template <int W>
struct Slots {
  float m[W][3];
  double d[W][5], far;
  float out[3];
};
template <int W, int N>
__device__ inline void team_max(float (&x)[N], Slots<W>& s) {
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = wave_max(x[i]);
  if constexpr (W == 1) return;
  if (threadIdx.x % 64 == 0) {
#pragma unroll
    for (int i = 0; i < N; ++i) s.m[threadIdx.x / 64][i] = x[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    x[i] = s.m[0][i];
#pragma unroll
    for (int w = 1; w < W; ++w) x[i] = fmaxf(x[i], s.m[w][i]);
  }
}
template <int W, int N>
__device__ inline void team_sum(double (&x)[N], Slots<W>& s) {
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = wave_sum(x[i]);
  if constexpr (W == 1) return;
  if (threadIdx.x % 64 == 0) {
#pragma unroll
    for (int i = 0; i < N; ++i) s.d[threadIdx.x / 64][i] = x[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    x[i] = s.d[0][i];
#pragma unroll
    for (int w = 1; w < W; ++w) x[i] += s.d[w][i];
  }
}

__device__ inline int wave_id() { return __builtin_amdgcn_readfirstlane(threadIdx.x / 64); }

template <int W>
constexpr int threads_of() {
  return W == 1 ? 256 : W * 64;  // four rows share a workgroup of single waves
}

// A row as its team walks it: vectors j * NT + thread from the row's first
// 16-byte boundary on, and the loose elements before it and behind the last whole
// vector, one per thread. Row pointers are the same for a whole wave, so that an
// access is a scalar base, one offset register and no more. (Vectors from the
// row's start, off the boundary: distillation of 1500 rows of 100003 fp16 logits
// 177 us, 155 this way.)
template <int DT, int W, int NV>
struct Row {
  static constexpr int E = Elem<DT>::kPerVec, NT = W * 64, kHeld = NV > 0 ? NV : 1;
  static constexpr int U = 4;  // vectors requested ahead of their use, and again as many in use
  int head, whole, loose, id;  // id: the thread in its team
  u32x4_any q[kHeld];
  float single = 0.f;

  __device__ inline Row(int vocab, const char* row) : id(threadIdx.x % NT) {
    head = min((int)(-reinterpret_cast<uintptr_t>(row) & 15) / Elem<DT>::kBytes, vocab);
    whole = (vocab - head) / E;
    loose = vocab - whole * E;
  }
  // The thread's loose token.
  __device__ inline int loose_of() const { return id < head ? id : whole * E + id; }
  // The thread that has a token.
  __device__ inline int owner_of(int token) const {
    const int v = token - head;
    return v < 0 ? token : v < whole * E ? v / E % NT : token - whole * E;
  }

  // Vector j of the thread; threads behind the last whole vector read that one. What
  // is read once (ONCE) goes past the caches (log-probabilities of 1024 rows of 151936
  // fp32 logits: 109 us, 98 this way).
  template <bool ONCE>
  __device__ inline u32x4_any load(const char* row, int j) const {
    const uint32_t at = min((uint32_t)id, (uint32_t)(whole - 1 - j * NT)) * 16u;
    const u32x4_any* from = reinterpret_cast<const u32x4_any*>(row + head * Elem<DT>::kBytes + (size_t)j * (NT * 16) + at);
    if constexpr (ONCE) return __builtin_nontemporal_load(from);
    else return *from;
  }
  __device__ inline void put(char* out, int j, const float (&x)[E]) const {
    u32x4_any* at =
        reinterpret_cast<u32x4_any*>(out + head * Elem<DT>::kBytes + (size_t)j * (NT * 16) + (uint32_t)id * 16u);
    // Past the caches (4096 rows of 32000 bf16 logits: 107 us, 102 this way).
    __builtin_nontemporal_store(pack<DT>(x), at);
  }
  __device__ inline void fetch_all(const char* row) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (j * NT < whole) q[j] = load<true>(row, j);
    if (id < loose) single = Elem<DT>::get(row, loose_of());
  }
  // f(vector, logits); the loose ones as a vector `whole` of one logit and -inf.
  template <bool ONCE, class F>
  __device__ inline void each(const char* row, const F& f) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if (j * NT < whole) visit(j, q[j], f);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (NV * NT < whole) {
      u32x4_any next[U];
#pragma unroll
      for (int i = 0; i < U; ++i)
        if ((NV + i) * NT < whole) next[i] = load<ONCE>(row, NV + i);
      for (int j0 = NV; j0 * NT < whole; j0 += U) {
        u32x4_any now[U];
#pragma unroll
        for (int i = 0; i < U; ++i) now[i] = next[i];
#pragma unroll
        for (int i = 0; i < U; ++i)
          if ((j0 + U + i) * NT < whole) next[i] = load<ONCE>(row, j0 + U + i);
#pragma unroll
        for (int i = 0; i < U; ++i) {
          if ((j0 + i) * NT < whole) visit(j0 + i, now[i], f);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
    if (loose > 0) {
      float x[E];
#pragma unroll
      for (int k = 0; k < E; ++k) x[k] = -INFINITY;
      x[0] = id < loose ? single : -INFINITY;
      f(whole, x);
    }
  }
  // Threads behind the last whole vector see -inf.
  template <class F>
  __device__ inline void visit(int j, u32x4_any bits, const F& f) const {
    const int v = j * NT + id;
    if ((j + 1) * NT > whole) {
      constexpr uint32_t none = DT == RP_LOGITS_BF16 ? 0xFF80FF80u : DT == RP_LOGITS_F16 ? 0xFC00FC00u : 0xFF800000u;
#pragma unroll
      for (int k = 0; k < 4; ++k) bits[k] = v < whole ? bits[k] : none;
    }
    float x[E];
    unpack<DT>(bits, x);
    f(v, x);
  }
  // The vector that each() called v (whole: the thread's loose logit).
  __device__ inline void again(const char* row, int v, float (&x)[E]) const {
    if (v < whole) {
      unpack<DT>(*reinterpret_cast<const u32x4_any*>(row + head * Elem<DT>::kBytes + (size_t)v * 16), x);
      return;
    }
#pragma unroll
    for (int k = 0; k < E; ++k) x[k] = -INFINITY;
    x[0] = single;
  }
  template <class F>
  __device__ inline void store(const char* row, char* out, const F& f) {
    each<true>(row, [&](int v, const float (&x)[E]) {
      float y[E];
#pragma unroll
      for (int k = 0; k < E; ++k) y[k] = f(x[k]);
      if (v < whole) put(out, v / NT, y);
    });
    if (id < loose) put_elem<DT>(out, loose_of(), f(single));
  }
  __device__ inline void zero(char* out) const {
    const float none[E] = {};
    for (int j = 0; j * NT + id < whole; ++j) put(out, j, none);
    if (id < loose) put_elem<DT>(out, loose_of(), 0.f);
  }
};

template <int DT>
__device__ inline const char* row_of(const LogitArgs& l, int n) {
  return static_cast<const char*>(l.data) + (long long)n * l.stride * Elem<DT>::kBytes;
}
template <int DT>
__device__ inline char* grad_row(void* g, long long stride, int n) {
  return static_cast<char*>(g) + (long long)n * stride * Elem<DT>::kBytes;
}

// The row's maximum, and its sums of e and e d in 64 bits, in every thread. masked(v, x)
// takes what is not summed, nor looked at for the maximum, out of vector v. tops[0]
// becomes the maximum (fp32's least number where nothing is summed), other entries
// their own maxima over the team. Rows whose logits times c come near fp32's end are
// summed by the other form, (x - max) c.
template <int W, bool ONCE, int N, class R, class Masked>
__device__ inline float row_sums(R& r, const char* row, float c, const Masked& masked, Slots<W>& slots, double (&sums)[2],
                                 float (&tops)[N]) {
  constexpr int E = R::E;
  Stats st;
  r.template each<ONCE>(row, [&](int v, const float (&x)[E]) {
    float y[E];
#pragma unroll
    for (int k = 0; k < E; ++k) y[k] = x[k];
    masked(v, y);
    add_values(st, v, y, c);
  });
  tops[0] = st.top;
  team_max<W>(tops, slots);
  const float m = tops[0];
  const auto reload = [&](int v, float (&x)[E]) {
    r.again(row, v, x);
    masked(v, x);
  };
  if (fabsf(m * c) < kMostRef) {
    join<E>(st, m, c, sums[0], sums[1], reload);
  } else {
    sums[0] = sums[1] = 0.0;
    const Below below(m, c);
    for (int v = r.id; v < r.whole + (r.id < r.loose ? R::NT : 0); v += R::NT) {
      float x[E];
      reload(v < r.whole ? v : r.whole, x);
      for (int k = 0; k < E; ++k) {
        const float d = below(x[k]), e = fast_exp2(d);
        sums[0] += (double)e;
        sums[1] += (double)e * (double)fmaxf(d, kLeast);
      }
      if (v >= r.whole) break;
    }
  }
  return m;
}

// Bound by the read, with the vector units at work for two thirds of the cycles (12
// instructions a logit, counted): 8192 rows of 151936 bf16 logits 425 us, 5.9 TB/s (a
// large read reaches 7.0); 16 rows of 32000 fp16 7 us, a launch and the chain of a
// few loads, reductions and the logarithm.
template <int DT, int W>
__global__ __launch_bounds__(threads_of<W>()) void logprobs_kernel(const LogprobArgs a) {
  __shared__ Slots<W> slots;
  const int n = W == 1 ? blockIdx.x * 4 + wave_id() : blockIdx.x, V = a.logits.vocab;
  if (n >= a.logits.rows) return;
  const char* row = row_of<DT>(a.logits, n);
  Row<DT, W, 0> r(V, row);
  const int y = a.tokens[n];
  if ((unsigned)y >= (unsigned)V) {
    if (r.id == 0) {
      a.logprobs[n] = 0.f;
      if (a.entropy != nullptr) a.entropy[n] = 0.f;
    }
    return;
  }
  const float c = scale_of(a.inv_t), at = Elem<DT>::get(row, y);
  r.fetch_all(row);
  double sums[2];
  float tops[1];
  const float m = row_sums<W, true>(r, row, c, [](int, float (&)[Elem<DT>::kPerVec]) {}, slots, sums, tops);
  team_sum<W>(sums, slots);
  if (r.id == 0) {
    const bool empty = sums[0] == 0.0;
    const double ln_s = log(sums[0]);
    a.logprobs[n] = empty ? -INFINITY : (float)(((double)at - (double)m) * a.inv_t - ln_s);
    if (a.entropy != nullptr) a.entropy[n] = empty ? 0.f : (float)(ln_s - kLn2_64 * sums[1] / sums[0]);
  }
}

// Without a gradient (GRAD false) nothing is held. Bound by the copy that logits and
// gradient are: 2048 rows of 151936 bf16 logits 252 us, 4.8 TB/s, 1000 rows of 50257
// fp32 79 us, 5.1 TB/s (a large copy: 5.1).
template <int DT, int W, int NV, bool GRAD>
__global__ __launch_bounds__(threads_of<W>()) void policy_kernel(const PolicyArgs a) {
  __shared__ Slots<W> slots;
  const int n = W == 1 ? blockIdx.x * 4 + wave_id() : blockIdx.x, V = a.logits.vocab;
  if (n >= a.logits.rows) return;
  const char* row = row_of<DT>(a.logits, n);
  Row<DT, W, NV> r(V, row);
  char* out = GRAD ? grad_row<DT>(a.dlogits, a.dstride, n) : nullptr;
  const int y = a.tokens[n], seq = a.row_seq != nullptr ? a.row_seq[n] : n;
  if ((unsigned)y >= (unsigned)V || (unsigned)seq >= (unsigned)a.num_advantages) {
    if (r.id == 0) {
      a.losses[n] = 0.f;
      if (a.logprobs != nullptr) a.logprobs[n] = 0.f;
      if (a.entropy != nullptr) a.entropy[n] = 0.f;
    }
    if constexpr (GRAD) r.zero(out);
    return;
  }
  r.fetch_all(row);
  const float c = scale_of(a.inv_t), at = Elem<DT>::get(row, y);
  double sums[2];
  float tops[1];
  const float m = row_sums<W, !GRAD>(r, row, c, [](int, float (&)[Elem<DT>::kPerVec]) {}, slots, sums, tops);
  team_sum<W>(sums, slots);
  const bool empty = sums[0] == 0.0;
  const double w = a.weights != nullptr ? (double)a.weights[n] : 1.0;
  const bool none = empty || w == 0.0;
  float alpha = 0.f, beta = 0.f, own = 0.f;
  if (r.id < 64) {
    // One wave; its first lanes take an exponential each.
    const double ln_s = log(sums[0]);
    const double lp = empty ? -INFINITY : ((double)at - (double)m) * a.inv_t - ln_s;
    const double H = empty ? 0.0 : ln_s - kLn2_64 * sums[1] / sums[0];
    const double A = (double)a.advantages[seq], gap = a.ref_logprobs != nullptr ? (double)a.ref_logprobs[n] - lp : 0.0;
    // A token that cannot occur has r = 0, whatever the old policy gave it; r stays finite,
    // so that an advantage of 0 leaves no surrogate (a NaN passes both).
    const double log_r = lp == -INFINITY ? lp : lp - (double)a.old_logprobs[n];
    const double e = exp(r.id == 0 ? (log_r > 700.0 ? 700.0 : log_r) : r.id == 1 ? gap : lp);
    const double ratio = __shfl(e, 0), e_gap = __shfl(e, 1), p = __shfl(e, 2);
    // 1 - p, also where lp is small: -lp - lp^2 / 2 - lp^3 / 6 is 4e-14 off at 1e-4.
    const double not_p = lp > -1e-4 ? -lp * (1.0 + lp * (0.5 + lp * (1.0 / 6.0))) : 1.0 - p;
    const double free_s = ratio * A, held = fmin(fmax(ratio, 1.0 - a.clip_low), 1.0 + a.clip_high) * A;
    // Written so that a NaN on either side stays one.
    const bool is_free = !(held < free_s);
    double loss = -(is_free ? free_s : held) - a.entropy_coef * H, g = is_free ? -free_s : 0.0;
    if (a.ref_logprobs != nullptr) {
      loss += a.kl_beta * (e_gap - gap - 1.0);
      g += a.kl_beta * (1.0 - e_gap);
    }
    if (r.id == 0) {
      a.losses[n] = none ? 0.f : (float)(w * loss);
      if (a.logprobs != nullptr) a.logprobs[n] = (float)lp;
      if (a.entropy != nullptr) a.entropy[n] = (float)H;
    }
    // d loss / d x_i = w / T (g ([i = y] - p_i) + b p_i (ln p_i + H)), ln p_i = d_i ln 2 - ln S.
    const double per = w * a.inv_t, b = a.entropy_coef;
    alpha = (float)(per * (b * (H - ln_s) - g) / sums[0]);
    beta = (float)(per * b * kLn2_64 / sums[0]);
    own = (float)(per * (g * not_p + (b != 0.0 && p > 0.0 ? b * p * (lp + H) : 0.0)));
  }
  if constexpr (GRAD) {
    if (none) {
      r.zero(out);
      return;
    }
    if constexpr (W > 1) {
      if (r.id == 0) {
        slots.out[0] = alpha;
        slots.out[1] = beta;
        slots.out[2] = own;
      }
      __syncthreads();
      alpha = slots.out[0];
      beta = slots.out[1];
      own = slots.out[2];
    }
    const Below below(m, c);
    r.store(row, out, [&](float x) {
      const float d = below(x);
      return fast_exp2(d) * fmaf(beta, fmaxf(d, kLeast), alpha);
    });
    // The token's own element comes after its vector, from the same thread.
    if (r.id == r.owner_of(y)) put_elem<DT>(out, y, own);
  }
}

// Entry j < k of a row's list counts where its id is in the vocabulary, is not
// listed before it and its value is above -inf.
struct Entry {
  int id;    // -1: does not count
  float x;   // its logit, then its gradient
  double e;  // of the student (not divided by S)
  double t;  // the teacher's value, then, but for REVERSE, its probability (TOPK: not divided by their sum)
};

// Words of the bits, with those of the vectors that no row has (a team's threads
// behind the last one look there too).
__host__ __device__ inline int bits_words(int vocab, int threads) { return cdiv(vocab, 32) + threads / 4; }

// Bound by the copy, as the policy loss: 2048 rows of 151936 bf16 logits with lists of
// 64 264 us, 4.6 TB/s; 1500 rows of 100003 fp16 with lists of 200 152 us, 4.0 TB/s,
// where seven of eight rows begin off a 16-byte boundary. The bits (a look-up a vector)
// keep the listed tokens out of the sums: subtracting them afterwards would leave the
// difference of two nearly equal numbers as the mass outside.
template <int DT, int W, int NV, bool GRAD>
__global__ __launch_bounds__(threads_of<W>()) void distill_kernel(const DistillArgs a) {
  static_assert(W > 1, "a workgroup per row");
  __shared__ Slots<W> slots;
  extern __shared__ __align__(16) char dynamic[];
  constexpr int NT = W * 64, E = Elem<DT>::kPerVec;
  const int V = a.logits.vocab, K = a.k, tid = threadIdx.x;
  Entry* list = reinterpret_cast<Entry*>(dynamic);
  uint32_t* listed = reinterpret_cast<uint32_t*>(list + K);  // a bit per token of the vocabulary
  const uint8_t* listed8 = reinterpret_cast<const uint8_t*>(listed);
  const float c = scale_of(a.inv_t);
  const int n = blockIdx.x;
  const char* row = row_of<DT>(a.logits, n);
  Row<DT, W, NV> r(V, row);
  char* out = GRAD ? grad_row<DT>(a.dlogits, a.dstride, n) : nullptr;
  const float w = a.weights != nullptr ? a.weights[n] : 1.f;
  if (w == 0.f) {
    if (tid == 0) a.losses[n] = 0.f;
    if constexpr (GRAD) r.zero(out);
    return;
  }
  r.fetch_all(row);
  for (int i = tid; i < bits_words(V, NT); i += NT) listed[i] = 0;
  // A vector's tokens have neighbouring bits, from a multiple of E on.
  const auto bit_of = [&](int id) { return id >= r.head ? id - r.head : V - r.head + id; };
  bool again = false;
  __syncthreads();
  for (int j = tid; j < K; j += NT) {
    int id = a.ids[(long long)n * K + j];
    const float value = a.values[(long long)n * K + j];
    if ((unsigned)id >= (unsigned)V || value == -INFINITY) id = -1;
    list[j].id = id;
    list[j].t = (double)value;
    if (id < 0) continue;
    list[j].x = Elem<DT>::get(row, id);
    const int bit = bit_of(id);
    again |= (atomicOr(&listed[bit / 32], 1u << (bit % 32)) >> (bit % 32) & 1u) != 0;
  }
  if (__syncthreads_or(again)) {
    // Some id is listed twice: its first place counts.
    bool drop[kMaxListed / NT];
#pragma unroll
    for (int i = 0; i < kMaxListed / NT; ++i) {
      const int j = i * NT + tid;
      drop[i] = false;
      if (j < K && list[j].id >= 0)
        for (int b = 0; b < j; ++b) drop[i] = drop[i] || list[b].id == list[j].id;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kMaxListed / NT; ++i)
      if (drop[i]) list[i * NT + tid].id = -1;
    __syncthreads();
  }
  // The largest logits outside the list and in it, and the list's largest value.
  float tops[3] = {-INFINITY, -INFINITY, -INFINITY};
  for (int j = tid; j < K; j += NT) {
    if (list[j].id < 0) continue;
    tops[1] = fmaxf(tops[1], list[j].x);
    tops[2] = fmaxf(tops[2], (float)list[j].t);
  }
  // The sum So over the tokens outside the list, relative to the largest of those, m_o:
  // however far they lie below the list, their mass has a logarithm and each has its
  // share e / So of it. Those of the list are added apart, so that a small mass
  // outside is no difference of large ones.
  double so_t[2];
  const float m_o = row_sums<W, !GRAD>(r, row, c, [&](int v, float (&x)[E]) {
    const int bit = v < r.whole || r.id >= r.loose ? v * E : bit_of(r.loose_of());
    uint32_t hit;
    if constexpr (E == 8) hit = v < r.whole ? listed8[v] : listed[bit / 32] >> (bit % 32) & 1u;
    else hit = listed[bit / 32] >> (bit % 32) & (v < r.whole ? 15u : 1u);
    if (hit == 0) return;
#pragma unroll
    for (int k = 0; k < E; ++k) x[k] = hit >> k & 1 ? -INFINITY : x[k];
  }, slots, so_t, tops);
  const float m = fmaxf(m_o, tops[1]), tm = tops[2];
  // Entry K stands for what is outside: its largest e.
  // So, and over the list: e, P, and the loss's terms but for ln S:
  // P (ln P - z) with P = exp(t) / total, or e (z - ln P).
  double sums[4] = {so_t[0], 0.0, 0.0, 0.0};
  for (int j = tid; j <= K; j += NT) {
    if (j < K && list[j].id < 0) continue;
    const double z = ((double)(j < K ? list[j].x : m_o) - (double)m) * a.inv_t, e = exp(z);
    if (j == K) {
      slots.far = e;
      continue;
    }
    const double t = a.kind == RP_DISTILL_TOPK ? (list[j].t - (double)tm) * a.inv_t : list[j].t;
    const double P = exp(t);
    list[j].e = e;
    if (a.kind != RP_DISTILL_REVERSE) list[j].t = P;
    sums[1] += e;
    sums[2] += P;
    // (0 P: a teacher's NaN or +inf stays.)
    if (a.kind == RP_DISTILL_REVERSE) sums[3] += e == 0.0 ? 0.0 * P : e * (z - t);
    else sums[3] += P == 0.0 ? 0.0 : P * (t - z);
  }
  team_sum<W>(sums, slots);
  const double So = sums[0], so = So * slots.far, s = so + sums[1], P_sum = sums[2];
  const bool empty = s == 0.0;
  const bool outside = !(So == 0.0);  // a NaN stays
  const double qo = so / s, per = (double)w * a.inv_t;
  const double left = 1.0 - P_sum, rest = left < 0x1p-24 ? 0x1p-24 : left;  // a NaN stays here too
  // The first lanes of every wave take a logarithm each.
  const int lane = tid % 64;
  const double logs = log(lane == 0 ? s : lane == 1 ? P_sum : lane == 2 ? So : rest);
  const double ln_s = __shfl(logs, 0), ln_P = __shfl(logs, 1);
  const double gap = __shfl(logs, 2) + ((double)m_o - (double)m) * a.inv_t - ln_s - __shfl(logs, 3);
  double loss, whole = 1.0, others;  // others: a token outside has e / So of it as its gradient
  if (a.kind == RP_DISTILL_TOPK) {
    const bool lists = !(P_sum == 0.0);  // an empty list teaches nothing
    loss = lists ? sums[3] / P_sum - ln_P + ln_s : 0.0 * s;
    others = lists ? qo : 0.0;
  } else if (a.kind == RP_DISTILL_TAIL) {
    loss = sums[3] + P_sum * ln_s - (outside ? rest * gap : 0.0);
    whole = P_sum + (outside ? rest : 0.0);
    others = whole * qo - rest;
  } else {
    loss = (sums[3] - ln_s * sums[1]) / s + (outside ? qo * gap : 0.0);
    others = qo * (gap - loss);
  }
  if (tid == 0) a.losses[n] = empty ? 0.f : (float)((double)w * loss);
  for (int j = tid; GRAD && j < K; j += NT) {
    if (list[j].id < 0) continue;
    const double q = list[j].e / s;
    double g;
    if (a.kind == RP_DISTILL_TOPK) g = q - list[j].t / P_sum;
    else if (a.kind == RP_DISTILL_TAIL) g = whole * q - list[j].t;
    else g = q == 0.0 ? 0.0 : q * (((double)list[j].x - (double)m) * a.inv_t - ln_s - list[j].t - loss);
    list[j].x = (float)(per * g);
  }
  if constexpr (GRAD) {
    if (empty) {
      r.zero(out);
      return;
    }
    // With nothing outside every other token is masked: 0, or NaN in a row that has one.
    const float alpha = outside ? (float)(per * others / So) : (float)(0.0 * s);
    const Below below(m_o, c);
    r.store(row, out, [&](float x) { return fast_exp2(below(x)) * alpha; });
    __syncthreads();  // the list's elements come after their vectors
    for (int j = tid; j < K; j += NT)
      if (list[j].id >= 0) put_elem<DT>(out, list[j].id, list[j].x);
  }
}

// Waves to a row, the same with and without a gradient, so that losses do not
// hang on it. Rows of up to 4096 vectors are held whole, by one wave or four.
// Longer ones go to eight waves, two rows to a compute unit, one computing while
// the other loads or stores (policy loss of 2048 rows of 151936 bf16 logits: 262
// us; sixteen waves, one row to a unit, 280; held whole in sixteen waves'
// registers, where every unit computes at the same time, 382); sixteen where
// there are too few rows for that (512 rows of 151936 fp32 logits: 139 us, 145;
// 24 rows of 32000 bf16: 13.9 us with four, 12.4).
template <int DT>
int waves_of(const LogitArgs& l) {
  const int vectors = cdiv(l.vocab, Elem<DT>::kPerVec);
  if (vectors <= 1024) return 1;
  if (vectors <= 4096) return l.rows > l.num_cus ? 4 : 16;
  return l.rows > 2 * l.num_cus ? 8 : 16;
}

template <int DT>
hipError_t logprobs(const LogprobArgs& a, hipStream_t stream) {
  const int rows = a.logits.rows;
  switch (waves_of<DT>(a.logits)) {
    case 1: logprobs_kernel<DT, 1><<<dim3(cdiv(rows, 4)), dim3(256), 0, stream>>>(a); break;
    case 4: logprobs_kernel<DT, 4><<<dim3(rows), dim3(256), 0, stream>>>(a); break;
    case 8: logprobs_kernel<DT, 8><<<dim3(rows), dim3(512), 0, stream>>>(a); break;
    default: logprobs_kernel<DT, 16><<<dim3(rows), dim3(1024), 0, stream>>>(a); break;
  }
  return hipGetLastError();
}

template <int DT>
hipError_t policy(const PolicyArgs& a, hipStream_t stream) {
  const int rows = a.logits.rows;
  const bool grad = a.dlogits != nullptr;
  switch (waves_of<DT>(a.logits)) {
    case 1:
      if (grad) policy_kernel<DT, 1, 16, true><<<dim3(cdiv(rows, 4)), dim3(256), 0, stream>>>(a);
      else policy_kernel<DT, 1, 0, false><<<dim3(cdiv(rows, 4)), dim3(256), 0, stream>>>(a);
      break;
    case 4:
      if (grad) policy_kernel<DT, 4, 16, true><<<dim3(rows), dim3(256), 0, stream>>>(a);
      else policy_kernel<DT, 4, 0, false><<<dim3(rows), dim3(256), 0, stream>>>(a);
      break;
    case 8:
      if (grad) policy_kernel<DT, 8, 14, true><<<dim3(rows), dim3(512), 0, stream>>>(a);
      else policy_kernel<DT, 8, 0, false><<<dim3(rows), dim3(512), 0, stream>>>(a);
      break;
    default:
      if (grad) policy_kernel<DT, 16, 12, true><<<dim3(rows), dim3(1024), 0, stream>>>(a);
      else policy_kernel<DT, 16, 0, false><<<dim3(rows), dim3(1024), 0, stream>>>(a);
      break;
  }
  return hipGetLastError();
}

template <int DT>
hipError_t distill(const DistillArgs& a, hipStream_t stream) {
  const dim3 grid(a.logits.rows);
  const bool grad = a.dlogits != nullptr;
  const auto lds = [&](int threads) { return sizeof(Entry) * a.k + (size_t)bits_words(a.logits.vocab, threads) * 4; };
  switch (waves_of<DT>(a.logits)) {
    case 1:
    case 4:
      if (grad) distill_kernel<DT, 4, 15, true><<<grid, dim3(256), lds(256), stream>>>(a);
      else distill_kernel<DT, 4, 0, false><<<grid, dim3(256), lds(256), stream>>>(a);
      break;
    case 8:
      if (grad) distill_kernel<DT, 8, 10, true><<<grid, dim3(512), lds(512), stream>>>(a);
      else distill_kernel<DT, 8, 0, false><<<grid, dim3(512), lds(512), stream>>>(a);
      break;
    default:
      if (grad) distill_kernel<DT, 16, 8, true><<<grid, dim3(1024), lds(1024), stream>>>(a);
      else distill_kernel<DT, 16, 0, false><<<grid, dim3(1024), lds(1024), stream>>>(a);
      break;
  }
  return hipGetLastError();
}

}  // namespace

#define RP_BY_DTYPE(f)                                        \
  switch (dtype) {                                            \
    case RP_LOGITS_BF16: return f<RP_LOGITS_BF16>(a, stream); \
    case RP_LOGITS_F16: return f<RP_LOGITS_F16>(a, stream);   \
    default: return f<RP_LOGITS_F32>(a, stream);              \
  }
hipError_t launch_logprobs(const LogprobArgs& a, int dtype, hipStream_t stream) { RP_BY_DTYPE(logprobs) }
hipError_t launch_policy(const PolicyArgs& a, int dtype, hipStream_t stream) { RP_BY_DTYPE(policy) }
hipError_t launch_distill(const DistillArgs& a, int dtype, hipStream_t stream) { RP_BY_DTYPE(distill) }
#undef RP_BY_DTYPE

}  // namespace rp
