// Sampling from rows of logits with temperature, top-k, top-p and min-p: one
// workgroup per row.
//
// In the order of falling logits (the lowest index first among equals) the
// kept tokens are a prefix, so they are described by a cut: every token whose
// key (its logit as an ordered integer) is above the cut's, and the first
// `ties` tokens, by index, at it. What decides (top-p's mass, the border that
// the random number falls on) are sums of weights 2^((x - max) log2(e) / T),
// and a border may be any of 10^5 tokens: in 32 bits some of them would move
// past each other. The weights are computed in 64 bits (a polynomial, 4e-14),
// and summed in 64 bits, or as integers in steps of 2^-S of the largest, which
// any order of additions sums alike.
//
// One pass over the row finds its maximum, its sum (in 32 bits where no border
// hangs on it) and the largest key of every vector, which stays in LDS: later
// passes load only vectors that hold a token they look for. Few tokens above a
// threshold (all that top-k, or a nucleus of usual size, can keep) become a
// list in LDS, and the cut and the token are found there by histograms over
// slices of the keys, and of the indices. Where what is kept is more than a list
// holds, a histogram of the whole row says between which two logits the cut lies,
// and one pass sums what is above them and lists what is between them.
//
// What bounds it (256 rows of 151936 bf16 logits, 11 us to read): without filters
// 46 us, in which a unit is busy for 104e3 cycles: 33 vector instructions a logit
// (counted), 18 of them in 64 bits at 4 cycles for a wave and the others at 2, are
// 60e3 of those, and loads and the chain behind the pass the rest; top-k 30 and min-p
// 27 us (35 where rows are flat), the first pass 23 (32-bit weights) and the rest the
// chain of short steps between barriers; a nucleus of 10^5 tokens 106 us, the row's
// two further passes, one of them in 64-bit weights. A single row takes 15 to 25 us,
// nearly all in that chain.
#include "rp_rows.h"

namespace rp {
namespace {

typedef unsigned long long u64;
constexpr int kBins = 1024;
constexpr int kNoCrossing = 0x7FFFFFFF;
// A stretch whose kept weight is less adds nothing. Above it, some token there has a
// weight of its own above 0, whichever way the sum was taken.
constexpr double kLeastSum = 0x1p-1000;

// A listed token: its place in the order of keys, then of falling indices, and its weight.
struct Token {
  u64 place;
  u64 mass;
  __device__ inline uint32_t key() const { return (uint32_t)(place >> 32); }
  __device__ inline uint32_t late() const { return (uint32_t)place; }  // ~index: more for lower indices
};

template <int NT>
struct Lds {
  static constexpr int kWaves = NT / 64;
  static constexpr int kEntries = NT == 256 ? 16 : 32;  // largest keys kept per thread
  static constexpr int kList = 2 * NT;
  float f[kWaves];
  double d[kWaves];
  int i[kWaves];
  u64 q[kWaves];
  static constexpr int kSmall = NT == 256 ? 128 : 256;  // lists that are sorted by counting
  u64 hist[kBins];
  Token list[kList];
  uint32_t work[kList];
  u64 over[kSmall];
  int rank[kSmall];
  uint16_t top[kEntries * NT];
  u64 above;
  int bin, count, works, first, spare;
  uint32_t least, most;
};

// Logits as unsigned numbers of the same order, -0 and 0 the same; the bits
// that 16-bit types leave constant are shifted out.
template <int DT>
struct Key {
  static constexpr int kShift = DT == RP_LOGITS_BF16 ? 16 : DT == RP_LOGITS_F16 ? 13 : 0;
  static constexpr uint32_t kNegInf = 0x007FFFFFu >> kShift;
  static __device__ inline uint32_t of(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return (u & 0x80000000u ? ~u : u | 0x80000000u) >> kShift;
  }
  static __device__ inline float logit(uint32_t key) {
    const uint32_t o = key << kShift;
    return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~(o | ((1u << kShift) - 1)));
  }
  // The upper 16 bits of the order: what LDS keeps of a vector's largest key.
  static __device__ inline uint32_t upper(uint32_t key) { return (key << kShift) >> 16; }
};

// 2^y for -1500 <= y, to 4e-14: y = n + f with |f| <= 1/2, and 2^f by the
// polynomial of degree 9 that is 1 at 0 and interpolates 2^f at the zeros of
// the Chebyshev polynomial of degree 9, scaled to [-1/2, 1/2].
__device__ inline double pow2(double y) {
  constexpr double kRound = 0x1.8p52;
  const double t = y + kRound;
  const double f = y - (t - kRound);
  double p = 0x1.b63881021ff95p-24;
  p = fma(p, f, 0x1.63d13637e6ed6p-20);
  p = fma(p, f, 0x1.ffcb95154c637p-17);
  p = fma(p, f, 0x1.4308ac85a8c94p-13);
  p = fma(p, f, 0x1.5d87fe86fea1bp-10);
  p = fma(p, f, 0x1.3b2ab7181b769p-7);
  p = fma(p, f, 0x1.c6b08d7047e52p-5);
  p = fma(p, f, 0x1.ebfbdff823cedp-3);
  p = fma(p, f, 0x1.62e42fefa39efp-1);
  p = fma(p, f, 1.0);
  return ldexp(p, __double2loint(t));
}

// Weights relative to the logit `ref`: exactly 0 for -inf.
__device__ inline double weight(float x, float ref, double c) {
  return pow2(fmax(((double)x - (double)ref) * c, -1500.0));
}
// N at once: their chains of products interleave.
template <int N>
__device__ __attribute__((always_inline)) inline void weights(const float (&x)[N], float ref, double c, double (&w)[N]) {
  constexpr double kRound = 0x1.8p52;
  constexpr double kPoly[] = {0x1.b63881021ff95p-24, 0x1.63d13637e6ed6p-20, 0x1.ffcb95154c637p-17, 0x1.4308ac85a8c94p-13,
                              0x1.5d87fe86fea1bp-10, 0x1.3b2ab7181b769p-7,  0x1.c6b08d7047e52p-5,  0x1.ebfbdff823cedp-3,
                              0x1.62e42fefa39efp-1,  1.0};
  constexpr int G = 4;
  static_assert(N % G == 0, "whole groups");
#pragma unroll
  for (int g = 0; g < N; g += G) {
    double f[G], p[G];
    int n[G];
#pragma unroll
    for (int i = 0; i < G; ++i) f[i] = fmax(((double)x[g + i] - (double)ref) * c, -1500.0);
#pragma unroll
    for (int i = 0; i < G; ++i) {
      const double t = f[i] + kRound;
      n[i] = __double2loint(t);
      f[i] -= t - kRound;
      p[i] = kPoly[0];
    }
#pragma unroll
    for (int k = 1; k < 10; ++k) {
#pragma unroll
      for (int i = 0; i < G; ++i) p[i] = fma(p[i], f[i], kPoly[k]);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int i = 0; i < G; ++i) w[g + i] = ldexp(p[i], n[i]);
  }
}
// In steps of 2^-S, scale = 2^S <= 2^50.
__device__ inline u64 mass_of(double w, double scale) {
  return (u64)__double_as_longlong(fma(w, scale, 0x1p52)) & ((1ull << 52) - 1);
}

// The row, and which vectors of it a thread has: wave w has the stretch of
// `steps` * 64 vectors from w * steps * 64 on, in the order of indices; entry g of
// a thread is the largest key of its vectors j with j >> shift == g.
template <int DT, int NT>
struct Row {
  static constexpr int E = Elem<DT>::kPerVec;
  const void* data;
  int vocab, steps, shift, entries;
  float max;
  double c;
  __device__ inline Row(const LogitArgs& l, int n)
      : data(static_cast<const char*>(l.data) + (long long)n * l.stride * Elem<DT>::kBytes),
        vocab(l.vocab),
        steps(cdiv(cdiv(l.vocab, E), NT)),
        shift(0) {
    while (cdiv(steps, 1 << shift) > Lds<NT>::kEntries) ++shift;
    entries = cdiv(steps, 1 << shift);
  }
  __device__ inline int vec(int thread, int j) const { return (thread / 64 * steps + j) * 64 + thread % 64; }
  __device__ inline bool has(int thread, int j) const { return j < steps && vec(thread, j) * E < vocab; }
  // f(vector, its logits) for this thread's vectors whose largest key is `upper` or more;
  // U of them requested ahead (the code is U times there).
  template <int U, class F>
  __device__ __attribute__((always_inline)) inline void each(const Lds<NT>& l, uint32_t upper, const F& f) const {
    const int tid = threadIdx.x;
    u32x4_any next[U];
    uint32_t wanted = 0;
    const auto fetch = [&](int j0) __attribute__((always_inline)) {
      wanted = 0;
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int j = j0 + i;
        if (!has(tid, j) || l.top[(j >> shift) * NT + tid] < upper) continue;
        next[i] = load_vec<DT>(data, vec(tid, j), vocab);
        wanted |= 1u << i;
      }
    };
    fetch(0);
#pragma unroll 1
    for (int j0 = 0; j0 < steps; j0 += U) {
      u32x4_any now[U];
#pragma unroll
      for (int i = 0; i < U; ++i) now[i] = next[i];
      const uint32_t take = wanted;
      fetch(j0 + U);
#pragma unroll
      for (int i = 0; i < U; ++i) {
        if (!(take >> i & 1)) continue;
        float x[E];
        unpack<DT>(now[i], x);
        f(vec(tid, j0 + i), x);
      }
    }
  }
};

// How row n is sampled. Greedy is top-1 at T = 1. c = log2(e) / T stays above 0, so
// that -inf weighs nothing at T = inf too, in 64 bits. In 32 bits c would be 0 there,
// and where T is far from 1 it loses digits, or a difference of logits that still
// counts passes fp32's largest number (odd): such rows are done in 64 bits throughout.
struct How {
  int k;        // vocab: all
  double p, q;  // 1 and 0: all
  double inv_t, c;
  bool all, light;  // all: a border hangs on every token's weight; light: k few enough for a list
  bool odd, exact;  // exact: the row's sum is in 64 bits
  __device__ inline How(const SampleArgs& a, int n, int lightest) {
    const int V = a.logits.vocab;
    const float T = a.temperature != nullptr ? a.temperature[n] : 1.f;
    const bool greedy = !(T > 0.f);
    const int asked_k = greedy ? 1 : a.top_k != nullptr ? a.top_k[n] : 0;
    const float asked_p = greedy || a.top_p == nullptr ? 1.f : a.top_p[n];
    const float asked_q = greedy || a.min_p == nullptr ? 0.f : a.min_p[n];
    k = asked_k > 0 && asked_k < V ? asked_k : V;
    p = asked_p < 1.f ? fmax((double)asked_p, 0.0) : 1.0;
    q = asked_q > 0.f && T < INFINITY ? fmin((double)asked_q, 1.0) : 0.0;  // at T = inf all weigh 1
    inv_t = greedy ? 1.0 : fmax(1.0 / (double)T, 1e-300);
    c = kLog2e64 * inv_t;
    odd = !(c >= 1e-30 && c <= 1e38);
    light = k < V && k <= lightest;
    all = k >= V && p >= 1.0 && q == 0.0;
    exact = all || odd;
  }
};

// What a pass over some of a stretch's vectors finds: the largest logit, and the
// weights' sum relative to `ref`: in 64 bits (s), or in 32, the vector with the
// largest logit (at) apart from the others.
struct Scan {
  float top = -INFINITY, ref = -INFINITY, group = 0.f, rest = 0.f;
  double s = 0.0;
  int at = -1;
  bool bad = false;  // a NaN or +inf
};

// Entries first, first + stride, .. of the thread's vectors; put(entry, largest key).
template <int DT, int NT, class Put>
__device__ __attribute__((always_inline)) inline Scan scan(const Row<DT, NT>& r, int thread, int first, int stride,
                                                           bool exact, const Put& put) {
  constexpr int E = Elem<DT>::kPerVec, U = 4;
  typedef Key<DT> K;
  Scan o;
  const float c32 = (float)r.c;
  const int each = (1 << r.shift) - 1, count = r.entries > first ? cdiv(r.entries - first, stride) << r.shift : 0;
  const auto at = [&](int i) { return ((i >> r.shift) * stride + first) << r.shift | (i & each); };
  u32x4_any next[U];
  const auto fetch = [&](int i0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (i0 + i < count && r.has(thread, at(i0 + i))) next[i] = load_vec<DT>(r.data, r.vec(thread, at(i0 + i)), r.vocab);
  };
  uint32_t entry = 0;
  fetch(0);
#pragma unroll 1
  for (int i0 = 0; i0 < count; i0 += U) {
    u32x4_any now[U];
#pragma unroll
    for (int i = 0; i < U; ++i) now[i] = next[i];
    fetch(i0 + U);
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (i0 + i >= count) break;
      const int j = at(i0 + i);
      if (r.has(thread, j)) {
        float x[E];
        unpack<DT>(now[i], x);
        float most = x[0];  // a NaN passes through
#pragma unroll
        for (int e = 1; e < E; ++e) most = __builtin_elementwise_maximum(most, x[e]);
        o.bad = o.bad || !(most < INFINITY);
        entry = max(entry, K::upper(K::of(most)));
        if (!(most > -INFINITY)) {
          // nothing to sum
        } else if (exact) {
          // The reference moves when a weight would pass 2^256, which 64 bits hold.
          if (!((double)(most - o.ref) * r.c < 256.0)) {
            o.s *= weight(o.ref, most, r.c);
            o.ref = most;
          }
          double w[E];
          weights(x, o.ref, r.c, w);
#pragma unroll
          for (int e = 1; e < E; ++e) w[0] += w[e];
          o.s += w[0];
        } else {
          const bool more = most > o.top;
          if (more) {
            o.rest = (o.rest + o.group) * fast_exp2((o.top - most) * c32);
            o.ref = most;
            o.at = r.vec(thread, j);
          }
          float s = 0.f;
#pragma unroll
          for (int e = 0; e < E; ++e) s += fast_exp2((x[e] - o.ref) * c32);
          if (more) o.group = s;
          else o.rest += s;
        }
        o.top = fmaxf(o.top, most);
      }
      if (((i0 + i) & each) == each) {
        put(j >> r.shift, (uint16_t)entry);
        entry = 0;
      }
    }
  }
  return o;
}

// A scan's sum relative to the maximum of the scans that it is joined with.
template <int DT, int NT>
__device__ inline double sum_to(const Scan& o, const Row<DT, NT>& r, float max, bool exact) {
  if (!(o.ref > -INFINITY)) return 0.0;
  if (exact) return o.s * weight(o.ref, max, r.c);
  const float c32 = (float)r.c;
  if (o.top < max) return (double)((o.rest + o.group) * fast_exp2((o.ref - max) * c32));
  // The vector with the maximum again, in 64 bits: where one token has nearly all
  // the mass, ln Z is that of the rest.
  float x[Elem<DT>::kPerVec];
  unpack<DT>(load_vec<DT>(r.data, o.at, r.vocab), x);
  double s = (double)o.rest;
#pragma unroll
  for (int e = 0; e < Elem<DT>::kPerVec; ++e) s += (double)fast_exp2((x[e] - max) * c32);
  return s;
}

// Few rows leave most of the chip idle, so their stretches are scanned by workgroups
// of their own (scan_kernel); their results, and the entries, go through memory.
struct Part {
  float top;
  int bad;
  double s;
};
constexpr int kSplit = 16, kSplitThreads = 1024, kScanThreads = 256;
struct SplitRow {
  Part part[kSplit];
  uint16_t top[32 * kSplitThreads];
};
static_assert(kSplit * 64 == kSplitThreads && Lds<kSplitThreads>::kEntries == 32, "a stretch per wave");

template <int DT>
__global__ __launch_bounds__(kScanThreads) void scan_kernel(const SampleArgs a) {
  __shared__ float lds_f[kScanThreads / 64];
  __shared__ double lds_d[kScanThreads / 64];
  const int n = blockIdx.x / kSplit, stretch = blockIdx.x % kSplit, tid = threadIdx.x;
  SplitRow& out = static_cast<SplitRow*>(a.workspace)[n];
  Row<DT, kSplitThreads> r(a.logits, n);
  const How how(a, n, kSplitThreads / 2);
  r.c = how.c;
  const int thread = stretch * 64 + tid % 64;
  const Scan o = scan(r, thread, tid / 64, kScanThreads / 64, how.exact,
                      [&](int g, uint16_t key) { out.top[g * kSplitThreads + thread] = key; });
  const float top = block_max<kScanThreads>(o.top, lds_f);
  const bool bad = __syncthreads_or(o.bad);
  const double s = block_sum<kScanThreads>(bad ? 0.0 : sum_to(o, r, top, how.exact), lds_d);
  if (tid == 0) out.part[stretch] = {top, bad ? 1 : 0, s};
}

// The place, from the top of BINS bins, where the sums of value(bin) reach `need`
// (at most all of it): its bin, the sum above, and that of all bins. A barrier has to
// lie between whatever last read l.q, l.bin or l.above and this, which writes them
// before its own first one.
struct Place {
  int bin;
  u64 above, all;
};
template <int NT, int BINS, class Value>
__device__ inline Place find_top(Lds<NT>& l, u64 need, const Value& value) {
  constexpr int PER = BINS / NT;
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  u64 h[PER], sum = 0;
#pragma unroll
  for (int k = 0; k < PER; ++k) sum += h[k] = value(BINS - 1 - (tid * PER + k));
  u64 upto = sum;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const u64 u = __shfl_up(upto, o);
    if (lane >= o) upto += u;
  }
  if (lane == 63) l.q[wave] = upto;
  if (tid == 0) {
    l.bin = 0;
    l.above = 0;
  }
  __syncthreads();
  u64 all = 0;
#pragma unroll
  for (int w = 0; w < Lds<NT>::kWaves; ++w) {
    if (w < wave) upto += l.q[w];
    all += l.q[w];
  }
  need = need < all ? need : all;
  u64 run = upto - sum;
  if (run < need && need <= upto) {
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      if (run < need && need <= run + h[k]) {
        l.bin = BINS - 1 - (tid * PER + k);
        l.above = run;
      }
      run += h[k];
    }
  }
  __syncthreads();
  return {l.bin, l.above, all};
}

template <int NT>
__device__ inline Place find_top(Lds<NT>& l, u64 need) {
  return find_top<NT, kBins>(l, need, [&](int bin) { return l.hist[bin]; });
}

template <int NT>
__device__ inline void clear(u64 (&hist)[kBins]) {
#pragma unroll
  for (int b = 0; b < kBins; b += NT) hist[b + threadIdx.x] = 0;
}

// The largest key in [lo, hi] at which the masses from hi down reach `need`,
// with what lies above it. items(f) calls f(key, mass) for a thread's items.
struct Cut {
  uint32_t key;
  u64 above;
};
template <int NT, class Items>
__device__ __attribute__((always_inline)) inline Cut descend(Lds<NT>& l, uint32_t lo, uint32_t hi, u64 need, const Items& items) {
  u64 over = 0;
  uint32_t width = hi - lo;
  while (true) {
    const int s = max(22 - __clz((int)(width | 1)), 0);  // slices of 2^s keys, at most kBins of them
    __syncthreads();
    clear<NT>(l.hist);
    __syncthreads();
    items([&](uint32_t key, u64 mass) {
      if (key - lo <= width) atomicAdd(&l.hist[(key - lo) >> s], mass);
    });
    __syncthreads();
    const Place at = find_top(l, need);
    const uint32_t bin = (uint32_t)at.bin;
    need -= at.above < need ? at.above : need;
    over += at.above;
    lo += bin << s;
    if (s == 0) return {lo, over};
    width = min(width - (bin << s), (1u << s) - 1);
  }
}

// Lists the tokens whose key is tau or more; whether they fit.
template <int DT, int NT>
__device__ inline bool gather(Lds<NT>& l, const Row<DT, NT>& r, uint32_t tau, double scale) {
  constexpr int E = Elem<DT>::kPerVec;
  const int tid = threadIdx.x, entries = cdiv(r.steps, 1 << r.shift);
  const uint32_t upper = Key<DT>::upper(tau);
  __syncthreads();
  if (tid == 0) l.count = l.works = 0;
  __syncthreads();
  for (int g = 0; g < entries; ++g) {
    if (l.top[g * NT + tid] < upper) continue;
    const int at = atomicAdd(&l.works, 1);
    if (at < Lds<NT>::kList) l.work[at] = g * NT + tid;
  }
  __syncthreads();
  const int works = l.works;
  if (works > Lds<NT>::kList) return false;
  for (int i = tid; i < works << r.shift; i += NT) {
    const int item = l.work[i >> r.shift], j = (item / NT << r.shift) + (i & ((1 << r.shift) - 1));
    const int v = r.vec(item % NT, j);
    if (j >= r.steps || v * E >= r.vocab) continue;
    float x[E];
    unpack<DT>(load_vec<DT>(r.data, v, r.vocab), x);
#pragma unroll
    for (int k = 0; k < E; ++k) {
      const uint32_t key = Key<DT>::of(x[k]);
      if (key < tau) continue;
      const int at = atomicAdd(&l.count, 1);
      if (at >= Lds<NT>::kList) continue;
      l.list[at] = {(u64)key << 32 | ~(uint32_t)(v * E + k), mass_of(weight(x[k], r.max, r.c), scale)};
    }
  }
  __syncthreads();
  return l.count <= Lds<NT>::kList;
}

// SPLIT: scan_kernel has been over the row.
template <int DT, int NT, bool SPLIT>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(4))) void sample_kernel(const SampleArgs a) {
  __shared__ Lds<NT> l;
  typedef Key<DT> K;
  constexpr int E = Elem<DT>::kPerVec, kWaves = Lds<NT>::kWaves;
  const int n = blockIdx.x, V = a.logits.vocab, tid = threadIdx.x, wave = tid / 64, lane = tid % 64;
  Row<DT, NT> r(a.logits, n);
  const How how(a, n, NT / 2);
  r.c = how.c;
  const int k = how.k;
  const double p = how.p, q = how.q, inv_t = how.inv_t;
  const bool light_k = how.light, all = how.all;

  float top = -INFINITY;  // the thread's largest logit (SPLIT: or less than that, by the bits that the entries lack)
  bool bad = false;
  if constexpr (SPLIT) {
    const SplitRow& in = static_cast<const SplitRow*>(a.workspace)[n];
    const Part part = in.part[tid % kSplit];
    r.max = wave_max(part.top);
    bad = __ballot(part.bad != 0) != 0;
    if (tid < kSplit && part.top > -INFINITY)
      l.d[tid] = part.s * (how.exact ? weight(part.top, r.max, r.c)
                                     : (double)fast_exp2((part.top - r.max) * (float)r.c));
    else if (tid < kSplit) l.d[tid] = 0.0;
    uint32_t most = 0;
    for (int g = 0; g < r.entries; ++g) {
      const uint16_t key = in.top[g * NT + tid];
      l.top[g * NT + tid] = key;
      most = max(most, (uint32_t)key);
    }
    const uint32_t o = most << 16;
    if (most > 0x007Fu) top = __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o);
  } else {
    const Scan o = scan(r, tid, 0, 1, how.exact, [&](int g, uint16_t key) { l.top[g * NT + tid] = key; });
    top = o.top;
    r.max = block_max<NT>(top, l.f);
    bad = __syncthreads_or(o.bad);
    if (!bad && r.max > -INFINITY) {
      const double s = wave_sum(sum_to(o, r, r.max, how.exact));
      if (lane == 0) l.d[wave] = s;
    }
  }
  if (bad || r.max == -INFINITY) {
    if (tid == 0) {
      const float none = bad ? NAN : -INFINITY;
      a.tokens[n] = -1;
      if (a.logprobs != nullptr) a.logprobs[n] = none;
      if (a.kept != nullptr) a.kept[n] = none;
    }
    return;
  }
  __syncthreads();
  double Z = 0.0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) Z += l.d[w];
  int spread;
  (void)frexp(Z, &spread);
  const double scale = ldexp(1.0, min(50, 60 - spread));  // masses sum to less than 2^62

  float u = a.u[n];
  if (!(u >= 0.f)) u = 0.f;
  const double part = (double)fminf(u, 0x1.fffffep-1f);

  const auto finish = [&](int token, double total) __attribute__((always_inline)) {
    const double z = ((double)Elem<DT>::get(r.data, max(token, 0)) - (double)r.max) * inv_t;
    a.tokens[n] = token;
    if (a.logprobs != nullptr) a.logprobs[n] = (float)(z - log(Z));
    if (a.kept != nullptr) a.kept[n] = (float)(z - log(total));
  };

  uint32_t cut = K::kNegInf;  // keys above it are kept, and the first `ties` at it
  int ties = 0;
  bool listed = false, summed = all;  // summed: l.d and l.i hold the stretches' kept weight and ties
  if (all && lane == 0) l.i[wave] = 0;
  if (!all) {
    // A key down to which the threads' largest logits alone are `need` tokens (or, by
    // mass, weigh that much), so that all that is kept lies there; 0 if they never do.
    const float least_top = -block_max<NT>(top > -INFINITY ? -top : -INFINITY, l.f);
    const auto reached = [&](bool by_mass, u64 need) __attribute__((always_inline)) {
      const float fit = fmaxf(fminf(r.max - least_top, 1e30f), 1e-30f);
      const int bin = kBins - 1 - (int)fminf((r.max - top) * ((kBins - 2) / fit), kBins - 1.f);
      const bool has = top > -INFINITY;
      const u64 mine = !has ? 0 : by_mass ? mass_of(weight(top, r.max, r.c), scale) : 1;
      __syncthreads();
      clear<NT>(l.hist);
      if (tid == 0) l.least = 0xFFFFFFFFu;
      __syncthreads();
      if (has) atomicAdd(&l.hist[bin], mine);
      __syncthreads();
      const Place at = find_top(l, need);
      if (at.all < need) return 0u;
      if (has && bin >= at.bin) atomicMin(&l.least, K::of(top));
      __syncthreads();
      return l.least;
    };
    const auto from_list = [&](auto&& f) __attribute__((always_inline)) {
      const int count = l.count;
      for (int i = tid; i < count; i += NT) f(l.list[i].key(), l.list[i].late(), l.list[i].mass);
    };
    const uint32_t most = K::of(r.max);
    const bool probe = k >= V && p < 1.0;
    // The mass of the nucleus, where every token counts, for which Z in 32 bits leaves
    // a range: a term is off by (3 |d| + 2) 2^-24, |d| ln 2 averages at most ln V < 14,
    // and a thread adds `steps` of them, in vectors of 8. (Rows of 2^20 rising fp32 logits,
    // whose reference moves with every vector, were off by up to 18 of the 640 steps of
    // 2^-24 that this leaves.)
    const double off = (128.0 + r.steps) * 0x1p-24;
    const u64 need_lo = (u64)fmax(ceil(p * Z * (1.0 - off) * scale), 1.0);
    const u64 need_hi = max((u64)ceil(p * Z * (1.0 + off) * scale), need_lo);
    uint32_t key_q = 0;  // the least key of weight q or more
    if (q > 0.0) {
      const double least = (double)r.max + log2(q) / r.c;
      key_q = K::of((float)least);
      if (!((double)K::logit(key_q) >= least)) ++key_q;
      key_q = min(max(key_q, K::kNegInf + 1), most);
    }
    uint32_t tau = 0;
    if (light_k) tau = max(reached(false, (u64)k), K::kNegInf + 1);
    else if (probe) tau = reached(true, need_hi);
    else if (k >= V) tau = key_q;
    if (tau != 0)
      listed = gather(l, r, tau, scale);

    // A short list: every token counts those before it, in the order of keys and in
    // that of indices, the waves sharing out whom they count.
    while (listed && l.count <= Lds<NT>::kSmall) {
      const int count = l.count, blocks = cdiv(count, 64), shares = kWaves / blocks;
      const int at = wave % blocks * 64 + lane, share = wave / blocks;
      const int from = share * count / shares, to = share < shares ? (share + 1) * count / shares : from;
      const bool is = tid < count;
      const auto tally = [&](auto&& add) __attribute__((always_inline)) {
        if (at < count) add(l.list[at].place);
      };
      if (is) {
        l.rank[tid] = 0;
        l.over[tid] = 0;
      }
      __syncthreads();
      tally([&](u64 place) {
        int rank = 0;
        u64 over = 0;
        for (int j = from; j < to; ++j) {
          const Token t = l.list[j];
          rank += t.place > place ? 1 : 0;
          over += t.place > place ? t.mass : 0;
        }
        if (from < to) {
          atomicAdd(&l.rank[at], rank);
          atomicAdd(&l.over[at], over);
        }
      });
      __syncthreads();
      const Token mine = is ? l.list[tid] : Token{0, 0};
      bool in = is && l.rank[tid] < k;
      if (p < 1.0) {
        u64 need = need_lo;
        if (k < V) need = (u64)fmax(ceil(p * (double)block_sum<NT>(in ? mine.mass : 0, l.q)), 1.0);
        const bool kept = in && l.over[tid] < need;
        if (probe && __syncthreads_or(in && !kept && l.over[tid] < need_hi)) {
          listed = false;  // Z in 32 bits does not tell
          break;
        }
        in = kept;
      }
      in = in && mine.key() >= key_q;
      const u64 mass = in ? mine.mass : 0, sum = block_sum<NT>(mass, l.q);
      const u64 need = min((u64)floor(part * (double)sum) + 1, sum);
      if (is) {
        l.list[tid].mass = mass;
        l.over[tid] = 0;
      }
      __syncthreads();
      tally([&](u64 place) {
        u64 upto = 0;
        for (int j = from; j < to; ++j) {
          const Token t = l.list[j];
          upto += t.late() >= (uint32_t)place ? t.mass : 0;
        }
        if (from < to) atomicAdd(&l.over[at], upto);
      });
      __syncthreads();
      if (mass > 0 && l.over[tid] >= need && l.over[tid] - mass < need) finish((int)~mine.late(), (double)sum / scale);
      return;
    }
    const int listed_n = l.count;

    // The key at which the tokens' masses (their number, where `count`) reach
    // `need`, from the row itself: by equal steps of the logits down to `low`,
    // then within one of those.
    const auto from_row = [&](bool count, u64 need, float low, uint32_t upper) __attribute__((always_inline)) {
      const float fit = fmaxf(fminf(r.max - low, 1e30f), 1e-30f), per = (kBins - 2) / fit;
      const auto step = [&](float x) __attribute__((always_inline)) { return kBins - 1 - (int)fminf((r.max - x) * per, kBins - 1.f); };
      const auto one = [&](float x) __attribute__((always_inline)) { return count ? 1ull : mass_of(weight(x, r.max, r.c), scale); };
      __syncthreads();
      clear<NT>(l.hist);
      if (tid == 0) {
        l.least = 0xFFFFFFFFu;
        l.most = 0;
      }
      __syncthreads();
      r.template each<1>(l, upper, [&](int, const float (&x)[E]) {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (x[e] > -INFINITY) atomicAdd(&l.hist[step(x[e])], one(x[e]));
      });
      __syncthreads();
      const Place place = find_top(l, need);
      const int at = place.bin;
      need -= place.above < need ? place.above : need;
      // The keys of that step, and a threshold for the vectors that hold them.
      const float edge = at == 0 ? -INFINITY : r.max - (float)(kBins - at) / per;
      const float slack = at == 0 ? 0.f : fabsf(edge) * 1e-5f + fit * 1e-4f;
      const uint32_t edge_upper = max(upper, at == 0 ? 0u : K::upper(K::of(edge - slack)));
      uint32_t lo = 0xFFFFFFFFu, hi = 0;
      r.template each<1>(l, edge_upper, [&](int, const float (&x)[E]) {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (x[e] > -INFINITY && step(x[e]) == at) {
            lo = min(lo, K::of(x[e]));
            hi = max(hi, K::of(x[e]));
          }
      });
      atomicMin(&l.least, lo);
      atomicMax(&l.most, hi);
      __syncthreads();
      lo = l.least;
      hi = l.most;
      Cut found = descend(l, lo, hi, need, [&](auto&& f) {
        r.template each<1>(l, edge_upper, [&](int, const float (&x)[E]) {
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const uint32_t key = K::of(x[e]);
            if (key >= lo && key <= hi) f(key, one(x[e]));
          }
        });
      });
      found.above += place.above;
      return found;
    };

    const auto tokens_at_all = [&] __attribute__((always_inline)) {
      int finite = 0;
      r.template each<1>(l, 0, [&](int, const float (&x)[E]) {
#pragma unroll
        for (int e = 0; e < E; ++e) finite += x[e] > -INFINITY ? 1 : 0;
      });
      return block_sum<NT>(finite, l.i);
    };
    // Where the tokens that are kept are many: their number, or their weight in steps
    // of 2^-31 of the row's, by equal steps of the logits says which of those the cut
    // lies in; then one pass sums what is above those steps, by stretch, and lists what
    // is in them. Tokens at `least` and below do not count: LDS would add to one bin
    // for most of a wave. False where that does not settle it. (512 flat rows of 50257
    // fp32 logits: 89 us; three passes with 64-bit masses in the bins, from_row, 186.)
    bool settled = false;  // cut and ties are known
    bool whole_sum = how.odd;  // Z is the sum in 64 bits
    const auto wide = [&](bool by_mass, u64 from, u64 to, float low, uint32_t upper, float least) __attribute__((always_inline)) {
      constexpr int BINS = 2 * kBins;
      uint32_t* counts = reinterpret_cast<uint32_t*>(l.hist);
      const float c32 = (float)r.c, fine = (float)(0x1p31 / Z);
      const float fit = fmaxf(fminf(r.max - low, 1e30f), 1e-30f), per = (BINS - 2) / fit;
      const auto step = [&](float x) __attribute__((always_inline)) { return BINS - 1 - (int)fminf((r.max - x) * per, BINS - 1.f); };
      __syncthreads();
      clear<NT>(l.hist);
      __syncthreads();
      r.template each<4>(l, upper, [&](int, const float (&x)[E]) {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (x[e] > least) {
            // (Whole numbers: LDS adds floats one lane after the other, 192 cycles a wave.)
            const uint32_t one = by_mass ? (uint32_t)fmaf(fast_exp2((x[e] - r.max) * c32), fine, 0.5f) : 1u;
            atomicAdd(&counts[step(x[e])], one);
          }
      });
      __syncthreads();
      const auto value = [&](int bin) __attribute__((always_inline)) {
        return by_mass ? (u64)((double)counts[bin] * (0x1p-31 * Z * scale)) : (u64)counts[bin];
      };
      const u64 slack = by_mass ? (u64)(Z * scale * (V * 0x1p-32 + off)) : 0;  // half a step a token, and Z's
      const int hi = find_top<NT, BINS>(l, from > slack ? from - slack : 1, value).bin;
      __syncthreads();
      const int lo = by_mass ? find_top<NT, BINS>(l, to + slack, value).bin : hi;
      if (lo <= 0) return false;
      if (key_q > 0 && step(K::logit(key_q)) > hi) {
        cut = key_q;
        ties = V;
        settled = true;
        return false;
      }
      // Those steps as logits, with room for roundings: what lies there is listed.
      const auto room = [&](float edge) { return fabsf(edge) * 1e-5f + fit * 1e-5f; };
      const float first = r.max - (float)(BINS - lo) / per, last = r.max - (float)(BINS - 1 - hi) / per;
      const float x_lo = first - room(first), x_hi = last + room(last);
      // Z is summed on the way, over every vector.
      const uint32_t edge_upper = by_mass ? 0 : max(upper, K::upper(K::of(x_lo)));
      __syncthreads();
      if (tid == 0) {
        l.count = 0;
        l.least = 0xFFFFFFFFu;
        l.most = 0;
      }
      __syncthreads();
      double s = 0.0, every = 0.0;
      int n_over = 0;
      r.template each<4>(l, edge_upper, [&](int v, const float (&x)[E]) {
        uint32_t in = 0;
        double w[E];
        weights(x, r.max, r.c, w);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const bool over = x[e] > x_hi;
          s += over ? w[e] : 0.0;
          every += w[e];
          n_over += over ? 1 : 0;
          in |= x[e] >= x_lo && !over ? 1u << e : 0u;
        }
        for (; in != 0; in &= in - 1) {
          const int i = v * E + __builtin_ctz(in), place = atomicAdd(&l.count, 1);
          const float y = Elem<DT>::get(r.data, i);
          const uint32_t key = K::of(y);
          atomicMin(&l.least, key);
          atomicMax(&l.most, key);
          if (place < Lds<NT>::kList)
            l.list[place] = {(u64)key << 32 | ~(uint32_t)i, mass_of(weight(y, r.max, r.c), scale)};
        }
      });
      s = wave_sum(s);
      if (lane == 0) l.d[wave] = s;
      __syncthreads();
      double over = 0.0;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) over += l.d[w];
      u64 need = from;
      if (by_mass) {
        Z = block_sum<NT>(every, reinterpret_cast<double*>(l.q));
        whole_sum = true;
        need = (u64)fmax(ceil(p * Z * scale), 1.0);
      }
      if (l.count > Lds<NT>::kList || l.count == 0) return false;
      u64 sum = 0;
      from_list([&](uint32_t, uint32_t, u64 mass) { sum += by_mass ? mass : 1; });
      sum = block_sum<NT>(sum, l.q);
      const u64 so_far = by_mass ? (u64)(over * scale) : (u64)block_sum<NT>(n_over, l.i);
      if (so_far >= need || so_far + sum < need) return false;
      const Cut found = descend(l, l.least, l.most, need - so_far, [&](auto&& f) {
        from_list([&](uint32_t key, uint32_t, u64 mass) { f(key, by_mass ? mass : 1ull); });
      });
      const u64 rest = need - so_far - found.above;
      const u64 each = by_mass ? mass_of(weight(K::logit(found.key), r.max, r.c), scale) : 1;
      cut = found.key;
      ties = (int)min(each > 0 ? (rest + each - 1) / each : (u64)V, (u64)V);
      if (key_q > cut) {
        cut = key_q;
        ties = V;
      }
      // What the list adds to each stretch.
      __syncthreads();
      if (tid < kWaves) {
        l.q[tid] = 0;
        l.i[tid] = 0;
      }
      __syncthreads();
      from_list([&](uint32_t key, uint32_t late, u64 mass) {
        const int w = (int)(~late) / (r.steps * 64 * E);
        if (key > cut) atomicAdd(&l.q[w], mass);
        if (key == cut) atomicAdd(&l.i[w], 1);
      });
      __syncthreads();
      if (tid < kWaves) l.d[tid] += (double)l.q[tid] / scale;
      __syncthreads();
      return true;
    };
    const auto set_cut = [&](const Cut& found, u64 need) __attribute__((always_inline)) {
      const u64 each = mass_of(weight(K::logit(found.key), r.max, r.c), scale);
      const u64 rest = need > found.above ? need - found.above : 1;
      const u64 some = each > 0 ? (rest + each - 1) / each : (u64)V;
      if (found.key > cut || (found.key == cut && ties > 0)) {
        ties = found.key > cut ? (int)min(some, (u64)V) : min(ties, (int)min(some, (u64)V));
        cut = found.key;
      }
      return found.above + some * each;
    };
    if (probe && listed) {
      const Cut found = descend(l, K::kNegInf + 1, most, need_lo, [&](auto&& f) {
        from_list([&](uint32_t key, uint32_t, u64 mass) { f(key, mass); });
      });
      listed = settled = set_cut(found, need_lo) >= need_hi;  // else Z in 32 bits does not tell
    }
    // Tokens of less than (1 - p) Z / V each sum to less than (1 - p) Z: none of them is in the nucleus.
    const float low = probe ? fmaxf((float)((double)r.max + log2((1.0 - p) * Z * (1.0 - off) / V) / r.c), -3e38f) : 0.f;
    const float low_slack = fabsf(low) * 1e-5f + (r.max - low) * 1e-5f;
    const bool sure = probe && low > -3e38f;
    const uint32_t low_upper = sure ? K::upper(K::of(low - low_slack)) : 0;
    if (probe && !listed) {
      cut = K::kNegInf;
      ties = 0;
      summed = !how.odd && wide(true, need_lo, need_hi, low, low_upper, sure ? low - low_slack : -INFINITY);
    } else if (!listed && !how.odd && k < V && p >= 1.0 && tokens_at_all() > k) {
      summed = wide(false, (u64)k, (u64)k, r.max - 2.f * (r.max - least_top), 0, -INFINITY);
    }

    u64 kept_mass = 0;  // of the top-k tokens
    if (k < V && !summed) {
      Cut found = {K::kNegInf, 0};
      bool whole = false;
      if (listed) {
        whole = listed_n <= k;
        if (!whole)
          found = descend(l, K::kNegInf + 1, most, (u64)k, [&](auto&& f) {
            from_list([&](uint32_t key, uint32_t, u64) { f(key, 1ull); });
          });
      } else {
        whole = tokens_at_all() <= k;
        if (!whole) found = from_row(true, (u64)k, r.max - 2.f * (r.max - least_top), 0);
      }
      if (!whole) {
        cut = found.key;
        ties = k - (int)found.above;
      }
      if (p < 1.0) {
        u64 sum = 0;
        if (listed) {
          from_list([&](uint32_t key, uint32_t, u64 mass) { sum += key > cut ? mass : 0; });
        } else {
          r.template each<1>(l, K::upper(cut), [&](int, const float (&x)[E]) {
#pragma unroll
            for (int e = 0; e < E; ++e)
              if (K::of(x[e]) > cut) sum += mass_of(weight(x[e], r.max, r.c), scale);
          });
        }
        kept_mass = block_sum<NT>(sum, l.q);
        if (ties > 0) kept_mass += (u64)ties * mass_of(weight(K::logit(cut), r.max, r.c), scale);
      }
    }
    if (p < 1.0 && !summed && !settled) {
      if (probe && !whole_sum) {
        double s = 0.0;
        r.template each<1>(l, 0, [&](int, const float (&x)[E]) {
          double w[E];
          weights(x, r.max, r.c, w);
#pragma unroll
          for (int e = 0; e < E; ++e) s += w[e];
        });
        Z = block_sum<NT>(s, l.d);
      }
      const u64 need = (u64)fmax(ceil(p * (k < V ? (double)kept_mass : Z * scale)), 1.0);
      if (listed) {
        set_cut(descend(l, K::kNegInf + 1, most, need, [&](auto&& f) {
          from_list([&](uint32_t key, uint32_t, u64 mass) { f(key, mass); });
        }), need);
      } else {
        set_cut(from_row(false, need, probe ? low : r.max - 2.f * (r.max - least_top), low_upper), need);
      }
    }
    if (key_q > cut && !summed) {
      cut = key_q;
      ties = V;
    }

    // ---- the token, where all that may be kept fits into a list
    if (!listed && !summed)
      listed = gather(l, r, max(cut, K::kNegInf + 1), scale);
    if (listed) {
      int equal = 0;
      from_list([&](uint32_t key, uint32_t, u64) { equal += key == cut ? 1 : 0; });
      equal = block_sum<NT>(equal, l.i);
      // Indices count from the end, so that the lowest come first from the top.
      uint32_t last_tie = 0;
      if (ties > 0 && ties < equal)
        last_tie = descend(l, ~(uint32_t)(V - 1), ~0u, (u64)ties, [&](auto&& f) {
          from_list([&](uint32_t key, uint32_t late, u64) {
            if (key == cut) f(late, 1ull);
          });
        }).key;
      const auto kept = [&](auto&& f) __attribute__((always_inline)) {
        from_list([&](uint32_t key, uint32_t late, u64 mass) {
          if (key > cut || (key == cut && ties > 0 && late >= last_tie)) f(late, mass);
        });
      };
      u64 sum = 0;
      kept([&](uint32_t, u64 mass) { sum += mass; });
      sum = block_sum<NT>(sum, l.q);
      const u64 need = min((u64)floor(part * (double)sum) + 1, sum);
      const uint32_t at = descend(l, ~(uint32_t)(V - 1), ~0u, need, kept).key;
      if (tid == 0) finish((int)~at, (double)sum / scale);
      return;
    }
  }

  // ---- the token from the row: the kept weight of every wave's stretch, then
  // the stretch that the border lies in.
  const uint32_t upper = K::upper(cut);
  const double w_cut = ties > 0 ? weight(K::logit(cut), r.max, r.c) : 0.0;
  const auto held = [&](double mass, int count) __attribute__((always_inline)) { return mass + w_cut * (double)min(count, ties); };
  const auto add = [&](float x, double& s, int& t) __attribute__((always_inline)) {
    const uint32_t key = K::of(x);
    if (key > cut) s += weight(x, r.max, r.c);
    if (key == cut) ++t;
  };
  if (!summed) {
    double s = 0.0;
    int t = 0;
    r.template each<1>(l, upper, [&](int, const float (&x)[E]) {
#pragma unroll
      for (int e = 0; e < E; ++e) add(x[e], s, t);
    });
    s = wave_sum(s);
    t = wave_sum(t);
    __syncthreads();
    if (lane == 0) {
      l.d[wave] = s;
      l.i[wave] = t;
    }
  }
  __syncthreads();
  // Every wave finds the stretch, its lanes w < kWaves holding the sums up to stretch w.
  const double own_w = lane < kWaves ? l.d[lane] : 0.0;
  const int own_t = lane < kWaves ? l.i[lane] : 0;
  double upto_w = own_w;
  int ties_w = own_t;
#pragma unroll
  for (int o = 1; o < kWaves; o <<= 1) {
    const double us = __shfl_up(upto_w, o);
    const int ut = __shfl_up(ties_w, o);
    if (lane >= o) {
      upto_w += us;
      ties_w += ut;
    }
  }
  const double total = held(__shfl(upto_w, kWaves - 1), __shfl(ties_w, kWaves - 1)), target = part * total;
  // Running sums that are added in different orders differ by roundings, also between two
  // neighbours of which the second keeps nothing. So the border is looked for where
  // something is added (here, and among vectors and tokens below), and lies in the last
  // of those where no sum passes the target.
  const bool adds_w = own_w > kLeastSum || (own_t > 0 && ties_w - own_t < ties && w_cut > 0.0);
  const u64 adding = __ballot(adds_w), crossed = __ballot(adds_w && held(upto_w, ties_w) > target);
  const int where = crossed != 0 ? __builtin_ctzll(crossed) : 63 - __builtin_clzll(adding);
  double before = where > 0 ? __shfl(upto_w, max(where - 1, 0)) : 0.0;
  int tie_before = where > 0 ? __shfl(ties_w, max(where - 1, 0)) : 0;
  const int base = where * r.steps * 64, vectors = r.steps * 64;
  int spare_v = -1, spare_t = 0;
  double spare_s = 0.0;
  // The first kept token of a vector that passes the limit, or its last one.
  const auto walk = [&](int v, double ms, int mt, double limit) __attribute__((always_inline)) {
    float x[E];
    unpack<DT>(load_vec<DT>(r.data, v, V), x);
    int found = -1, last = -1;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      double own = 0.0;
      const int before_t = mt;
      add(x[e], own, mt);
      ms += own;
      if (!(own > 0.0 || (mt > before_t && before_t < ties && w_cut > 0.0))) continue;
      last = v * E + e;
      if (held(ms, mt) > limit && found < 0) found = last;
    }
    return found >= 0 ? found : last;
  };
  __syncthreads();
  if (tid == 0) {
    l.first = kNoCrossing;
    l.spare = -1;
  }
  for (int i0 = 0; i0 < vectors; i0 += NT) {
    const int v = base + i0 + tid;
    double s = 0.0;
    int t = 0;
    if (i0 + tid < vectors && v * E < V) {
      float x[E];
      unpack<DT>(load_vec<DT>(r.data, v, V), x);
#pragma unroll
      for (int e = 0; e < E; ++e)
        add(x[e], s, t);
    }
    double upto = s;
    int upto_t = t;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const double us = __shfl_up(upto, o);
      const int ut = __shfl_up(upto_t, o);
      if (lane >= o) {
        upto += us;
        upto_t += ut;
      }
    }
    __syncthreads();
    if (lane == 63) {
      l.d[wave] = upto;
      l.i[wave] = upto_t;
    }
    __syncthreads();
    double round = 0.0;
    int round_t = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      if (w == wave) {
        upto += before + round;
        upto_t += tie_before + round_t;
      }
      round += l.d[w];
      round_t += l.i[w];
    }
    const double from = upto - s;
    const int from_t = upto_t - t;
    const bool adds = s > 0.0 || (t > 0 && from_t < ties && w_cut > 0.0);
    if (adds) {
      spare_v = v;
      spare_s = from;
      spare_t = from_t;
    }
    const bool over = adds && held(upto, upto_t) > target;
    if (over) atomicMin(&l.first, v);
    __syncthreads();
    if (l.first != kNoCrossing) {
      if (l.first == v) finish(walk(v, from, from_t, target), total);
      return;
    }
    before += round;
    tie_before += round_t;
  }
  if (spare_v >= 0) atomicMax(&l.spare, spare_v);
  __syncthreads();
  if (spare_v >= 0 && l.spare == spare_v) finish(walk(spare_v, spare_s, spare_t, INFINITY), total);
}

// Whether rows are scanned by workgroups of their own: where the second launch costs
// less than the units that one workgroup a row leaves idle (all tokens kept of 1, 64,
// 128, 192 rows of 128000 bf16 logits: 39, 39, 40, 40 us with a workgroup each, 21, 28,
// 37, 45 split; of 1, 64, 128 rows of 40000: 20, 21, 22 us, 20, 22, 27 split).
bool sample_splits(int rows, int vocab, int per_vec) {
  const int vectors = cdiv(vocab, per_vec);
  return vectors > 6144 && rows <= vectors / 112;
}

template <int DT>
void launch(const SampleArgs& a, hipStream_t stream) {
  const dim3 grid(a.logits.rows);
  const int vectors = cdiv(a.logits.vocab, Elem<DT>::kPerVec);
  if (sample_splits(a.logits.rows, a.logits.vocab, Elem<DT>::kPerVec)) {
    scan_kernel<DT><<<dim3(a.logits.rows * kSplit), dim3(kScanThreads), 0, stream>>>(a);
    sample_kernel<DT, kSplitThreads, true><<<grid, dim3(kSplitThreads), 0, stream>>>(a);
    return;
  }
  // Most of a short row's time goes to reductions and barriers, fewer with fewer waves,
  // and four workgroups to a unit fill each other's waits; longer rows want more loads
  // and weights at once. Mixed filters, bf16, 256 / 512 / 1024 threads, in us:
  //   600 x 2000: 21, 27, 49; 300 x 8000: 22, 20, 32; 2000 x 8000: 45, 62, 124;
  //   256 x 32000: 34, 26, 30; 1000 x 32000: 55, 51, 78; 2000 x 32000: 74, 85, 152;
  //   512 x 64000: -, 63, 73; 256 x 151936: -, 107, 100; 1024 x 151936: 263, 157, 202.
  const int rows = a.logits.rows, cus = a.logits.num_cus;
  if (vectors <= 512 || (vectors <= 4096 && rows > (vectors <= 2048 ? 2 : 4) * cus))
    sample_kernel<DT, 256, false><<<grid, dim3(256), 0, stream>>>(a);
  else if (vectors <= 10240 || rows > cus)
    sample_kernel<DT, 512, false><<<grid, dim3(512), 0, stream>>>(a);
  else
    sample_kernel<DT, 1024, false><<<grid, dim3(1024), 0, stream>>>(a);
}

}  // namespace

size_t sample_workspace(int rows, int vocab, int dtype) {
  return sample_splits(rows, vocab, dtype == RP_LOGITS_F32 ? 4 : 8) ? sizeof(SplitRow) * (size_t)rows : 0;
}

hipError_t launch_sample(const SampleArgs& a, int dtype, hipStream_t stream) {
  switch (dtype) {
    case RP_LOGITS_BF16: launch<RP_LOGITS_BF16>(a, stream); break;
    case RP_LOGITS_F16: launch<RP_LOGITS_F16>(a, stream); break;
    default: launch<RP_LOGITS_F32>(a, stream); break;
  }
  return hipGetLastError();
}

}  // namespace rp
