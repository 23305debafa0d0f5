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
// slices of the keys, and of the indices. Longer lists are found the same way
// from the row itself.
#include "rp_rows.h"

namespace rp {
namespace {

typedef unsigned long long u64;
constexpr int kBins = 1024;
constexpr int kNoCrossing = 0x7FFFFFFF;

template <int NT>
struct Lds {
  static constexpr int kWaves = NT / 64;
  static constexpr int kEntries = NT == 256 ? 16 : 32;  // largest keys kept per thread
  static constexpr int kList = 2 * NT;
  float f[kWaves];
  double d[kWaves];
  int i[kWaves];
  u64 q[kWaves];
  u64 hist[kBins];
  u64 mass[kList];
  uint32_t key[kList], index[kList], work[kList];
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
// In steps of 2^-S, scale = 2^S <= 2^50.
__device__ inline u64 mass_of(double w, double scale) {
  return (u64)__double_as_longlong(fma(w, scale, 0x1p52)) & ((1ull << 52) - 1);
}

// The row, and which vectors of it a thread has: wave w has the stretch of
// `steps` * 64 vectors from w * steps * 64 on, in the order of indices.
template <int DT, int NT>
struct Row {
  static constexpr int E = Elem<DT>::kPerVec;
  const void* data;
  int vocab, steps, shift;  // vectors j >> shift of a thread share an entry of lds.top
  float max;
  double c;
  __device__ inline int vec(int thread, int j) const { return (thread / 64 * steps + j) * 64 + thread % 64; }
  // f(vector, its logits) for this thread's vectors whose largest key is `upper` or more.
  template <class F>
  __device__ inline void each(const Lds<NT>& l, uint32_t upper, const F& f) const {
    constexpr int U = 4;
    for (int j0 = 0; j0 < steps; j0 += U) {
      u32x4_any q[U];
      bool has[U];
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const int j = j0 + k, v = vec(threadIdx.x, j);
        has[k] = j < steps && v * E < vocab && l.top[(j >> shift) * NT + threadIdx.x] >= upper;
        if (has[k]) q[k] = load_vec<DT>(data, v, vocab);
      }
#pragma unroll
      for (int k = 0; k < U; ++k) {
        if (!has[k]) continue;
        float x[E];
        unpack<DT>(q[k], x);
        f(vec(threadIdx.x, j0 + k), x);
      }
    }
  }
};

// The place, from the top of lds.hist, where the sums reach `need` (at most all
// of it): its bin, and the sum above.
template <int NT>
__device__ inline int find_top(Lds<NT>& l, u64 need, u64& above) {
  constexpr int PER = kBins / NT;
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  u64 h[PER], sum = 0;
#pragma unroll
  for (int k = 0; k < PER; ++k) sum += h[k] = l.hist[kBins - 1 - (tid * PER + k)];
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
        l.bin = kBins - 1 - (tid * PER + k);
        l.above = run;
      }
      run += h[k];
    }
  }
  __syncthreads();
  above = l.above;
  return l.bin;
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
__device__ inline Cut descend(Lds<NT>& l, uint32_t lo, uint32_t hi, u64 need, const Items& items) {
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
    u64 above;
    const uint32_t bin = (uint32_t)find_top(l, need, above);
    need -= above < need ? above : need;
    over += above;
    lo += bin << s;
    if (s == 0) return {lo, over};
    width = min(width - (bin << s), (1u << s) - 1);
  }
}

// Lists the tokens that `keep` takes, from vectors whose largest key is `upper` or more; whether they fit.
template <int DT, int NT, class Keep>
__device__ inline bool gather(Lds<NT>& l, const Row<DT, NT>& r, uint32_t upper, double scale, const Keep& keep) {
  constexpr int E = Elem<DT>::kPerVec;
  const int tid = threadIdx.x, entries = cdiv(r.steps, 1 << r.shift);
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
      if (!keep(x[k], key)) continue;
      const int at = atomicAdd(&l.count, 1);
      if (at >= Lds<NT>::kList) continue;
      l.key[at] = key;
      l.index[at] = v * E + k;
      l.mass[at] = mass_of(weight(x[k], r.max, r.c), scale);
    }
  }
  __syncthreads();
  return l.count <= Lds<NT>::kList;
}

template <int DT, int NT>
__global__ __launch_bounds__(NT) void sample_kernel(const SampleArgs a) {
  __shared__ Lds<NT> l;
  typedef Key<DT> K;
  constexpr int E = Elem<DT>::kPerVec, kWaves = Lds<NT>::kWaves;
  const int n = blockIdx.x, V = a.logits.vocab, tid = threadIdx.x, wave = tid / 64, lane = tid % 64;
  Row<DT, NT> r;
  r.data = static_cast<const char*>(a.logits.data) + (long long)n * a.logits.stride * Elem<DT>::kBytes;
  r.vocab = V;
  r.steps = cdiv(cdiv(V, E), NT);
  r.shift = 0;
  while (cdiv(r.steps, 1 << r.shift) > Lds<NT>::kEntries) ++r.shift;

  // Greedy is top-1 at T = 1. c stays above 0, so that -inf weighs nothing at T = inf too.
  float T = a.temperature != nullptr ? a.temperature[n] : 1.f;
  const bool greedy = !(T > 0.f);
  const int asked_k = greedy ? 1 : a.top_k != nullptr ? a.top_k[n] : 0;
  const int k = asked_k > 0 && asked_k < V ? asked_k : V;
  const float asked_p = greedy || a.top_p == nullptr ? 1.f : a.top_p[n];
  const double p = asked_p < 1.f ? fmax((double)asked_p, 0.0) : 1.0;
  const float asked_q = greedy || a.min_p == nullptr ? 0.f : a.min_p[n];
  const double q = asked_q > 0.f ? fmin((double)asked_q, 1.0) : 0.0;
  const double inv_t = greedy ? 1.0 : fmax(1.0 / (double)T, 1e-300);
  r.c = kLog2e64 * inv_t;
  const float c32 = (float)fmin(r.c, 3e38);
  const bool light_k = k < V && k <= NT / 2;
  const bool all = k >= V && p >= 1.0 && q == 0.0;
  const bool exact = k >= V && (p < 1.0 || q == 0.0);

  // ---- the row's maximum, its sum and the vectors' largest keys
  // In 32 bits: sums of the vector with the thread's largest logit, and of the others.
  float top = -INFINITY, ref = -INFINITY, group = 0.f, rest = 0.f;
  double s64 = 0.0;
  int at_top = -1;
  bool bad = false;
  for (int g = 0; g < Lds<NT>::kEntries; ++g) l.top[g * NT + tid] = 0;
  {
    constexpr int U = 4;
    u32x4_any next[U];
    const auto fetch = [&](int j0) {
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int v = r.vec(tid, j0 + i);
        if (j0 + i < r.steps && v * E < V) next[i] = load_vec<DT>(r.data, v, V);
      }
    };
    fetch(0);
    for (int j0 = 0; j0 < r.steps; j0 += U) {
      u32x4_any now[U];
#pragma unroll
      for (int i = 0; i < U; ++i) now[i] = next[i];
      fetch(j0 + U);
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int j = j0 + i;
        if (j >= r.steps || r.vec(tid, j) * E >= V) continue;
        float x[E];
        unpack<DT>(now[i], x);
        float most = x[0];
#pragma unroll
        for (int e = 0; e < E; ++e) {
          most = fmaxf(most, x[e]);
          bad = bad || !(x[e] < INFINITY);
        }
        if (!(most > -INFINITY)) continue;
        const uint16_t entry = (uint16_t)K::upper(K::of(most));
        uint16_t& slot = l.top[(j >> r.shift) * NT + tid];
        slot = max(slot, entry);
        if (exact) {
          // The reference moves when a weight would pass 2^256, which 64 bits hold.
          if (!((double)(most - ref) * r.c < 256.0)) {
            s64 *= weight(ref, most, r.c);
            ref = most;
          }
          double s = 0.0;
#pragma unroll
          for (int e = 0; e < E; ++e) s += weight(x[e], ref, r.c);
          s64 += s;
        } else {
          const bool more = most > top;
          if (more) {
            rest = (rest + group) * fast_exp2((top - most) * c32);
            ref = most;
            at_top = r.vec(tid, j);
          }
          float s = 0.f;
#pragma unroll
          for (int e = 0; e < E; ++e) s += fast_exp2((x[e] - ref) * c32);
          if (more) group = s;
          else rest += s;
        }
        top = fmaxf(top, most);
      }
    }
  }
  r.max = block_max<NT>(top, l.f);
  bad = __syncthreads_or(bad);
  if (bad || r.max == -INFINITY) {
    if (tid == 0) {
      const float none = bad ? NAN : -INFINITY;
      a.tokens[n] = -1;
      if (a.logprobs != nullptr) a.logprobs[n] = none;
      if (a.kept != nullptr) a.kept[n] = none;
    }
    return;
  }
  if (exact) {
    if (ref > -INFINITY) s64 *= weight(ref, r.max, r.c);
  } else {
    // The vector with the row's maximum again, in 64 bits: where one token has nearly
    // all the mass, ln Z is that of the rest.
    if (top == r.max) {
      float x[E];
      unpack<DT>(load_vec<DT>(r.data, at_top, V), x);
      s64 = (double)rest;
#pragma unroll
      for (int e = 0; e < E; ++e) s64 += (double)fast_exp2((x[e] - top) * c32);
    } else if (ref > -INFINITY) {
      s64 = (double)((rest + group) * fast_exp2((ref - r.max) * c32));
    }
  }
  const double wave_part = wave_sum(s64);
  __syncthreads();
  if (lane == 0) l.d[wave] = wave_part;
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

  const auto finish = [&](int token, double total) {
    const double z = ((double)Elem<DT>::get(r.data, max(token, 0)) - (double)r.max) * inv_t;
    a.tokens[n] = token;
    if (a.logprobs != nullptr) a.logprobs[n] = (float)(z - log(Z));
    if (a.kept != nullptr) a.kept[n] = (float)(z - log(total));
  };

  uint32_t cut = K::kNegInf;  // keys above it are kept, and the first `ties` at it
  int ties = 0;
  bool listed = false;
  if (!all) {
    // A key that `want` threads' largest ones, and so as many tokens, reach.
    const float least_top = -block_max<NT>(top > -INFINITY ? -top : -INFINITY, l.f);
    const auto reached = [&](int want) {
      const float fit = fmaxf(fminf(r.max - least_top, 1e30f), 1e-30f);
      const int bin = kBins - 1 - (int)fminf((r.max - top) * ((kBins - 2) / fit), kBins - 1.f);
      const bool has = top > -INFINITY;
      __syncthreads();
      clear<NT>(l.hist);
      if (tid == 0) l.least = 0xFFFFFFFFu;
      __syncthreads();
      if (has) atomicAdd(&l.hist[bin], 1ull);
      const int threads = __syncthreads_count(has);
      if (threads < want) return K::kNegInf + 1;
      u64 above;
      const int at = find_top(l, (u64)want, above);
      if (has && bin >= at) atomicMin(&l.least, K::of(top));
      __syncthreads();
      return l.least;
    };
    const auto from_list = [&](auto&& f) {
      const int count = l.count;
      for (int i = tid; i < count; i += NT) f(l.key[i], l.index[i], l.mass[i]);
    };
    const uint32_t most = K::of(r.max);
    const bool probe = k >= V && p < 1.0;
    if (light_k || probe) {
      const uint32_t tau = reached(light_k ? k : NT / 2);
      listed = gather<DT, NT>(l, r, K::upper(tau), scale, [&](float, uint32_t key) { return key >= tau; });
    }
    const int listed_n = l.count;

    // The key at which the tokens' masses (their number, where `count`) reach
    // `need`, from the row itself: by equal steps of the logits down to `low`,
    // then within one of those.
    const auto from_row = [&](bool count, u64 need, float low, uint32_t upper) {
      const float fit = fmaxf(fminf(r.max - low, 1e30f), 1e-30f), per = (kBins - 2) / fit;
      const auto step = [&](float x) { return kBins - 1 - (int)fminf((r.max - x) * per, kBins - 1.f); };
      const auto one = [&](float x) { return count ? 1ull : mass_of(weight(x, r.max, r.c), scale); };
      __syncthreads();
      clear<NT>(l.hist);
      if (tid == 0) {
        l.least = 0xFFFFFFFFu;
        l.most = 0;
      }
      __syncthreads();
      r.each(l, upper, [&](int, const float (&x)[E]) {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (x[e] > -INFINITY) atomicAdd(&l.hist[step(x[e])], one(x[e]));
      });
      __syncthreads();
      u64 above;
      const int at = find_top(l, need, above);
      need -= above < need ? above : need;
      // Every key of that step, and a threshold for the vectors that hold them.
      const float edge = at == 0 ? -INFINITY : r.max - (float)(kBins - at) / per;
      const float slack = at == 0 ? 0.f : fabsf(edge) * 1e-5f + fit * 1e-4f;
      const uint32_t edge_upper = max(upper, at == 0 ? 0u : K::upper(K::of(edge - slack)));
      const bool fits = gather<DT, NT>(l, r, edge_upper, scale, [&](float x, uint32_t key) {
        const bool in = x > -INFINITY && step(x) == at;
        if (in) {
          atomicMin(&l.least, key);
          atomicMax(&l.most, key);
        }
        return in;
      });
      Cut found;
      if (fits) {
        found = descend(l, l.least, l.most, need, [&](auto&& f) {
          from_list([&](uint32_t key, uint32_t, u64 mass) { f(key, count ? 1ull : mass); });
        });
      } else {
        __syncthreads();
        if (tid == 0) {
          l.least = 0xFFFFFFFFu;
          l.most = 0;
        }
        __syncthreads();
        uint32_t lo = 0xFFFFFFFFu, hi = 0;
        r.each(l, edge_upper, [&](int, const float (&x)[E]) {
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
        found = descend(l, lo, hi, need, [&](auto&& f) {
          r.each(l, edge_upper, [&](int, const float (&x)[E]) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
              const uint32_t key = K::of(x[e]);
              if (key >= lo && key <= hi) f(key, one(x[e]));
            }
          });
        });
      }
      found.above += above;
      return found;
    };

    u64 kept_mass = 0;  // of the top-k tokens
    if (k < V) {
      Cut found = {K::kNegInf, 0};
      bool whole = false;
      if (listed) {
        whole = listed_n <= k;
        if (!whole)
          found = descend(l, K::kNegInf + 1, most, (u64)k, [&](auto&& f) {
            from_list([&](uint32_t key, uint32_t, u64) { f(key, 1ull); });
          });
      } else {
        int finite = 0;
        r.each(l, 0, [&](int, const float (&x)[E]) {
#pragma unroll
          for (int e = 0; e < E; ++e) finite += x[e] > -INFINITY ? 1 : 0;
        });
        whole = block_sum<NT>(finite, l.i) <= k;
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
          r.each(l, K::upper(cut), [&](int, const float (&x)[E]) {
#pragma unroll
            for (int e = 0; e < E; ++e)
              if (K::of(x[e]) > cut) sum += mass_of(weight(x[e], r.max, r.c), scale);
          });
        }
        kept_mass = block_sum<NT>(sum, l.q);
        if (ties > 0) kept_mass += (u64)ties * mass_of(weight(K::logit(cut), r.max, r.c), scale);
      }
    }
    if (p < 1.0) {
      const double want = p * (k < V ? (double)kept_mass : Z * scale);
      const u64 need = (u64)fmax(ceil(want), 1.0);
      bool enough = listed;
      if (probe && listed) {
        u64 sum = 0;
        from_list([&](uint32_t, uint32_t, u64 mass) { sum += mass; });
        enough = block_sum<NT>(sum, l.q) >= need;
      }
      Cut found;
      if (enough) {
        found = descend(l, K::kNegInf + 1, most, need, [&](auto&& f) {
          from_list([&](uint32_t key, uint32_t, u64 mass) { f(key, mass); });
        });
      } else {
        // Tokens of less than (1 - p) Z / V each sum to less than (1 - p) Z: none of them is in the nucleus.
        const float low = (float)((double)r.max + log2((1.0 - p) * Z / V) / r.c);
        const float slack = fabsf(low) * 1e-5f + (r.max - low) * 1e-5f;
        const bool sure = probe && low > -3e38f;
        found = from_row(false, need, fmaxf(low, -3e38f), sure ? K::upper(K::of(low - slack)) : 0);
        listed = false;
      }
      const u64 each = mass_of(weight(K::logit(found.key), r.max, r.c), scale);
      const u64 rest = need > found.above ? need - found.above : 1;
      const u64 some = each > 0 ? (rest + each - 1) / each : (u64)V;
      if (found.key > cut || (found.key == cut && ties > 0)) {
        ties = found.key > cut ? (int)min(some, (u64)V) : min(ties, (int)min(some, (u64)V));
        cut = found.key;
      }
    }
    if (q > 0.0) {
      // The least logit of weight q or more.
      const double least = (double)r.max + log2(q) / r.c;
      float x = (float)least;
      uint32_t key = K::of(x);
      if (!((double)K::logit(key) >= least)) ++key;
      key = min(key, most);
      if (key > cut) {
        cut = key;
        ties = V;
      }
    }

    // ---- the token, where all that may be kept fits into a list
    if (!listed)
      listed = gather<DT, NT>(l, r, K::upper(cut), scale, [&](float x, uint32_t key) {
        return key >= cut && x > -INFINITY;
      });
    if (listed) {
      int equal = 0;
      from_list([&](uint32_t key, uint32_t, u64) { equal += key == cut ? 1 : 0; });
      equal = block_sum<NT>(equal, l.i);
      // Indices count from the end, so that the lowest come first from the top.
      uint32_t last_tie = 0;
      if (ties > 0 && ties < equal)
        last_tie = descend(l, ~(uint32_t)(V - 1), ~0u, (u64)ties, [&](auto&& f) {
          from_list([&](uint32_t key, uint32_t index, u64) {
            if (key == cut) f(~index, 1ull);
          });
        }).key;
      const auto kept = [&](auto&& f) {
        from_list([&](uint32_t key, uint32_t index, u64 mass) {
          if (key > cut || (key == cut && ties > 0 && ~index >= last_tie)) f(~index, mass);
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
  const auto held = [&](double mass, int count) { return mass + w_cut * (double)min(count, ties); };
  const auto add = [&](float x, double& s, int& t) {
    const uint32_t key = K::of(x);
    if (key > cut) s += weight(x, r.max, r.c);
    if (key == cut) ++t;
  };
  if (!all) {
    double s = 0.0;
    int t = 0;
    r.each(l, upper, [&](int, const float (&x)[E]) {
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
    __syncthreads();
  } else if (lane == 0) {
    l.i[wave] = 0;
  }
  __syncthreads();
  double before = 0.0, total_mass = 0.0;
  int tie_before = 0, total_ties = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    total_mass += l.d[w];
    total_ties += l.i[w];
  }
  const double total = held(total_mass, total_ties), target = part * total;
  int where = 0;
  for (; where < kWaves - 1 && !(held(before + l.d[where], tie_before + l.i[where]) > target); ++where) {
    before += l.d[where];
    tie_before += l.i[where];
  }
  // Sums in another order may miss the crossing by a rounding; then it is the stretch's last kept token.
  const int base = where * r.steps * 64, vectors = r.steps * 64;
  int spare_v = -1, spare_t = 0;
  double spare_s = 0.0;
  const auto walk = [&](int v, double ms, int mt, double limit) {
    int found = -1, last = -1;
    double at = held(ms, mt);
    for (int e = 0; e < E && v * E + e < V; ++e) {
      add(Elem<DT>::get(r.data, v * E + e), ms, mt);
      if (held(ms, mt) > limit && found < 0) found = v * E + e;
      if (held(ms, mt) > at) last = v * E + e;
      at = held(ms, mt);
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
        if (v * E + e < V) add(x[e], s, t);
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
    if (held(from + s, upto_t) > held(from, from_t)) {
      spare_v = v;
      spare_s = from;
      spare_t = from_t;
    }
    const bool over = held(upto, upto_t) > target;
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

template <int DT>
void launch(const SampleArgs& a, hipStream_t stream) {
  const int vectors = cdiv(a.logits.vocab, Elem<DT>::kPerVec);
  const dim3 grid(a.logits.rows);
  if (vectors <= 4096) sample_kernel<DT, 256><<<grid, dim3(256), 0, stream>>>(a);
  else if (vectors <= 16384) sample_kernel<DT, 512><<<grid, dim3(512), 0, stream>>>(a);
  else sample_kernel<DT, 1024><<<grid, dim3(1024), 0, stream>>>(a);
}

}  // namespace

hipError_t launch_sample(const SampleArgs& a, int dtype, hipStream_t stream) {
  switch (dtype) {
    case RP_LOGITS_BF16: launch<RP_LOGITS_BF16>(a, stream); break;
    case RP_LOGITS_F16: launch<RP_LOGITS_F16>(a, stream); break;
    default: launch<RP_LOGITS_F32>(a, stream); break;
  }
  return hipGetLastError();
}

}  // namespace rp
