// Sampling from rows of logits with temperature, top-k, top-p and min-p: one
// workgroup per row.
//
// In the order of falling logits (the lowest index first among equals) the
// kept tokens are a prefix, so they are described by a cut: every token whose
// logit is above the cut's, and the first `ties` tokens, by index, at it. The
// prefix sums that decide (top-p's mass, the border that the random number
// falls on) are of weights 2^((x - max) log2(e) / T) in 64 bits: a border may
// be any of 10^5 tokens, and 32 bits would move it past some of them.
#include "rp_rows.h"

namespace rp {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;

// Order of logits as unsigned numbers, -0 and 0 the same.
__device__ inline uint32_t order_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ inline float logit_of(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o); }

struct Shared {
  float f[kWaves];
  double d[kWaves];
  int i[kWaves];
};

struct Row {
  const void* data;
  int vocab;
  float max;
  double c;  // log2(e) / T
};

__device__ inline double weight(float x, const Row& r) {
  return x > -INFINITY ? exp2(((double)x - (double)r.max) * r.c) : 0.0;
}

// Tokens at or above a place of the order, and their weight, over the row.
template <int DT>
__device__ void at_or_above(const Row& r, uint32_t place, Shared& lds, int& count, double& mass) {
  int n = 0;
  double s = 0.0;
  for (int v = threadIdx.x; v * Elem<DT>::kPerVec < r.vocab; v += kThreads) {
    float x[Elem<DT>::kPerVec];
    unpack<DT>(load_vec<DT>(r.data, v, r.vocab), x);
#pragma unroll
    for (int k = 0; k < Elem<DT>::kPerVec; ++k) {
      if (order_of(x[k]) < place || v * Elem<DT>::kPerVec + k >= r.vocab) continue;
      ++n;
      s += weight(x[k], r);
    }
  }
  count = block_sum<kThreads>(n, lds.i);
  mass = block_sum<kThreads>(s, lds.d);
}

template <int DT>
__global__ __launch_bounds__(kThreads) void sample_kernel(const SampleArgs a) {
  __shared__ Shared lds;
  constexpr int E = Elem<DT>::kPerVec;
  const int n = blockIdx.x, V = a.logits.vocab, tid = threadIdx.x;
  const void* row = static_cast<const char*>(a.logits.data) + (long long)n * a.logits.stride * Elem<DT>::kBytes;
  float top = -INFINITY;
  bool bad = false;
  for (int v = tid; v * E < V; v += kThreads) {
    float x[E];
    unpack<DT>(load_vec<DT>(row, v, V), x);
#pragma unroll
    for (int k = 0; k < E; ++k) {
      top = fmaxf(top, x[k]);
      bad = bad || !(x[k] < INFINITY);
    }
  }
  top = block_max<kThreads>(top, lds.f);
  bad = __syncthreads_or(bad);
  if (bad || top == -INFINITY) {
    if (tid == 0) {
      const float none = bad ? NAN : -INFINITY;
      a.tokens[n] = -1;
      if (a.logprobs != nullptr) a.logprobs[n] = none;
      if (a.kept != nullptr) a.kept[n] = none;
    }
    return;
  }
  const float T = a.temperature != nullptr ? a.temperature[n] : 1.f;
  const bool greedy = !(T > 0.f);
  const Row r = {row, V, top, greedy ? kLog2e64 : kLog2e64 / (double)T};
  int all;
  double whole;
  at_or_above<DT>(r, 0, lds, all, whole);

  // The cut.
  uint32_t cut = 0;
  int ties = V;
  if (greedy) {
    cut = order_of(top);
    ties = 1;
  } else {
    const int k = a.top_k != nullptr && a.top_k[n] > 0 ? a.top_k[n] : V;
    if (k < V) {
      // The largest place with k tokens at or above it.
      for (int bit = 31; bit >= 0; --bit) {
        int count;
        double mass;
        at_or_above<DT>(r, cut | 1u << bit, lds, count, mass);
        if (count >= k) cut |= 1u << bit;
      }
      int above;
      double mass;
      at_or_above<DT>(r, cut + 1, lds, above, mass);
      ties = k - above;
    }
    const float p = a.top_p != nullptr ? a.top_p[n] : 1.f;
    if (p < 1.f) {
      int count;
      double mass, left = whole;
      if (k < V) {
        at_or_above<DT>(r, cut + 1, lds, count, left);
        left += ties * weight(logit_of(cut), r);
      }
      const double want = fmax((double)p, 0.0) * left;
      uint32_t place = 0;
      for (int bit = 31; bit >= 0; --bit) {
        at_or_above<DT>(r, place | 1u << bit, lds, count, mass);
        if (mass >= want && count > 0) place |= 1u << bit;
      }
      if (place >= cut) {
        at_or_above<DT>(r, place + 1, lds, count, mass);
        const double need = ceil((want - mass) / weight(logit_of(place), r));
        const int some = need > 1.0 ? (int)fmin(need, (double)V) : 1;
        ties = place > cut ? some : min(ties, some);
        cut = place;
      }
    }
    const float asked = a.min_p != nullptr ? a.min_p[n] : 0.f;
    if (asked > 0.f) {
      const float q = fminf(asked, 1.f);
      // Least logit with weight >= q.
      const double least = (double)top + log2((double)q) / r.c;
      float x = (float)least;
      if ((double)x < least) x = logit_of(order_of(x) + 1);
      const uint32_t place = min(order_of(x), order_of(top));
      if (place > cut) {
        cut = place;
        ties = V;
      }
    }
  }
  const double w_cut = cut > order_of(-INFINITY) ? weight(logit_of(cut), r) : 0.0;

  // Kept weight of each wave's stretch of the row, in the order of indices.
  const int wave = tid / 64, lane = tid % 64;
  const int steps = cdiv(cdiv(V, E), kThreads), first = wave * steps * 64;
  const auto lane_part = [&](int v, double& s, int& t) {
    s = 0.0;
    t = 0;
    if (v * E >= V) return;
    float x[E];
    unpack<DT>(load_vec<DT>(row, v, V), x);
    for (int k = 0; k < E; ++k) {
      if (v * E + k >= V) break;
      const uint32_t o = order_of(x[k]);
      if (o > cut) s += weight(x[k], r);
      if (o == cut) ++t;
    }
  };
  double s = 0.0;
  int t = 0;
  for (int i = 0; i < steps; ++i) {
    double si;
    int ti;
    lane_part(first + i * 64 + lane, si, ti);
    s += si;
    t += ti;
  }
  s = wave_sum(s);
  t = wave_sum(t);
  __syncthreads();
  if (lane == 0) {
    lds.d[wave] = s;
    lds.i[wave] = t;
  }
  __syncthreads();
  double kept = 0.0, before = 0.0;
  int tie = 0, tie_before = 0;
  const auto held = [&](double mass, int count) { return mass + w_cut * (double)min(count, ties); };
  for (int w = 0; w < kWaves; ++w) {
    if (w == wave) {
      before = kept;
      tie_before = tie;
    }
    kept += lds.d[w];
    tie += lds.i[w];
  }
  const double total = held(kept, tie);
  float u = a.u[n];
  if (!(u >= 0.f)) u = 0.f;
  const double target = (double)fminf(u, 0x1.fffffep-1f) * total;
  // One wave's stretch has the border: its first crossing is the token. Sums in
  // another order may miss it by a rounding; then it is the stretch's last token.
  if (held(before, tie_before) > target || !(held(before + s, tie_before + t) > target)) return;
  const auto walk = [&](int v, double ms, int mt) {
    double at = held(ms, mt);
    int found = -1, last_kept = -1;
    for (int k = 0; k < E; ++k) {
      if (v * E + k >= V) break;
      const float x = Elem<DT>::get(row, v * E + k);
      const uint32_t o = order_of(x);
      if (o > cut) ms += weight(x, r);
      if (o == cut) ++mt;
      if (held(ms, mt) > target && found < 0) found = v * E + k;
      if (held(ms, mt) > at) last_kept = v * E + k;
      at = held(ms, mt);
    }
    return found >= 0 ? found : last_kept;
  };
  int token = -1, spare_v = -1, spare_t = 0;
  double spare_s = 0.0;
  for (int i = 0; i < steps && token < 0; ++i) {
    const int v = first + i * 64 + lane;
    double si;
    int ti;
    lane_part(v, si, ti);
    double cs = si;
    int ct = ti;
    for (int o = 1; o < 64; o <<= 1) {
      const double us = __shfl_up(cs, o);
      const int ut = __shfl_up(ct, o);
      if (lane >= o) {
        cs += us;
        ct += ut;
      }
    }
    const double from = before + cs - si;
    const int from_t = tie_before + ct - ti;
    if (held(from + si, from_t + ti) > held(from, from_t)) {
      spare_v = v;
      spare_s = from;
      spare_t = from_t;
    }
    const unsigned long long over = __ballot(held(before + cs, tie_before + ct) > target);
    if (over != 0) {
      const int who = __builtin_ctzll(over);
      token = __shfl(lane == who ? walk(v, from, from_t) : -1, who);
    }
    before += __shfl(cs, 63);
    tie_before += __shfl(ct, 63);
  }
  if (token < 0) {
    int far = spare_v;
    for (int o = 32; o > 0; o >>= 1) far = max(far, __shfl_xor(far, o));
    const int who = __builtin_ctzll(__ballot(spare_v == far));
    token = __shfl(lane == who && spare_v >= 0 ? walk(spare_v, spare_s, spare_t) : -1, who);
  }
  if (lane != 0) return;
  const double z = ((double)Elem<DT>::get(row, max(token, 0)) - (double)top) * r.c * kLn2_64;
  a.tokens[n] = token;
  if (a.logprobs != nullptr) a.logprobs[n] = (float)(z - log(whole));
  if (a.kept != nullptr) a.kept[n] = greedy ? 0.f : (float)(z - log(total));
}

}  // namespace

hipError_t launch_sample(const SampleArgs& a, int dtype, hipStream_t stream) {
  const dim3 grid(a.logits.rows), block(kThreads);
  switch (dtype) {
    case RP_LOGITS_BF16: sample_kernel<RP_LOGITS_BF16><<<grid, block, 0, stream>>>(a); break;
    case RP_LOGITS_F16: sample_kernel<RP_LOGITS_F16><<<grid, block, 0, stream>>>(a); break;
    default: sample_kernel<RP_LOGITS_F32><<<grid, block, 0, stream>>>(a); break;
  }
  return hipGetLastError();
}

}  // namespace rp
