// Attention of a tree of drafted tokens per sequence over the paged cache and
// the tree itself: draft i of sequence s attends to its group's prefix, the
// sequence's response, and the drafts u with bit u of masks[i]. With s_u the
// scaled scores of one query row in units of log2,
//   lse = ln 2 (m + log2 sum 2^(s_u - m)),  out = sum 2^(s_u - m) v_u / sum 2^(s_u - m),
// in one pass over the keys with a running maximum m. Drafted K and V are
// dense bf16 rows and never enter the cache.
//
// Query rows (draft, query head of the kv-head) are the columns of
//   S^T  = K Q^T   on mfma 16x16x32 bf16 (16 tokens x 16 columns x 32 of head_dim)
//   O^T += V^T P^T on mfma 16x16x16 or 16x16x32 bf16
// CT tiles of 16 columns share every K and V element that a wave loads.
// A workgroup's four waves split a unit's keys, walk them independently and
// merge their states in LDS, so a unit writes one partial result per row.
#include "rp_device.h"
#include "rp_internal.h"

namespace rp {
namespace {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

constexpr int kWaves = kTreeWaves;

// Orders this wave's LDS accesses (its staging area is its own).
__device__ inline void wave_lds_sync() {
  __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// 8 e4m3 codes -> 8 bf16 values (exact).
template <bool HIGH>
__device__ inline uint32_t decode2(uint32_t w) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, HIGH));
}
__device__ inline u32x4_t decode8(uint32_t w0, uint32_t w1) {
  return u32x4_t{decode2<false>(w0), decode2<true>(w0), decode2<false>(w1), decode2<true>(w1)};
}

template <int D, bool FP8, int CT>
struct Shape {
  static constexpr int EB = FP8 ? 1 : 2;                  // bytes per cached element
  static constexpr int ROW_BYTES = D * EB;
  static constexpr int BLOCK_BYTES = kPage * ROW_BYTES;   // one (page, kv-head) block
  static constexpr int EPL = 16 / EB;                     // elements per 16-byte piece
  static constexpr int LOADS = BLOCK_BYTES / 1024;        // pieces per lane and block
  static constexpr int PAGES = 4 / LOADS;                 // pages per step: 8 KiB of K and V
  static constexpr int DT = D / 16;
  static constexpr int PITCH = D + 16;                    // staged V row: a transposing read meets no bank twice
  static constexpr int STAGE = PAGES * kPage * PITCH;     // per wave, bf16 elements
  static constexpr int COLS = 16 * CT;
  static constexpr int OPITCH = D + 4;                    // merged output row, floats
  // The query operands of four tiles of 128-wide heads take 64 registers, too
  // many beside the 128 of the output: they stay in LDS.
  static constexpr bool QLDS = CT * D >= 512;
  static constexpr int QPITCH = D + 8;
  static constexpr int LOOP_BYTES = (kWaves * STAGE + (QLDS ? COLS * QPITCH : 0)) * 2;
  static constexpr int MERGE_BYTES = kWaves * 16 * OPITCH * 4;
  static constexpr int BYTES = LOOP_BYTES > MERGE_BYTES ? LOOP_BYTES : MERGE_BYTES;
};

// What a unit reads: pages of two block tables in a row (a group's prefix and a
// sequence's response, or one of them), then drafted tokens.
struct Keys {
  const int *table_a, *table_b;
  int pages_a, pages_b;    // pages of each
  int tokens_a, tokens_b;  // tokens of each, the last page may be ragged
  int draft0, drafts;      // first drafted token and how many
};

template <int D, bool FP8, int CT>
struct Smem {
  __attribute__((aligned(16))) unsigned char buf[Shape<D, FP8, CT>::BYTES];
  unsigned long long mask[16 * CT];
  int row[16 * CT];  // query row (token * Hq + head), -1: unused column
  float m[kWaves][16 * CT], l[kWaves][16 * CT], r[kWaves][16 * CT];
  int sum[kWaves];
  int token[16 * CT];
};

// One wave's state: per tile the output accumulator (lane (r16, quad) of tile
// t: column r16, elements dt * 16 + quad * 4 + e), the running maximum of the
// column, and this lane's share of two sums of the probabilities: exact (for
// the lse), and as rounded to bf16 for the products. The output is normalised
// by the sum of what was multiplied, so a single dominant key gives its own v;
// an fp8 page's V scale is in its rounded probabilities, and its rows are
// normalised by the exact sum.
template <int D, bool FP8, int CT>
struct State {
  f32x4_t o[CT][D / 16];
  float m[CT], l[CT], r[CT];
};

// Adds N blocks of 16 tokens, scores s (log2 units, -inf where hidden) and
// staged V, to the state. vs: V scales of the blocks.
template <int D, bool FP8, int CT, int N, bool SCALED>
__device__ __forceinline__ void add_blocks(State<D, FP8, CT>& st, f32x4_t (&s)[CT][N], const float (&vs)[N],
                                           bf16x4_t (&pop)[CT][N]) {
  constexpr int DT = D / 16;
  float mx[CT];
  bool grow = false;
#pragma unroll
  for (int t = 0; t < CT; ++t) {
    mx[t] = -INFINITY;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) mx[t] = fmaxf(mx[t], s[t][i][e]);
    grow = grow || mx[t] > st.m[t] + kLazyMax;
  }
  // The maximum moves, and the accumulator is rescaled, only when a score
  // exceeds it by more than the headroom.
  if (__any(grow)) {
#pragma unroll
    for (int t = 0; t < CT; ++t) {
      const float x = max_xor16_32(mx[t]);
      const float now = x > st.m[t] + kLazyMax ? x : st.m[t];
      const float alpha = now == st.m[t] ? 1.f : fast_exp2(st.m[t] - now);
      st.m[t] = now;
      st.l[t] *= alpha;
      st.r[t] *= alpha;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) st.o[t][dt] *= alpha;
    }
  }
#pragma unroll
  for (int t = 0; t < CT; ++t) {
    const float mu = st.m[t] == -INFINITY ? 0.f : st.m[t];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float p[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) p[e] = fast_exp2(s[t][i][e] - mu);
      st.l[t] += (p[0] + p[1]) + (p[2] + p[3]);
      if constexpr (SCALED) {
#pragma unroll
        for (int e = 0; e < 4; ++e) p[e] *= vs[i];
      }
      const uint2 w = make_uint2(pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]));
      if constexpr (!FP8) {
        const bf16x2_t one = {(__bf16)1.0f, (__bf16)1.0f};
        st.r[t] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, w.x), one, st.r[t], false);
        st.r[t] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, w.y), one, st.r[t], false);
      }
      pop[t][i] = __builtin_bit_cast(bf16x4_t, w);
    }
  }
}

// One 16-byte piece of a token's bf16 row, or zeros.
__device__ inline u32x4_t piece(const uint16_t* p, bool ok) {
  u32x4_t w = {0, 0, 0, 0};
  if (ok) w = *reinterpret_cast<const u32x4_t*>(p);
  return w;
}

__device__ inline bool not_finite(uint32_t w) {
  return (w & 0x7F80u) == 0x7F80u || (w & 0x7F800000u) == 0x7F800000u;
}

// Walks this wave's share of the keys: blocks b0 .. b1 - 1 of the unit, of
// which the first pages_a + pages_b are pages and the others drafts.
template <int D, bool FP8, int CT>
__device__ __forceinline__ void walk(const TreeArgs& a, const Keys& k, int h, int b0, int b1,
                                     Smem<D, FP8, CT>& sm, State<D, FP8, CT>& st) {
  using G = Shape<D, FP8, CT>;
  constexpr int EPL = G::EPL, LOADS = G::LOADS, PAGES = G::PAGES, DT = G::DT, PITCH = G::PITCH;
  const int lane = threadIdx.x & 63, r16 = lane & 15, quad = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint16_t* vt = reinterpret_cast<uint16_t*>(sm.buf) + wave * G::STAGE;
  const uint16_t* ql = reinterpret_cast<const uint16_t*>(sm.buf) + kWaves * G::STAGE;
  const int Hkv = a.num_kv_heads;
  const int np = k.pages_a + k.pages_b;

  // Query operands: piece (j, hh) of head_dim, elements (quad + 4 j) EPL + 8 hh
  // on, as the K pieces come (the order of head_dim inside a product is free).
  bf16x8_t qreg[G::QLDS ? 1 : CT][LOADS][EPL / 8];
  if constexpr (!G::QLDS) {
#pragma unroll
    for (int t = 0; t < CT; ++t) {
      const int row = sm.row[t * 16 + r16];
#pragma unroll
      for (int j = 0; j < LOADS; ++j)
#pragma unroll
        for (int hh = 0; hh < EPL / 8; ++hh)
          qreg[t][j][hh] = __builtin_bit_cast(
              bf16x8_t, piece(a.q + (size_t)max(row, 0) * D + (quad + 4 * j) * EPL + hh * 8, row >= 0));
    }
  }
  const auto qop = [&](int t, int j, int hh) __attribute__((always_inline)) {
    if constexpr (G::QLDS)
      return *reinterpret_cast<const bf16x8_t*>(ql + (t * 16 + r16) * G::QPITCH + (quad + 4 * j) * EPL + hh * 8);
    else
      return qreg[t][j][hh];
  };
  const uint16_t* vtr = vt + (quad * 4 + r16 / 4) * PITCH + 4 * (r16 % 4);

  const int p0 = b0, npg = min(b1, np) - b0;
  if (npg > 0) {
    // Every page id of the share, two per lane, and for fp8 the pages' scales.
    int ids[2];
    float ksc[2] = {1.f, 1.f}, vsc[2] = {1.f, 1.f};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int b = p0 + min(64 * i + lane, npg - 1);
      ids[i] = clamp_page(b < k.pages_a ? k.table_a[b] : k.table_b[b - k.pages_a], a.num_pages);
      if constexpr (FP8) {
        ksc[i] = a.k_scale[(size_t)ids[i] * Hkv + h];
        vsc[i] = a.v_scale[(size_t)ids[i] * Hkv + h];
      }
    }
    const auto block = [&](int p) __attribute__((always_inline)) {
      const int q = min(p, npg - 1);
      const int x = __builtin_amdgcn_readlane(ids[0], q & 63), y = __builtin_amdgcn_readlane(ids[1], q & 63);
      return ((size_t)(q < 64 ? x : y) * Hkv + h) * G::BLOCK_BYTES;
    };
    const auto scale_at = [&](const float (&sc)[2], int p) __attribute__((always_inline)) {
      const int q = min(p, npg - 1);
      const int x = __builtin_amdgcn_readlane(__float_as_int(sc[0]), q & 63);
      const int y = __builtin_amdgcn_readlane(__float_as_int(sc[1]), q & 63);
      return __int_as_float(q < 64 ? x : y);
    };
    // Valid tokens of page p of the share; 0 behind its end.
    const auto valid = [&](int p) __attribute__((always_inline)) {
      const int b = p0 + p;
      const int left = b < k.pages_a ? k.tokens_a - b * kPage : k.tokens_b - (b - k.pages_a) * kPage;
      return p < npg ? min(left, kPage) : 0;
    };
    const char* kpool = static_cast<const char*>(a.k_pages) + r16 * G::ROW_BYTES + quad * 16;
    const char* vpool = static_cast<const char*>(a.v_pages) + lane * 16;
    u32x4_t kx[PAGES][LOADS], vx[PAGES][LOADS];
    const auto load_k = [&](int p) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < PAGES; ++i) {
        const char* b = kpool + block(p + i);
#pragma unroll
        for (int j = 0; j < LOADS; ++j) kx[i][j] = *reinterpret_cast<const u32x4_t*>(b + j * 64);
      }
    };
    const auto load_v = [&](int p) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < PAGES; ++i) {
        const char* b = vpool + block(p + i);
#pragma unroll
        for (int j = 0; j < LOADS; ++j) vx[i][j] = *reinterpret_cast<const u32x4_t*>(b + j * 1024);
      }
    };
    load_k(0);
    load_v(0);
    for (int p = 0; p < npg; p += PAGES) {
      f32x4_t s[CT][PAGES];
#pragma unroll
      for (int i = 0; i < PAGES; ++i) {
#pragma unroll
        for (int t = 0; t < CT; ++t) s[t][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
          const u32x4_t w = kx[i][j];
#pragma unroll
          for (int hh = 0; hh < EPL / 8; ++hh) {
            const u32x4_t kw = !FP8 ? w : hh == 0 ? decode8(w.x, w.y) : decode8(w.z, w.w);
#pragma unroll
            for (int t = 0; t < CT; ++t)
              s[t][i] = mfma16x16x32(__builtin_bit_cast(bf16x8_t, kw), qop(t, j, hh), s[t][i]);
          }
        }
      }
      // Each refill stays behind the last use of the registers it overwrites.
      __builtin_amdgcn_sched_barrier(0);
      load_k(p + PAGES);

      wave_lds_sync();  // the step before has read the staged V
      bool ragged = false;
#pragma unroll
      for (int i = 0; i < PAGES; ++i) ragged = ragged || valid(p + i) < kPage;
#pragma unroll
      for (int i = 0; i < PAGES; ++i) {
        const int nv = valid(p + i);
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
          const int e0 = (j * 64 + lane) * EPL, tok = e0 / D, col = e0 % D;
          u32x4_t* dst = reinterpret_cast<u32x4_t*>(vt + (i * kPage + tok) * PITCH + col);
          u32x4_t w = vx[i][j];
          if (ragged) w = tok < nv ? w : u32x4_t{0, 0, 0, 0};  // padding rows may hold anything
          if constexpr (!FP8) {
            dst[0] = w;
          } else {
            dst[0] = decode8(w.x, w.y);
            dst[1] = decode8(w.z, w.w);
          }
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      load_v(p + PAGES);

      float vs[PAGES];
#pragma unroll
      for (int i = 0; i < PAGES; ++i) {
        const float km = FP8 ? a.qk_scale * scale_at(ksc, p + i) : a.qk_scale;
        vs[i] = FP8 ? scale_at(vsc, p + i) : 1.f;
#pragma unroll
        for (int t = 0; t < CT; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[t][i][e] *= km;
      }
      if (ragged) {
#pragma unroll
        for (int i = 0; i < PAGES; ++i) {
          const int nv = valid(p + i);
#pragma unroll
          for (int t = 0; t < CT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[t][i][e] = quad * 4 + e < nv ? s[t][i][e] : -INFINITY;
        }
      }
      bf16x4_t pop[CT][PAGES];
      add_blocks<D, FP8, CT, PAGES, FP8>(st, s, vs, pop);

      wave_lds_sync();  // the staged V is visible to the whole wave
      if constexpr (PAGES == 1) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          const bf16x4_t v0 = lds_read_tr(vtr + dt * 16);
#pragma unroll
          for (int t = 0; t < CT; ++t) st.o[t][dt] = mfma16x16x16(v0, pop[t][0], st.o[t][dt]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < PAGES; i += 2)
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) {
            const bf16x4_t v0 = lds_read_tr(vtr + i * kPage * PITCH + dt * 16);
            const bf16x4_t v1 = lds_read_tr(vtr + (i + 1) * kPage * PITCH + dt * 16);
            const bf16x8_t vo = __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
            for (int t = 0; t < CT; ++t)
              st.o[t][dt] = mfma16x16x32(
                  vo, __builtin_shufflevector(pop[t][i], pop[t][i + 1], 0, 1, 2, 3, 4, 5, 6, 7), st.o[t][dt]);
          }
      }
    }
  }

  // The drafts of the share, 16 at a time.
  for (int b = max(b0, np); b < b1; ++b) {
    const int u0 = (b - np) * kPage, nv = min(k.drafts - u0, kPage);
    const size_t stride = (size_t)Hkv * D;
    const uint16_t* kd = a.k_draft + ((size_t)(k.draft0 + u0) * Hkv + h) * D;
    const uint16_t* vd = a.v_draft + ((size_t)(k.draft0 + u0) * Hkv + h) * D;
    constexpr int VL = kPage * D / 512;  // 16-byte pieces per lane of a bf16 block
    u32x4_t vx[VL];
    bool bad[VL], any_bad = false;
#pragma unroll
    for (int j = 0; j < VL; ++j) {
      const int e0 = (j * 64 + lane) * 8, tok = e0 / D, col = e0 % D;
      vx[j] = piece(vd + tok * stride + col, tok < nv);
      bad[j] = not_finite(vx[j].x) || not_finite(vx[j].y) || not_finite(vx[j].z) || not_finite(vx[j].w);
      any_bad = any_bad || bad[j];
    }
    f32x4_t s[CT][1];
#pragma unroll
    for (int t = 0; t < CT; ++t) s[t][0] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < LOADS; ++j)
#pragma unroll
      for (int hh = 0; hh < EPL / 8; ++hh) {
        const u32x4_t kw = piece(kd + r16 * stride + (quad + 4 * j) * EPL + hh * 8, r16 < nv);
#pragma unroll
        for (int t = 0; t < CT; ++t) s[t][0] = mfma16x16x32(__builtin_bit_cast(bf16x8_t, kw), qop(t, j, hh), s[t][0]);
      }
    // A draft that a row does not see may hold anything: its score is
    // replaced, and a V row with an infinity or NaN, which a weight of zero
    // would not hide in the product, is left out of it and added below to the
    // rows that see it.
    unsigned long long seen[CT];
#pragma unroll
    for (int t = 0; t < CT; ++t) {
      seen[t] = sm.mask[t * 16 + r16] >> u0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool ok = quad * 4 + e < nv && (seen[t] >> (quad * 4 + e) & 1);
        s[t][0][e] = ok ? s[t][0][e] * a.qk_scale : -INFINITY;
      }
    }
    int odd = 0;  // drafts of the block with such a V row
    if (__any(any_bad)) {
      constexpr int LPT = D / 8, TPL = 64 / LPT;  // lanes per token, tokens per load
#pragma unroll
      for (int j = 0; j < VL; ++j) {
        const unsigned long long w = __ballot(bad[j]);
#pragma unroll
        for (int i = 0; i < TPL; ++i) odd |= (w >> (i * LPT) & ((1ull << LPT) - 1)) != 0 ? 1 << (j * TPL + i) : 0;
      }
    }
    wave_lds_sync();
#pragma unroll
    for (int j = 0; j < VL; ++j) {
      const int e0 = (j * 64 + lane) * 8, tok = e0 / D, col = e0 % D;
      *reinterpret_cast<u32x4_t*>(vt + tok * PITCH + col) = odd >> tok & 1 ? u32x4_t{0, 0, 0, 0} : vx[j];
    }
    bf16x4_t pop[CT][1];
    const float none[1] = {1.f};
    add_blocks<D, FP8, CT, 1, false>(st, s, none, pop);
    wave_lds_sync();
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      const bf16x4_t v0 = lds_read_tr(vtr + dt * 16);
#pragma unroll
      for (int t = 0; t < CT; ++t) st.o[t][dt] = mfma16x16x16(v0, pop[t][0], st.o[t][dt]);
    }
    while (odd != 0) {
      const int u = __builtin_amdgcn_readfirstlane(__builtin_ctz(odd));
      odd &= odd - 1;
#pragma unroll
      for (int t = 0; t < CT; ++t) {
        const uint2 w = __builtin_bit_cast(uint2, pop[t][0]);
        const uint32_t word = u & 2 ? w.y : w.x;
        const float p = __shfl(u & 1 ? bf16_hi(word) : bf16_lo(word), (u >> 2) * 16 + r16);
        const bool ok = seen[t] >> u & 1;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          const uint2 x = *reinterpret_cast<const uint2*>(vd + u * stride + dt * 16 + quad * 4);
          const float v[4] = {bf16_lo(x.x), bf16_hi(x.x), bf16_lo(x.y), bf16_hi(x.y)};
#pragma unroll
          for (int e = 0; e < 4; ++e) st.o[t][dt][e] = ok ? fmaf(p, v[e], st.o[t][dt][e]) : st.o[t][dt][e];
        }
      }
    }
  }
}

// A unit: the columns in sm.row over `k`, split between the waves, merged and
// stored: final rows (slot < 0), or the partial results in their slot.
template <int D, bool FP8, int CT>
__device__ __forceinline__ void unit(const TreeArgs& a, const Keys& k, int h, int slot, Smem<D, FP8, CT>& sm) {
  using G = Shape<D, FP8, CT>;
  const int tid = threadIdx.x, lane = tid & 63, r16 = lane & 15, quad = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  if constexpr (G::QLDS) {
    uint16_t* ql = reinterpret_cast<uint16_t*>(sm.buf) + kWaves * G::STAGE;
    for (int i = tid; i < G::COLS * (D / 8); i += 64 * kWaves) {
      const int c = i / (D / 8), d = i % (D / 8) * 8, row = sm.row[c];
      *reinterpret_cast<u32x4_t*>(ql + c * G::QPITCH + d) = piece(a.q + (size_t)max(row, 0) * D + d, row >= 0);
    }
    __syncthreads();
  }
  State<D, FP8, CT> st;
#pragma unroll
  for (int t = 0; t < CT; ++t) {
    st.m[t] = -INFINITY;
    st.l[t] = st.r[t] = 0.f;
#pragma unroll
    for (int dt = 0; dt < G::DT; ++dt) st.o[t][dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  const int blocks = k.pages_a + k.pages_b + cdiv(k.drafts, kPage);
  const int per = cdiv(cdiv(blocks, kWaves), G::PAGES) * G::PAGES;
  const int b0 = min(wave * per, blocks), b1 = min(b0 + per, blocks);
  if (b0 < b1) walk<D, FP8, CT>(a, k, h, b0, b1, sm, st);

#pragma unroll
  for (int t = 0; t < CT; ++t) {
    const float l = xor_sum_from<16>(st.l[t]);
    const float r = FP8 ? l : xor_sum_from<16>(st.r[t]);
    if (quad == 0) {
      sm.m[wave][t * 16 + r16] = st.m[t];
      sm.l[wave][t * 16 + r16] = l;
      sm.r[wave][t * 16 + r16] = r;
    }
  }
  __syncthreads();  // also: every wave is done with sm.buf
  float* om = reinterpret_cast<float*>(sm.buf);
#pragma unroll
  for (int t = 0; t < CT; ++t) {
    if (t > 0 && sm.row[t * 16] < 0) break;  // columns are filled from the first on
    const int c = t * 16 + r16;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, sm.m[w][c]);
    float l = 0.f, r = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = sm.m[w][c] == top ? 1.f : fast_exp2(sm.m[w][c] - top);
      l += f * sm.l[w][c];
      r += f * sm.r[w][c];
    }
    const float mine = (st.m[t] == top ? 1.f : fast_exp2(st.m[t] - top)) * (r == 0.f ? 0.f : 1.f / r);
    if (t > 0) __syncthreads();  // the tile before has been read
#pragma unroll
    for (int dt = 0; dt < G::DT; ++dt) {
      const f32x4_t x = st.o[t][dt] * mine;
      *reinterpret_cast<f32x4_t*>(om + (wave * 16 + r16) * G::OPITCH + dt * 16 + quad * 4) = x;
    }
    const int row = sm.row[c];
    if (wave == 0 && quad == 0 && row >= 0) {
      const float lse = l == 0.f ? -INFINITY : (top + fast_log2(l)) * kLn2;
      if (slot < 0) {
        if (a.lse != nullptr) a.lse[row] = lse;
      } else {
        a.part_lse[(size_t)row * a.parts_per_row + slot] = lse;
      }
    }
    __syncthreads();
    constexpr int E = D / 16;  // elements per thread: 16 threads a column
    const int col = tid / 16, d0 = tid % 16 * E;
    const int orow = sm.row[t * 16 + col];
    float x[E];
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
#pragma unroll
      for (int e = 0; e < E; e += 4) {
        const f32x4_t y = *reinterpret_cast<const f32x4_t*>(om + (w * 16 + col) * G::OPITCH + d0 + e);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[e + i] += y[i];
      }
    if (orow >= 0) {
      if (slot < 0) {
        uint32_t* dst = reinterpret_cast<uint32_t*>(a.out + (size_t)orow * D + d0);
#pragma unroll
        for (int e = 0; e < E; e += 2) dst[e / 2] = pack_bf16x2(x[e], x[e + 1]);
      } else {
        float4* dst = reinterpret_cast<float4*>(a.part_o + ((size_t)orow * a.parts_per_row + slot) * D + d0);
#pragma unroll
        for (int e = 0; e < E; e += 4) dst[e / 4] = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
      }
    }
  }
}

__device__ inline int2 drafts_of(const TreeArgs& a, int s) {
  const int t0 = min(max(a.draft_offs[s], 0), a.num_drafts);
  return make_int2(t0, min(max(a.draft_offs[s + 1] - t0, 0), min(a.max_drafts, a.num_drafts - t0)));
}

// Columns c0 .. of the drafts of group g, in sequence order: the tokens are
// found by a scan over the sequences' groups and tree sizes. Returns whether
// there are any.
template <int D, bool FP8, int CT>
__device__ bool group_columns(const TreeArgs& a, int g, int h, int c0, Smem<D, FP8, CT>& sm) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int k0 = c0 >> a.rep_shift, k1 = (c0 + 16 * CT) >> a.rep_shift;
  __syncthreads();  // the columns before have been read
  int carry = 0;
  for (int base = 0; base < a.num_seqs && carry < k1; base += 64 * kWaves) {
    const int s = base + tid;
    int2 dr = make_int2(0, 0);
    if (s < a.num_seqs && clamp_group(a.seq_to_group[s], a.num_groups) == g) dr = drafts_of(a, s);
    int x = dr.y;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_up(x, o);
      x += lane >= o ? y : 0;
    }
    if (lane == 63) sm.sum[wave] = x;
    __syncthreads();
    int start = carry + x - dr.y;
    for (int w = 0; w < kWaves; ++w) {
      start += w < wave ? sm.sum[w] : 0;
      carry += sm.sum[w];
    }
    for (int i = max(k0 - start, 0); i < min(dr.y, k1 - start); ++i) sm.token[start + i - k0] = dr.x + i;
    __syncthreads();
  }
  if (carry <= k0) return false;
  if (tid < 16 * CT) {
    const int c = c0 + tid, rank = c >> a.rep_shift;
    const int rep = c & ((1 << a.rep_shift) - 1);
    sm.row[tid] = rank < carry ? sm.token[rank - k0] * a.num_q_heads + (h << a.rep_shift) + rep : -1;
  }
  __syncthreads();
  return true;
}

// Units of a launch: (group, chunk of prefix pages, kv-head), each several
// times where a group has many rows, then (sequence, piece of response pages,
// kv-head, block of rows). Row blocks of one unit follow each other on one XCD
// (workgroups are dealt to the 8 of them in turn), whose L2 then has the K and
// V that the first one read. A response's pieces are cut from its end, so its
// first piece is the short one; pieces are launched from the last to the first
// and the short ones end the launch. The first piece also takes the drafts.
// In the whole form a unit takes all keys of its rows, prefix included.
template <int D, bool FP8, int CT>
__global__ __launch_bounds__(64 * kWaves) void tree_kernel(const TreeArgs a) {
  __shared__ Smem<D, FP8, CT> sm;
  const int Hkv = a.num_kv_heads;
  const auto locate = [](int id, int repeats, int& u, int& r) {
    const int row = id / (8 * repeats), k = id - row * (8 * repeats);
    r = k / 8;
    u = row * 8 + k % 8;
  };
  int id = blockIdx.x;
  if (id < a.prefix_blocks) {
    int u, z;
    locate(id, a.prefix_repeats, u, z);
    if (u >= a.num_groups * a.max_prefix_chunks * Hkv) return;
    const int h = u % Hkv, chunk = u / Hkv % a.max_prefix_chunks, g = u / Hkv / a.max_prefix_chunks;
    const int P = clamp_len(a.prefix_lens[g], a.max_prefix_pages), first = chunk * a.prefix_chunk;
    const int pages = min(cdiv(P, kPage) - first, a.prefix_chunk);
    if (pages <= 0) return;
    Keys k = {};
    k.table_a = k.table_b = a.prefix_block_table + (size_t)g * a.max_prefix_pages + first;
    k.pages_a = pages;
    k.tokens_a = P - first * kPage;
    for (int rb = z; group_columns<D, FP8, CT>(a, g, h, rb * 16 * CT, sm); rb += a.prefix_repeats)
      unit<D, FP8, CT>(a, k, h, chunk, sm);
    return;
  }
  id -= a.prefix_blocks;
  int u, rb;
  locate(id, a.row_blocks, u, rb);
  const int per_piece = a.num_seqs * Hkv;
  const int piece_id = a.max_pieces - 1 - u / per_piece;
  if (piece_id < 0) return;
  const int s = u % per_piece / Hkv, h = u % Hkv;
  const int2 dr = drafts_of(a, s);
  const int c0 = rb * 16 * CT;
  if (c0 >= dr.y << a.rep_shift) return;
  const int g = clamp_group(a.seq_to_group[s], a.num_groups);
  const int L = clamp_len(a.resp_lens[s], a.max_resp_pages), P = clamp_len(a.prefix_lens[g], a.max_prefix_pages);
  const int pages = cdiv(L, kPage), prefix_pages = cdiv(P, kPage);
  Keys k = {};
  k.table_a = k.table_b = a.resp_block_table + (size_t)s * a.max_resp_pages;
  int slot = -1;
  if (a.whole) {
    k.table_a = a.prefix_block_table + (size_t)g * a.max_prefix_pages;
    k.pages_a = prefix_pages;
    k.tokens_a = P;
    k.pages_b = pages;
    k.tokens_b = L;
  } else {
    const int pieces = max(cdiv(pages, a.piece_pages), 1);
    if (piece_id >= pieces) return;
    const int first = piece_id == 0 ? 0 : pages - (pieces - piece_id) * a.piece_pages;
    const int end = pages - (pieces - 1 - piece_id) * a.piece_pages;
    const int chunks = cdiv(prefix_pages, a.prefix_chunk);
    k.table_b += first;
    k.pages_b = end - first;
    k.tokens_b = L - first * kPage;
    if (chunks + pieces > 1) slot = chunks + piece_id;
    // Rows whose result is stored here have no partial results to merge.
    if (piece_id == 0 && h == 0)
      for (int i = threadIdx.x; i < 16 * CT; i += 64 * kWaves) {
        const int c = c0 + i;
        if (c < dr.y << a.rep_shift && (c & ((1 << a.rep_shift) - 1)) == 0)
          a.token_parts[dr.x + (c >> a.rep_shift)] = chunks + pieces > 1 ? chunks + pieces : 0;
      }
  }
  if (piece_id == 0) {
    k.draft0 = dr.x;
    k.drafts = dr.y;
  }
  for (int i = threadIdx.x; i < 16 * CT; i += 64 * kWaves) {
    const int c = c0 + i, t = c >> a.rep_shift;
    const bool live = t < dr.y;
    sm.row[i] = live ? (dr.x + t) * a.num_q_heads + (h << a.rep_shift) + (c & ((1 << a.rep_shift) - 1)) : -1;
    sm.mask[i] = live && piece_id == 0 ? a.masks[dr.x + t] : 0;
  }
  __syncthreads();
  unit<D, FP8, CT>(a, k, h, slot, sm);
}

template <int D, bool FP8>
hipError_t by_tiles(const TreeArgs& a, int tiles, unsigned blocks, hipStream_t st) {
  const dim3 grid(blocks), threads(64 * kWaves);
  switch (tiles) {
    case 1: tree_kernel<D, FP8, 1><<<grid, threads, 0, st>>>(a); break;
    case 2: tree_kernel<D, FP8, 2><<<grid, threads, 0, st>>>(a); break;
    case 4: tree_kernel<D, FP8, 4><<<grid, threads, 0, st>>>(a); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_tree_attn(const TreeArgs& a, int head_dim, bool fp8, int tiles, long long blocks,
                            hipStream_t stream) {
  if (blocks <= 0) return hipSuccess;
  if (blocks >= (1ll << 31)) return hipErrorInvalidValue;
  const unsigned n = (unsigned)blocks;
  if (head_dim == 128) return fp8 ? by_tiles<128, true>(a, tiles, n, stream) : by_tiles<128, false>(a, tiles, n, stream);
  if (head_dim == 64) return fp8 ? by_tiles<64, true>(a, tiles, n, stream) : by_tiles<64, false>(a, tiles, n, stream);
  return hipErrorInvalidValue;
}

}  // namespace rp
