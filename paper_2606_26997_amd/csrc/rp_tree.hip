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
// Two forms, by the query rows of a unit of keys:
//   split  the four waves of a workgroup split a unit's keys, each walks its
//          share for CT tiles of 16 columns, and their states are merged in
//          LDS;
//   rows   the waves share the unit's keys, 32 at a time in LDS, and have RT
//          tiles of 16 rows each: K and V are read once for 64 RT rows.
// Group prefixes, whose rows are those of all members, always take the second.
#include "rp_device.h"
#include "rp_internal.h"
#include "rp_stage.h"

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

// 16 codes, decoded, to 32 bytes of LDS. Neighbouring lanes' pieces follow each
// other there, so with the halves in one order half of the banks would get all
// of a write: odd lanes write their second half first.
__device__ inline void store_decoded(u32x4_t* dst, const u32x4_t& w, int odd) {
  dst[odd] = decode8(odd ? w.z : w.x, odd ? w.w : w.y);
  dst[1 - odd] = decode8(odd ? w.x : w.z, odd ? w.y : w.w);
}

template <int D, bool FP8, int CT>
struct Shape {
  static constexpr int EB = FP8 ? 1 : 2;                  // bytes per cached element
  static constexpr int ROW_BYTES = D * EB;
  static constexpr int BLOCK_BYTES = kPage * ROW_BYTES;   // one (page, kv-head) block
  static constexpr int EPL = 16 / EB;                     // elements per 16-byte piece
  static constexpr int LOADS = BLOCK_BYTES / 1024;        // pieces per lane and block
  // Pages per step: 8 KiB of K and V, half of that where the scores of four
  // tiles for them would not fit the registers.
  static constexpr int PAGES = 4 / LOADS / (FP8 && CT == 4 ? 2 : 1);
  static constexpr int DT = D / 16;
  static constexpr int PITCH = D + 16;                    // staged V row: a transposing read meets no bank twice
  static constexpr bool PAIR = PAGES == 1 && CT == 4;     // P V of two one-page steps at once
  static constexpr int STAGE = (PAIR ? 2 : PAGES) * kPage * PITCH;  // per wave, bf16 elements
  static constexpr int COLS = 16 * CT;
  static constexpr int OPITCH = D + 4;                    // merged output row, floats
  // The query operands of four tiles of 128-wide heads take 64 registers, too
  // many beside the 128 of the output: they stay in LDS.
  static constexpr bool QLDS = CT * D >= 512;
  static constexpr int QPITCH = D + 16;
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
};

// One wave's state: per tile the output accumulator (lane (r16, quad) of tile
// t: column r16, elements dt * 16 + quad * 4 + e), minus the column's running
// maximum (0 until it has one), the threshold over it that moves it (-inf until
// then), and this lane's share of two sums of the probabilities: exact (for the
// lse), and as rounded to bf16 for the products. The output is normalised by
// the sum of what was multiplied, so a single dominant key gives its own v. An
// fp8 page's V scale is in its rounded probabilities, whose sum is divided by
// it again: the rounding of a scale is then in both and cancels (relative rms
// error over 25 to 43 tokens 0.0019, over 8192 to 32768 0.0018; with the exact
// sum below them up to 0.0027 and 0.0023, the latter in 0.95 of the time).
template <int D, int T>
struct State {
  f32x4_t o[T][D / 16];
  float neg[T], thr[T], l[T], r[T];
  __device__ void clear() {
#pragma unroll
    for (int t = 0; t < T; ++t) {
      neg[t] = l[t] = r[t] = 0.f;
      thr[t] = -INFINITY;
#pragma unroll
      for (int dt = 0; dt < D / 16; ++dt) o[t][dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
  }
};

// The softmax step of tile t over N blocks of 16 keys: scores x (log2 units,
// less the running maximum, -inf where hidden) become rounded probabilities,
// times the blocks' V scales vs where SCALED. The maximum moves, and the
// accumulator is rescaled, only when a score exceeds it by more than the
// headroom; before() then comes first.
template <int D, int T, int N, bool SCALED, class Before>
__device__ __forceinline__ void softmax_step(State<D, T>& st, int t, f32x4_t (&x)[N], const float (&vs)[N],
                                             bf16x4_t (&pop)[N], Before before) {
  float mx = -INFINITY;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) mx = fmaxf(mx, x[i][e]);
  if (__any(mx > st.thr[t])) {
    before();
    mx = max_xor16_32(mx);
    const float up = mx > st.thr[t] ? mx : 0.f;
    const float alpha = st.thr[t] == -INFINITY ? 0.f : fast_exp2(-up);  // nothing yet: 0 times it
    st.thr[t] = mx > st.thr[t] ? kLazyMax : st.thr[t];
    st.neg[t] -= up;
    st.l[t] *= alpha;
    st.r[t] *= alpha;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] -= up;
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) st.o[t][dt] *= alpha;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float p[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) p[e] = fast_exp2(x[i][e]);
    const float sum = (p[0] + p[1]) + (p[2] + p[3]);
    st.l[t] += sum;
    if constexpr (SCALED) {
#pragma unroll
      for (int e = 0; e < 4; ++e) p[e] *= vs[i];
    }
    const uint2 w = make_uint2(pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]));
    const bf16x2_t one = {(__bf16)1.0f, (__bf16)1.0f};
    float r = SCALED ? 0.f : st.r[t];
    r = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, w.x), one, r, false);
    r = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, w.y), one, r, false);
    // A page of zeros has no scale to divide by.
    if constexpr (SCALED) st.r[t] = vs[i] > 1e-30f ? fmaf(r, __builtin_amdgcn_rcpf(vs[i]), st.r[t]) : st.r[t] + sum;
    else st.r[t] = r;
    pop[i] = __builtin_bit_cast(bf16x4_t, w);
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

// Where a unit's results go: partial results follow each other as the query
// rows do in the order (kv-head, token, query head of the kv-head), from `base`
// on; kFinal: they are stored at once.
constexpr long long kFinal = -(1ll << 62);
__device__ inline long long part_of(const TreeArgs& a, int row, long long base) {
  const int t = row / a.num_q_heads, j = row - t * a.num_q_heads;
  const int h = j >> a.rep_shift, rep = j & ((1 << a.rep_shift) - 1);
  return base + (((long long)h * a.num_drafts + t) << a.rep_shift) + rep;
}

// A lane's part of row `row` (-1: none) of a 16-row tile: elements dt * 16 +
// quad * 4 + e.
template <int D>
__device__ inline void store_row(const TreeArgs& a, int row, long long part, int quad, const f32x4_t (&o)[D / 16],
                                 float inv, float lse) {
  if (row < 0) return;
  if (part == kFinal) {
    uint16_t* dst = a.out + (size_t)row * D + quad * 4;
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) {
      const f32x4_t x = o[dt] * inv;
      *reinterpret_cast<uint2*>(dst + dt * 16) = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
    }
    if (a.lse != nullptr && quad == 0) a.lse[row] = lse;
  } else {
    const long long at = part_of(a, row, part);
    float* dst = a.part_o + at * D + quad * 4;
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) *reinterpret_cast<f32x4_t*>(dst + dt * 16) = o[dt] * inv;
    if (quad == 0) a.part_lse[at] = lse;
  }
}

// Walks this wave's share of the keys: blocks b0 .. b1 - 1 of the unit, of
// which the first pages_a + pages_b are pages and the others drafts. In LDS: vt
// is the wave's staging area, ql the query rows (where they are there), rows
// and masks the columns'.
template <int D, bool FP8, int CT>
__device__ __forceinline__ void walk(const TreeArgs& a, const Keys& k, int h, int b0, int b1, uint16_t* vt,
                                     const uint16_t* ql, const int* rows, const unsigned long long* masks,
                                     State<D, CT>& st) {
  using G = Shape<D, FP8, CT>;
  constexpr int EPL = G::EPL, LOADS = G::LOADS, PAGES = G::PAGES, DT = G::DT, PITCH = G::PITCH;
  const int lane = threadIdx.x & 63, r16 = lane & 15, quad = lane >> 4;
  const int Hkv = a.num_kv_heads;
  const int np = k.pages_a + k.pages_b;

  // Query operands: piece (j, hh) of head_dim, elements (quad + 4 j) EPL + 8 hh
  // on, as the K pieces come (the order of head_dim inside a product is free).
  bf16x8_t qreg[G::QLDS ? 1 : CT][LOADS][EPL / 8];
  if constexpr (!G::QLDS) {
#pragma unroll
    for (int t = 0; t < CT; ++t) {
      const int row = rows[t * 16 + r16];
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
      return *reinterpret_cast<const bf16x8_t*>(ql + (t * 16 + r16) * G::QPITCH + (j * (EPL / 8) + hh) * 32 + quad * 8);
    else
      return qreg[t][j][hh];
  };
  const uint16_t* vtr = vt + (quad * 4 + r16 / 4) * PITCH + 4 * (r16 % 4);

  // 128 pages at a time: their ids, two per lane, and for fp8 their scales.
#pragma unroll 1
  for (int p0 = b0; p0 < min(b1, np); p0 += 128) {
    const int npg = min(min(b1, np) - p0, 128);
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
        for (int j = 0; j < LOADS; ++j)
          vx[i][j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(b + j * 1024));
      }
    };
    load_k(0);
    load_v(0);
    // Scores, staged V (page `at` of the staging area) and probabilities of one
    // step; before(t): see softmax_step.
    const auto scores = [&](int p, int at, bf16x4_t (&pop)[CT][PAGES], auto before) __attribute__((always_inline)) {
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
          u32x4_t* dst = reinterpret_cast<u32x4_t*>(vt + ((at + i) * kPage + tok) * PITCH + col);
          u32x4_t w = vx[i][j];
          if (ragged) w = tok < nv ? w : u32x4_t{0, 0, 0, 0};  // padding rows may hold anything
          if constexpr (!FP8) dst[0] = w;
          else store_decoded(dst, w, lane & 1);
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
          for (int e = 0; e < 4; ++e) s[t][i][e] = fmaf(s[t][i][e], km, st.neg[t]);
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
#pragma unroll
      for (int t = 0; t < CT; ++t)
        softmax_step<D, CT, PAGES, FP8>(st, t, s[t], vs, pop[t], [&] { before(t); });
      wave_lds_sync();  // the staged V is visible to the whole wave
    };
    // O^T += V^T P^T of one page, of tile t; of two pages, all tiles.
    const auto add_page = [&](int at, int t, const bf16x4_t& pop) __attribute__((always_inline)) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
        st.o[t][dt] = mfma16x16x16(lds_read_tr(vtr + at * kPage * PITCH + dt * 16), pop, st.o[t][dt]);
    };
    const auto add_two = [&](int at, const bf16x4_t (&x)[CT], const bf16x4_t (&y)[CT]) __attribute__((always_inline)) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const bf16x4_t v0 = lds_read_tr(vtr + at * kPage * PITCH + dt * 16);
        const bf16x4_t v1 = lds_read_tr(vtr + (at + 1) * kPage * PITCH + dt * 16);
        const bf16x8_t vo = __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
        for (int t = 0; t < CT; ++t)
          st.o[t][dt] = mfma16x16x32(vo, __builtin_shufflevector(x[t], y[t], 0, 1, 2, 3, 4, 5, 6, 7), st.o[t][dt]);
      }
    };
    const auto nothing = [](int) {};
    if constexpr (G::PAIR) {
      // The products with V take two pages' probabilities at once, at twice the
      // rate. A maximum that moves in between first adds the first page's.
      bf16x4_t first[CT][1], second[CT][1];
      int p = 0;
      for (; p + 1 < npg; p += 2) {
        scores(p, 0, first, nothing);
        scores(p + 1, 1, second, [&](int t) __attribute__((always_inline)) {
          add_page(0, t, first[t][0]);
          first[t][0] = __builtin_bit_cast(bf16x4_t, make_uint2(0, 0));
        });
        bf16x4_t x[CT], y[CT];
#pragma unroll
        for (int t = 0; t < CT; ++t) x[t] = first[t][0], y[t] = second[t][0];
        add_two(0, x, y);
      }
      if (p < npg) {
        scores(p, 0, first, nothing);
#pragma unroll
        for (int t = 0; t < CT; ++t) add_page(0, t, first[t][0]);
      }
    } else {
      for (int p = 0; p < npg; p += PAGES) {
        bf16x4_t pop[CT][PAGES];
        scores(p, 0, pop, nothing);
        if constexpr (PAGES == 1) {
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) {
            const bf16x4_t v0 = lds_read_tr(vtr + dt * 16);
#pragma unroll
            for (int t = 0; t < CT; ++t) st.o[t][dt] = mfma16x16x16(v0, pop[t][0], st.o[t][dt]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < PAGES; i += 2) {
            bf16x4_t x[CT], y[CT];
#pragma unroll
            for (int t = 0; t < CT; ++t) x[t] = pop[t][i], y[t] = pop[t][i + 1];
            add_two(i, x, y);
          }
        }
      }
    }
  }

  // The drafts of the share, 16 at a time (before the pages, with those on
  // their way, is 1 us less for one sequence and 2 us more for eight: registers).
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
      seen[t] = masks[t * 16 + r16] >> u0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool ok = quad * 4 + e < nv && (seen[t] >> (quad * 4 + e) & 1);
        s[t][0][e] = ok ? fmaf(s[t][0][e], a.qk_scale, st.neg[t]) : -INFINITY;
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
#pragma unroll
    for (int t = 0; t < CT; ++t) softmax_step<D, CT, 1, false>(st, t, s[t], none, pop[t], [] {});
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
// stored: as final rows (part == kFinal), or as partial results from `part` on.
template <int D, bool FP8, int CT>
__device__ __forceinline__ void split_unit(const TreeArgs& a, const Keys& k, int h, long long part,
                                           Smem<D, FP8, CT>& sm) {
  using G = Shape<D, FP8, CT>;
  const int tid = threadIdx.x, lane = tid & 63, r16 = lane & 15, quad = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  if constexpr (G::QLDS) {
    uint16_t* ql = reinterpret_cast<uint16_t*>(sm.buf) + kWaves * G::STAGE;
    for (int i = tid; i < G::COLS * (D / 8); i += 64 * kWaves) {
      const int c = i / (D / 8), d = i % (D / 8) * 8, row = sm.row[c];
      // In the order of the reads, 8 elements of the four quads side by side.
      const int quad_ = d / G::EPL % 4, jh = d / G::EPL / 4 * (G::EPL / 8) + d % G::EPL / 8;
      *reinterpret_cast<u32x4_t*>(ql + c * G::QPITCH + jh * 32 + quad_ * 8) =
          piece(a.q + (size_t)max(row, 0) * D + d, row >= 0);
    }
    __syncthreads();
  }
  State<D, CT> st;
  st.clear();
  const int blocks = k.pages_a + k.pages_b + cdiv(k.drafts, kPage);
  const int per = cdiv(cdiv(blocks, kWaves), G::PAGES) * G::PAGES;
  const int b0 = min(wave * per, blocks), b1 = min(b0 + per, blocks);
  uint16_t* buf = reinterpret_cast<uint16_t*>(sm.buf);
  if (b0 < b1)
    walk<D, FP8, CT>(a, k, h, b0, b1, buf + wave * G::STAGE, buf + kWaves * G::STAGE, sm.row, sm.mask, st);

#pragma unroll
  for (int t = 0; t < CT; ++t) {
    const float l = xor_sum_from<16>(st.l[t]);
    const float r = xor_sum_from<16>(st.r[t]);
    if (quad == 0) {
      sm.m[wave][t * 16 + r16] = st.thr[t] == -INFINITY ? -INFINITY : -st.neg[t];
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
    const float own = sm.m[wave][c];
    const float mine = (own == top ? 1.f : fast_exp2(own - top)) * (r == 0.f ? 0.f : 1.f / r);
    if (t > 0) __syncthreads();  // the tile before has been read
#pragma unroll
    for (int dt = 0; dt < G::DT; ++dt) {
      const f32x4_t x = st.o[t][dt] * mine;
      *reinterpret_cast<f32x4_t*>(om + (wave * 16 + r16) * G::OPITCH + dt * 16 + quad * 4) = x;
    }
    const int row = sm.row[c];
    if (wave == 0 && quad == 0 && row >= 0) {
      const float lse = l == 0.f ? -INFINITY : (top + fast_log2(l)) * kLn2;
      if (part == kFinal) {
        if (a.lse != nullptr) a.lse[row] = lse;
      } else {
        a.part_lse[part_of(a, row, part)] = lse;
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
      if (part == kFinal) {
        uint32_t* dst = reinterpret_cast<uint32_t*>(a.out + (size_t)orow * D + d0);
#pragma unroll
        for (int e = 0; e < E; e += 2) dst[e / 2] = pack_bf16x2(x[e], x[e + 1]);
      } else {
        float4* dst = reinterpret_cast<float4*>(a.part_o + part_of(a, orow, part) * D + d0);
#pragma unroll
        for (int e = 0; e < E; e += 4) dst[e / 4] = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
      }
    }
  }
}

// ---- rows form -------------------------------------------------------------

constexpr int kRowsPages = 512;

template <int D, bool FP8, int RT>
struct RowsSmem {
  static constexpr int STAGES = FP8 ? 2 : 3;
  static constexpr int COLS = 64 * RT;
  __attribute__((aligned(16))) uint16_t stage[STAGES * KeyStage<D>::kStage];
  union {
    unsigned long long mask[COLS];
    int token[COLS];  // of a prefix's columns, which have no drafts to see
  };
  int row[COLS];
  int sum[kWaves];
  int odd[kWaves];
  int page[kRowsPages];                 // page ids, of so many pages at a time
  float2 scale[FP8 ? kRowsPages : 1];   // their K scales (times qk_scale) and V scales
};

// One block of 32 staged keys, two halves of 16 with score scales km and V
// scales vs (fp8 pages), of which the first n0 and n1 keys count; DRAFTS: those
// whose bit of `seen` is set. pop: the rounded probabilities. The mask of a
// ragged block is a branch of its own after the products: a second copy of the
// whole for it has its LDS reads hoisted and spills 80 registers.
template <int D, bool FP8, int RT, bool DRAFTS>
__device__ __forceinline__ void add_rows(const uint16_t* kst, const float (&km)[2], const float (&vs)[2], int n0, int n1,
                                         const uint32_t (&seen)[RT], const bf16x8_t (&qop)[RT][D / 32],
                                         State<D, RT>& st, bf16x4_t (&pop)[RT][2]) {
  using L = KeyStage<D>;
  constexpr int KB = D / 32, DT = D / 16;
  constexpr bool SCALED = FP8 && !DRAFTS;
  const int lane = threadIdx.x & 63, r16 = lane & 15, quad = lane >> 4;
  f32x4_t s[RT][2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    bf16x8_t kop[KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
      kop[kb] = *reinterpret_cast<const bf16x8_t*>(kst + L::row(r16) + L::row(i * 16) + kb * 32 + quad * 8);
#pragma unroll
    for (int t = 0; t < RT; ++t) s[t][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int t = 0; t < RT; ++t) s[t][i] = mfma16x16x32(kop[kb], qop[t][kb], s[t][i]);
  }
  const uint16_t* vtr = kst + L::kElems + L::row(quad * 4 + r16 / 4) + 4 * (r16 % 4);
  const auto read_vop = [&](int dt) __attribute__((always_inline)) {
    const bf16x4_t v0 = lds_read_tr(vtr + dt * 16);
    const bf16x4_t v1 = lds_read_tr(vtr + L::row(16) + dt * 16);
    return __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  // With one tile there are registers to request V ahead of the softmax.
  bf16x8_t vpre[DT];
  if constexpr (RT == 1) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) vpre[dt] = read_vop(dt);
    __builtin_amdgcn_sched_barrier(0);
  }
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[t][i][e] = fmaf(s[t][i][e], km[i], st.neg[t]);
        if constexpr (DRAFTS) s[t][i][e] = seen[t] >> (i * 16 + quad * 4 + e) & 1 ? s[t][i][e] : -INFINITY;
      }
  if (!DRAFTS && n0 + n1 < 2 * kPage) {
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[t][0][e] = quad * 4 + e < n0 ? s[t][0][e] : -INFINITY;
        s[t][1][e] = quad * 4 + e < n1 ? s[t][1][e] : -INFINITY;
      }
  }
#pragma unroll
  for (int t = 0; t < RT; ++t) softmax_step<D, RT, 2, SCALED>(st, t, s[t], vs, pop[t], [] {});
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) {
    const bf16x8_t vo = RT == 1 ? vpre[dt] : read_vop(dt);
#pragma unroll
    for (int t = 0; t < RT; ++t)
      st.o[t][dt] =
          mfma16x16x32(vo, __builtin_shufflevector(pop[t][0], pop[t][1], 0, 1, 2, 3, 4, 5, 6, 7), st.o[t][dt]);
  }
}

// A workgroup barrier behind this wave's LDS accesses that leaves its loads in
// flight (__syncthreads waits for those too).
__device__ inline void block_sync() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory"); }

// A unit: rows sm.row, RT tiles for each wave. Waves without rows only copy.
template <int D, bool FP8, int RT>
__device__ __forceinline__ void rows_unit(const TreeArgs& a, const Keys& k, int h, long long part,
                                          RowsSmem<D, FP8, RT>& sm) {
  using L = KeyStage<D>;
  constexpr int KB = D / 32, DT = D / 16, STAGES = RowsSmem<D, FP8, RT>::STAGES;
  constexpr int ROW_BYTES = D * (FP8 ? 1 : 2), BLOCK_BYTES = kPage * ROW_BYTES;
  const int tid = threadIdx.x, lane = tid & 63, r16 = lane & 15, quad = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int Hkv = a.num_kv_heads, pages = k.pages_a + k.pages_b;
  const int c0 = wave * RT * 16;
  const bool active = __builtin_amdgcn_readfirstlane(sm.row[c0]) >= 0;

  bf16x8_t qop[RT][KB];
  State<D, RT> st;
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int row = sm.row[c0 + t * 16 + r16];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
      qop[t][kb] = __builtin_bit_cast(bf16x8_t, piece(a.q + (size_t)max(row, 0) * D + kb * 32 + quad * 8, row >= 0));
  }
  st.clear();
  const uint32_t none[RT] = {};
  bf16x4_t pop[RT][2];

#pragma unroll 1
  for (int w0 = 0; w0 < pages; w0 += kRowsPages) {
    const int np = min(pages - w0, kRowsPages), nblk = cdiv(np, 2);
    if (w0 > 0) __syncthreads();  // the pages before have been read
    for (int i = tid; i < np; i += 64 * kWaves) {
      const int b = w0 + i;
      const int page = clamp_page(b < k.pages_a ? k.table_a[b] : k.table_b[b - k.pages_a], a.num_pages);
      sm.page[i] = page;
      if constexpr (FP8) {
        const size_t at = (size_t)page * Hkv + h;
        sm.scale[i] = make_float2(a.k_scale[at] * a.qk_scale, a.v_scale[at]);
      }
    }
    // The compiler's wait for the q rows belongs here: inside the loop it would
    // drain the copies in flight.
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) asm volatile("" : "+v"(qop[t][kb]));
    __syncthreads();
    const auto block = [&](int p) __attribute__((always_inline)) {
      return ((size_t)sm.page[min(p, np - 1)] * Hkv + h) * BLOCK_BYTES;
    };
    const auto valid = [&](int p) __attribute__((always_inline)) {
      const int b = w0 + p;
      const int left = b < k.pages_a ? k.tokens_a - b * kPage : k.tokens_b - (b - k.pages_a) * kPage;
      return p < np ? min(left, kPage) : 0;
    };
    const char* kpool = static_cast<const char*>(a.k_pages);
    const char* vpool = static_cast<const char*>(a.v_pages);
    const auto compute = [&](int blk, const uint16_t* kst) __attribute__((always_inline)) {
      const int n0 = valid(2 * blk), n1 = valid(2 * blk + 1);
      float km[2], vs[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float2 x = FP8 ? sm.scale[min(2 * blk + i, np - 1)] : make_float2(a.qk_scale, 1.f);
        km[i] = x.x;
        vs[i] = x.y;
      }
      if (active) add_rows<D, FP8, RT, false>(kst, km, vs, n0, n1, none, qop, st, pop);
    };

    if constexpr (!FP8) {
      // Direct copies, STAGES - 1 blocks ahead, one barrier per block.
      constexpr int CPW = L::kChunks / kWaves, HALF = L::kRows / 2;  // chunks per wave, slots per page
      const int slot_ = lane / (D / 8);
      const uint32_t in_page = (uint32_t)(((slot_ % HALF) * L::kChunks + wave * CPW) * ROW_BYTES + lane % (D / 8) * 16);
      const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint16_t*)sm.stage;
      const auto request = [&](int blk, int stage) __attribute__((always_inline)) {
        const size_t off = block(2 * blk + (slot_ >= HALF ? 1 : 0)) + in_page;
        const uint32_t to = lds0 + (uint32_t)((stage * L::kStage + wave * CPW * L::kPitch) * 2);
#pragma unroll
        for (int i = 0; i < CPW; ++i) copy_to_lds(to + i * L::kPitch * 2, kpool + off + i * ROW_BYTES);
#pragma unroll
        for (int i = 0; i < CPW; ++i) copy_to_lds(to + (L::kElems + i * L::kPitch) * 2, vpool + off + i * ROW_BYTES);
      };
      request(0, 0);
      if (nblk > 1) request(1, 1);
      int cur = 0;
      for (int blk = 0; blk < nblk; ++blk) {
        if ((STAGES == 3 || blk == 0) && blk + 1 < nblk) wait_copies<L::kPerWave>();
        else wait_copies<0>();
        if ((STAGES == 3 || blk > 0) && blk + STAGES - 1 < nblk) request(blk + STAGES - 1, cur == 0 ? STAGES - 1 : cur - 1);
        uint16_t* kst = sm.stage + cur * L::kStage;
        const int n0 = valid(2 * blk), n1 = valid(2 * blk + 1);
        if (n0 + n1 < 2 * kPage) {  // padding rows may hold anything
          for (int i = tid; i < kKeyBlk * (D / 8); i += 64 * kWaves) {
            const int r = i / (D / 8);
            if (r % kPage >= (r < kPage ? n0 : n1))
              *reinterpret_cast<u32x4_t*>(kst + L::kElems + L::row(r) + i % (D / 8) * 8) = u32x4_t{0, 0, 0, 0};
          }
          __syncthreads();
        }
        compute(blk, kst);
        cur = cur == STAGES - 1 ? 0 : cur + 1;
      }
    } else {
      // Codes go through registers, where they are decoded: 16 bytes of K and
      // of V for each thread (64-wide heads: of one of them).
      constexpr int TPR = D / 16;  // threads per row
      constexpr int DEPTH = 3;  // blocks requested ahead
      const int part = tid % (kKeyBlk * TPR), r = part / TPR, col = part % TPR * 16;
      const bool only_v = D == 64 && tid >= kKeyBlk * TPR;
      u32x4_t ahead[DEPTH][D / 64];
      const auto load = [&](int blk, u32x4_t (&x)[D / 64]) __attribute__((always_inline)) {
        const size_t off = block(2 * blk + (r >= kPage ? 1 : 0)) + (uint32_t)(r % kPage * ROW_BYTES + col);
        x[0] = *reinterpret_cast<const u32x4_t*>((only_v ? vpool : kpool) + off);
        if constexpr (D == 128) x[1] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(vpool + off));
      };
#pragma unroll
      for (int d = 0; d < DEPTH; ++d) load(d, ahead[d]);
      const auto step = [&](int blk, u32x4_t (&x)[D / 64]) __attribute__((always_inline)) {
        uint16_t* kst = sm.stage + (blk & 1) * L::kStage;
        const bool ok = r % kPage < (r < kPage ? valid(2 * blk) : valid(2 * blk + 1));
#pragma unroll
        for (int i = 0; i < D / 64; ++i) {
          u32x4_t* dst = reinterpret_cast<u32x4_t*>(kst + (only_v || i == 1 ? L::kElems : 0) + L::row(r) + col);
          store_decoded(dst, ok ? x[i] : u32x4_t{0, 0, 0, 0}, tid & 1);
        }
        load(blk + DEPTH, x);
        block_sync();  // the block is there, and the one before has been read
        compute(blk, kst);
      };
      // Whole rounds without a branch between the steps: the compiler's wait
      // for a step's loads then leaves the later ones in flight.
      int blk = 0;
      for (; blk + DEPTH <= nblk; blk += DEPTH) {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) step(blk + d, ahead[d]);
      }
#pragma unroll
      for (int d = 0; d < DEPTH - 1; ++d)
        if (blk + d < nblk) step(blk + d, ahead[d]);
    }
  }

  // The drafts, 32 at a time.
  for (int u0 = 0; u0 < k.drafts; u0 += kKeyBlk) {
    const int nv = min(k.drafts - u0, kKeyBlk);
    const size_t first = ((size_t)(k.draft0 + u0) * Hkv + h) * D, stride = (size_t)Hkv * D;
    constexpr int PER = kKeyBlk * (D / 8) / (64 * kWaves);  // pieces per thread
    u32x4_t kx[PER], vx[PER];
    bool bad[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int i = j * 64 * kWaves + tid, r = i / (D / 8), col = i % (D / 8) * 8;
      kx[j] = piece(a.k_draft + first + r * stride + col, r < nv);
      vx[j] = piece(a.v_draft + first + r * stride + col, r < nv);
    }
    __syncthreads();  // the stages have been read
    int odd = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int i = j * 64 * kWaves + tid, r = i / (D / 8), col = i % (D / 8) * 8;
      constexpr int LPT = D / 8, TPL = 64 / LPT;  // lanes per draft, drafts per wave and load
      bad[j] = not_finite(vx[j].x) || not_finite(vx[j].y) || not_finite(vx[j].z) || not_finite(vx[j].w);
      const unsigned long long w = __ballot(bad[j]);
      bool drop = false;
      if (w != 0) {
#pragma unroll
        for (int b = 0; b < TPL; ++b) {
          const bool is = (w >> (b * LPT) & ((1ull << LPT) - 1)) != 0;
          drop = drop || (is && lane / LPT == b);
          odd |= is ? 1 << (j * 64 * kWaves / LPT + wave * TPL + b) : 0;
        }
      }
      *reinterpret_cast<u32x4_t*>(sm.stage + L::row(r) + col) = kx[j];
      *reinterpret_cast<u32x4_t*>(sm.stage + L::kElems + L::row(r) + col) = drop ? u32x4_t{0, 0, 0, 0} : vx[j];
    }
    if (lane == 0) sm.odd[wave] = odd;
    __syncthreads();
    odd = sm.odd[0] | sm.odd[1] | sm.odd[2] | sm.odd[3];
    if (active) {
      const uint32_t in_tree = nv == 32 ? 0xFFFFFFFFu : (1u << nv) - 1;
      uint32_t seen[RT];
#pragma unroll
      for (int t = 0; t < RT; ++t) seen[t] = (uint32_t)(sm.mask[c0 + t * 16 + r16] >> u0) & in_tree;
      const float km[2] = {a.qk_scale, a.qk_scale}, vs[2] = {1.f, 1.f};
      add_rows<D, FP8, RT, true>(sm.stage, km, vs, 0, 0, seen, qop, st, pop);
      // V rows with an infinity or NaN, for the rows that see them alone: a
      // weight of zero would not hide them in the product.
      while (odd != 0) {
        const int u = __builtin_amdgcn_readfirstlane(__builtin_ctz(odd));
        odd &= odd - 1;
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          const uint2 w0 = __builtin_bit_cast(uint2, pop[t][0]), w1 = __builtin_bit_cast(uint2, pop[t][1]);
          const uint32_t word = u & 16 ? (u & 2 ? w1.y : w1.x) : (u & 2 ? w0.y : w0.x);
          const float p = __shfl(u & 1 ? bf16_hi(word) : bf16_lo(word), (u >> 2 & 3) * 16 + r16);
          const bool ok = seen[t] >> u & 1;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) {
            const uint2 x = *reinterpret_cast<const uint2*>(a.v_draft + first + u * stride + dt * 16 + quad * 4);
            const float v[4] = {bf16_lo(x.x), bf16_hi(x.x), bf16_lo(x.y), bf16_hi(x.y)};
#pragma unroll
            for (int e = 0; e < 4; ++e) st.o[t][dt][e] = ok ? fmaf(p, v[e], st.o[t][dt][e]) : st.o[t][dt][e];
          }
        }
      }
    }
  }

  if (!active) return;
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const float l = xor_sum_from<16>(st.l[t]);
    const float r = xor_sum_from<16>(st.r[t]);
    store_row<D>(a, sm.row[c0 + t * 16 + r16], part, quad, st.o[t], r == 0.f ? 0.f : 1.f / r,
                 l == 0.f ? -INFINITY : (fast_log2(l) - st.neg[t]) * kLn2);
  }
}

// ---- units -------------------------------------------------------------------

__device__ inline int2 drafts_of(const TreeArgs& a, int s) {
  const int t0 = min(max(a.draft_offs[s], 0), a.num_drafts);
  return make_int2(t0, min(max(a.draft_offs[s + 1] - t0, 0), min(a.max_drafts, a.num_drafts - t0)));
}

// Columns c0 .. of the drafts of group g, in sequence order: the tokens are
// found by a scan over the sequences' groups and tree sizes. Returns whether
// there are any.
template <int D, bool FP8, int RT>
__device__ bool group_columns(const TreeArgs& a, int g, int h, int c0, RowsSmem<D, FP8, RT>& sm) {
  constexpr int COLS = RowsSmem<D, FP8, RT>::COLS;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int k0 = c0 >> a.rep_shift, k1 = (c0 + COLS) >> a.rep_shift;
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
  if (tid < COLS) {
    const int c = c0 + tid, rank = c >> a.rep_shift;
    const int rep = c & ((1 << a.rep_shift) - 1);
    sm.row[tid] = rank < carry ? sm.token[rank - k0] * a.num_q_heads + (h << a.rep_shift) + rep : -1;
  }
  __syncthreads();
  return true;
}

// Row blocks of one unit follow each other on one XCD (workgroups are dealt to
// the 8 of them in turn), whose L2 then has the K and V that the first read.
__device__ inline void locate(int id, int repeats, int& u, int& r) {
  const int row = id / (8 * repeats), k = id - row * (8 * repeats);
  r = k / 8;
  u = row * 8 + k % 8;
}

// Pages of each of `count` pieces of `pages` pages, or of fewer.
__device__ inline int piece_pages(long long pages, int count) {
  return max((int)min((pages + count - 1) / count + 15, 1ll << 30) & ~15, kTreeLeastPages);
}

// Workgroup `id` of the group prefixes: (group, chunk of pages, kv-head), each
// several times where a group has many rows.
template <int D, bool FP8, int RT>
__device__ __forceinline__ void prefix_units(const TreeArgs& a, int id, RowsSmem<D, FP8, RT>& sm) {
  int u, z;
  locate(id, a.prefix_repeats, u, z);
  const int Hkv = a.num_kv_heads;
  if (u >= a.num_groups * a.max_prefix_chunks * Hkv) return;
  const int h = u % Hkv, chunk = u / Hkv % a.max_prefix_chunks, g = u / Hkv / a.max_prefix_chunks;
  const int P = clamp_len(a.prefix_lens[g], a.max_prefix_pages);
  const int each = piece_pages(cdiv(P, kPage), a.max_prefix_chunks), first = chunk * each;
  const int pages = min(cdiv(P, kPage) - first, each);
  if (pages <= 0) return;
  Keys k = {};
  k.table_a = k.table_b = a.prefix_block_table + (size_t)g * a.max_prefix_pages + first;
  k.pages_a = pages;
  k.tokens_a = P - first * kPage;
  for (int rb = z; group_columns<D, FP8, RT>(a, g, h, rb * RowsSmem<D, FP8, RT>::COLS, sm); rb += a.prefix_repeats)
    rows_unit<D, FP8, RT>(a, k, h, (long long)chunk * a.num_drafts * a.num_q_heads, sm);
}

// Pages that the units of sequence s walk: its response's, behind its group's
// prefix where that is not shared.
struct SeqPages {
  int group, prefix, prefix_tokens, resp, resp_tokens;
};
__device__ inline SeqPages seq_pages(const TreeArgs& a, int s) {
  const int g = clamp_group(a.seq_to_group[s], a.num_groups);
  const int L = clamp_len(a.resp_lens[s], a.max_resp_pages);
  const int P = clamp_len(a.prefix_lens[g], a.max_prefix_pages);
  return SeqPages{g, cdiv(P, kPage), P, cdiv(L, kPage), L};
}

// A piece of a sequence: pieces are cut from its end, `each` pages long, so its
// first piece (0) is the short one; it also takes the drafts. extra0: the place
// of piece 1 among all such pieces.
struct Place {
  int s, piece, pieces, each, extra0;
  SeqPages n;
  int2 drafts;
};
struct OrderSmem {
  float sum[kWaves];
  int most[kWaves], wave[kTreeOrderSeqs / 256][kWaves], count[64], start[64], bucket;
  Place place;
};
__device__ inline int wave_max(int x) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) x = max(x, __shfl_xor(x, o));
  return x;
}
__device__ inline float wave_sum(float x) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) x += __shfl_xor(x, o);
  return x;
}
// The sum of x over this lane and those before it.
__device__ inline int wave_scan(int x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o);
    x += lane >= o ? y : 0;
  }
  return x;
}

// Pages of a piece, from the longest sequence and the pages of all: the longest
// sequence over seq_pieces, for few sequences to fill the chip, but at most
// piece_share of all, so that a long one among short ones is divided, for which
// pieces go no lower than least_pages. At most max_extra pieces besides the
// sequences' first ones come of it; the share is rounded up by more than the
// error of the sum for that.
__device__ inline int seq_piece_pages(const TreeArgs& a, int most, float sum) {
  const int share = (int)fminf(sum * a.piece_share * 1.0001f + 1.f, 1e9f);
  return min(piece_pages(most, a.seq_pieces), piece_pages(max(share, a.least_pages), 1));
}

// Place u of the sequences' pieces, found by every workgroup from all lengths
// (a table's width says little about those): the pieces besides the first ones,
// all of one length, then the first pieces, where longest_first says so the
// longer before the shorter. Returns false behind the last. The workgroup's LDS
// is not in use yet. It takes about 1 us, which calls that need none of it are
// spared; one wave that does it alone for up to 64 sequences is no faster and
// costs registers.
__device__ bool find_piece(const TreeArgs& a, int u, OrderSmem& m, Place& x) {
  if (a.max_extra == 0 && a.longest_first == 0) {
    if (u >= a.num_seqs) return false;
    x = Place{u, 0, 1, 0, 0, seq_pages(a, u), drafts_of(a, u)};
    return x.drafts.y > 0;
  }
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  constexpr int PER = kTreeOrderSeqs / (64 * kWaves);
  SeqPages n[PER];
  int2 dr[PER];
  int total[PER], most = 0;  // total: pages, -1: without drafts
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int s = i * 64 * kWaves + tid;
    total[i] = -1;
    if (s < a.num_seqs) {
      dr[i] = drafts_of(a, s);
      n[i] = seq_pages(a, s);
      if (dr[i].y > 0) total[i] = n[i].resp + (a.share ? 0 : n[i].prefix);
    }
    most = max(most, total[i]);
    sum += (float)max(total[i], 0);
  }
  most = wave_max(most);
  sum = wave_sum(sum);
  if (lane == 0) m.most[wave] = most, m.sum[wave] = sum;
  if (tid < 64) m.count[tid] = 0;
  __syncthreads();
  sum = 0.f;
  for (int w = 0; w < kWaves; ++w) most = max(most, m.most[w]), sum += m.sum[w];
  const int each = seq_piece_pages(a, most, sum);

  // The pieces besides the first ones, and the sequences, before each sequence.
  int extra[PER], before[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    extra[i] = total[i] <= each ? 0 : (total[i] - 1) / each;
    const int y = extra[i] << 16 | (total[i] >= 0 ? 1 : 0), z = wave_scan(y);
    if (lane == 63) m.wave[i][wave] = z;
    before[i] = z - y;
  }
  __syncthreads();
  int all = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i)
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      if (w == wave) before[i] += all;
      all += m.wave[i][w];
    }
  const int extras = all >> 16, seqs = all & 0xffff;

  const auto take = [&](int i, int piece) __attribute__((always_inline)) {
    m.place = Place{i * 64 * kWaves + tid, piece, 1 + extra[i], each, before[i] >> 16, n[i], dr[i]};
  };
  if (u < extras) {
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if ((unsigned)(u - (before[i] >> 16)) < (unsigned)extra[i]) take(i, 1 + u - (before[i] >> 16));
  } else {
    int rank = u - extras;
    if (rank >= a.num_seqs) return false;
    if (a.longest_first > 0 && rank >= a.longest_first) rank = a.num_seqs - 1 - (rank - a.longest_first);
    if (rank >= seqs) return false;
    if (a.longest_first == 0) {
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (total[i] >= 0 && (before[i] & 0xffff) == rank) take(i, 0);
    } else {
      // Sorted by counting, to 1/64 of the longest, then in order.
      int bucket[PER];
      const int longest = max(min(most, each), 1);
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        bucket[i] = -1;
        if (total[i] >= 0) {
          bucket[i] = 63 - (int)((long long)(total[i] - extra[i] * each) * 63 / longest);
          atomicAdd(&m.count[bucket[i]], 1);
        }
      }
      __syncthreads();
      if (tid < 64) {
        const int c = m.count[tid], z = wave_scan(c);
        m.start[tid] = z - c;
        if (z - c <= rank && rank < z) m.bucket = tid;
      }
      __syncthreads();
      const int mine = m.bucket;
      int left = rank - m.start[mine];
      unsigned long long in[PER];
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        in[i] = __ballot(bucket[i] == mine);
        if (lane == 0) m.wave[i][wave] = __popcll(in[i]);
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < PER; ++i)
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          if (w == wave && bucket[i] == mine && __popcll(in[i] & ((1ull << lane) - 1)) == left) take(i, 0);
          left -= m.wave[i][w];
        }
    }
  }
  __syncthreads();
  // The same for all lanes: into scalar registers.
  static_assert(sizeof(Place) % sizeof(int) == 0, "read word by word");
  union {
    Place place;
    int word[sizeof(Place) / sizeof(int)];
  } y = {m.place};
#pragma unroll
  for (int& w : y.word) w = __builtin_amdgcn_readfirstlane(w);
  x = y.place;
  __syncthreads();
  return true;
}

// Unit u of the sequences, its columns from c0 on: a place of the pieces and a
// kv-head. Returns false where there is nothing to do.
struct SeqUnit {
  Keys k;
  int h, token0, tokens;
  long long part;
};
__device__ inline bool seq_unit(const TreeArgs& a, int u, int c0, bool note, OrderSmem& order, SeqUnit& x) {
  Place p;
  if (!find_piece(a, u / a.num_kv_heads, order, p)) return false;
  x.h = u % a.num_kv_heads;
  x.token0 = p.drafts.x;
  x.tokens = p.drafts.y;
  if (c0 >= x.tokens << a.rep_shift) return false;
  const SeqPages& n = p.n;
  const int before = a.share ? 0 : n.prefix, total = before + n.resp;
  const int first = p.piece == 0 ? 0 : total - (p.pieces - p.piece) * p.each;
  const int end = total - (p.pieces - 1 - p.piece) * p.each;
  const int chunks = a.share ? cdiv(n.prefix, piece_pages(n.prefix, a.max_prefix_chunks)) : 0;
  const int a0 = min(first, before), b0 = max(first - before, 0);
  Keys k = {};
  k.table_a = a.prefix_block_table + (size_t)n.group * a.max_prefix_pages + a0;
  k.pages_a = min(end, before) - a0;
  k.tokens_a = n.prefix_tokens - a0 * kPage;
  k.table_b = a.resp_block_table + (size_t)p.s * a.max_resp_pages + b0;
  k.pages_b = max(end - before, 0) - b0;
  k.tokens_b = n.resp_tokens - b0 * kPage;
  const bool final = chunks + p.pieces == 1;
  x.part = kFinal;
  if (!final && p.piece == 0) x.part = (long long)a.max_prefix_chunks * a.num_drafts * a.num_q_heads;
  if (p.piece > 0)
    x.part = a.pieces_at + ((long long)(p.extra0 + p.piece - 1) * a.num_kv_heads + x.h) * a.slot_rows -
             (((long long)x.h * a.num_drafts + x.token0) << a.rep_shift);
  // Rows whose result is stored at once have no partial results to merge.
  if (note && a.token_parts != nullptr && p.piece == 0 && x.h == 0 && c0 == 0)
    for (int i = threadIdx.x & 63; i < x.tokens; i += 64)
      a.token_parts[x.token0 + i] = make_int2(final ? 0 : p.pieces | i << 16, chunks | p.extra0 << 16);
  if (p.piece == 0) {
    k.draft0 = x.token0;
    k.drafts = x.tokens;
  }
  x.k = k;
  return true;
}
__device__ inline int column_row(const TreeArgs& a, const SeqUnit& x, int c) {
  const int t = c >> a.rep_shift;
  return t < x.tokens ? (x.token0 + t) * a.num_q_heads + (x.h << a.rep_shift) + (c & ((1 << a.rep_shift) - 1)) : -1;
}
__device__ inline unsigned long long column_mask(const TreeArgs& a, const SeqUnit& x, int c) {
  const int t = c >> a.rep_shift;
  return t < x.tokens && x.k.drafts > 0 ? a.masks[x.token0 + t] : 0;
}

// Bound by the reads of the cache: 256 sequences of 8 drafts over 64 to 512 +
// U[0, 4096] tokens (Hkv 8, d 128) 2.21 GB in 380 us, 5.8 TB/s, of the 7.0 that
// one large read reaches; 64 fp8 sequences of 1 to 32 drafts over 8192 to 32768
// tokens 2.70 GB in 540 to 590 us, 4.6 to 5.0 TB/s, with decoding and the softmax
// of four tiles between the reads (vector units 42% busy, matrix units 19%). Four
// tiles of 128-wide heads take all 256 registers and spill 28 bytes a lane (fp8:
// 12). Small calls are latency: lengths, then page ids, then pages, 7 us for 4
// sequences of 180 tokens.
template <int D, bool FP8, int CT>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2, 8)))
void tree_split_kernel(const TreeArgs a) {
  __shared__ union U {
    Smem<D, FP8, CT> split;
    Smem<D, FP8, 2> few;
    RowsSmem<D, FP8, 1> rows;
    OrderSmem order;
    __device__ U() {}
  } sm;
  int id = blockIdx.x;
  if (id < a.prefix_blocks) {
    prefix_units<D, FP8, 1>(a, id, sm.rows);
    return;
  }
  id -= a.prefix_blocks;
  int u, rb;
  locate(id, a.row_blocks, u, rb);
  SeqUnit x;
  const int c0 = rb * 16 * CT;
  if (!seq_unit(a, u, c0, threadIdx.x < 64, sm.order, x)) return;
  const auto take = [&](auto& m) __attribute__((always_inline)) {
    constexpr int COLS = sizeof(m.row) / sizeof(int);
    if ((int)threadIdx.x < COLS) {
      m.row[threadIdx.x] = column_row(a, x, c0 + threadIdx.x);
      m.mask[threadIdx.x] = column_mask(a, x, c0 + threadIdx.x);
    }
    __syncthreads();
    split_unit<D, FP8, COLS / 16>(a, x.k, x.h, x.part, m);
  };
  if (CT > 2 && (x.tokens << a.rep_shift) - c0 <= 32) take(sm.few);
  else take(sm.split);
}

// Bound by the chain of scores, softmax and products that each wave waits for, with
// two waves per SIMD (236 registers): 32 sequences of 64 drafts with 8 query heads
// per kv-head over 1024 + U[0, 2048] tokens (Hkv 4, d 128) 69 GFLOP in 103 to 105
// us among others of their kind, 660 TFLOP/s, of the 1170 to 1220 of a large
// product, and 117 to 121 apart under a kernel trace; matrix units 25% busy, vector
// units 30%.
template <int D, bool FP8, int RT>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2, 8)))
void tree_rows_kernel(const TreeArgs a) {
  __shared__ union U {
    RowsSmem<D, FP8, RT> rows;
    OrderSmem order;
    __device__ U() {}
  } u_;
  RowsSmem<D, FP8, RT>& sm = u_.rows;
  constexpr int COLS = RowsSmem<D, FP8, RT>::COLS;
  int id = blockIdx.x;
  if (id < a.prefix_blocks) {
    prefix_units<D, FP8, RT>(a, id, sm);
    return;
  }
  id -= a.prefix_blocks;
  int u, rb;
  locate(id, a.row_blocks, u, rb);
  SeqUnit x;
  const int c0 = rb * COLS;
  if (!seq_unit(a, u, c0, threadIdx.x < 64, u_.order, x)) return;
  for (int i = threadIdx.x; i < COLS; i += 64 * kWaves) {
    sm.row[i] = column_row(a, x, c0 + i);
    sm.mask[i] = column_mask(a, x, c0 + i);
  }
  __syncthreads();
  rows_unit<D, FP8, RT>(a, x.k, x.h, x.part, sm);
}

template <int N>
struct Batch {
  static constexpr int value = N;
};

// Merges the partial results of every row:
//   lse = ln sum_i exp(lse_i),  out = sum_i exp(lse_i - lse) o_i
// over the row's parts that are not empty (lse_i = -inf), as one pass with a
// running maximum. D / 4 lanes hold a row; rows in the order of the parts. Bound
// by latency: the token's parts, then the parts, 4.8 us for 136 tokens of 16
// heads with 1 to 4 parts, 3 to 4 us where no row has any.
template <int D>
__global__ __launch_bounds__(256) void tree_merge_kernel(const TreeArgs a) {
  constexpr int LPR = D / 4;
  const long long rows = (long long)a.num_drafts * a.num_q_heads;
  const long long i = ((long long)blockIdx.x * 256 + threadIdx.x) / LPR;
  if (i >= rows) return;
  const int per_head = a.num_drafts << a.rep_shift;
  const int h = (int)(i / per_head), c = (int)(i - (long long)h * per_head), t = c >> a.rep_shift;
  if (t >= a.draft_offs[a.num_seqs]) return;  // behind the last sequence
  const int2 p = a.token_parts[t];
  if ((p.x & 0xffff) == 0) return;  // stored already
  const int sub = threadIdx.x % LPR, chunks = min(p.y & 0xffff, a.max_prefix_chunks);
  const int extra0 = min((int)((unsigned)p.y >> 16), a.max_extra);
  const int n = chunks + 1 + min((p.x & 0xffff) - 1, a.max_extra - extra0);
  const long long stride = (long long)a.num_kv_heads * a.slot_rows;
  const int own = min((int)((unsigned)p.x >> 16), a.max_drafts - 1);
  const long long extra = a.pieces_at + (long long)h * a.slot_rows + (extra0 - chunks - 1) * stride +
                          (own << a.rep_shift) + (c & ((1 << a.rep_shift) - 1));
  // Part k: a prefix chunk, the first piece, another piece.
  const auto place = [&](int k) {
    return k <= chunks ? (k < chunks ? k : a.max_prefix_chunks) * rows + i : extra + k * stride;
  };
  const f32x4_t* o = reinterpret_cast<const f32x4_t*>(a.part_o) + sub;
  float m = -INFINITY, w = 0.f;
  f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
  int k = 0;
  const auto step = [&](auto batch) __attribute__((always_inline)) {
    constexpr int B = decltype(batch)::value;
    float l[B];
    f32x4_t x[B];
#pragma unroll
    for (int b = 0; b < B; ++b) {
      const long long at = place(min(k + b, n - 1));
      l[b] = a.part_lse[at];
      x[b] = o[at * LPR];
    }
    float top = m;
#pragma unroll
    for (int b = 0; b < B; ++b) {
      if (k + b >= n) l[b] = -INFINITY;
      top = fmaxf(top, l[b]);
    }
    const float f = m == top ? 1.f : fast_exp2((m - top) * kLog2e);
    w *= f;
    acc *= f;
#pragma unroll
    for (int b = 0; b < B; ++b) {
      if (l[b] == -INFINITY) continue;
      const float e = l[b] == top ? 1.f : fast_exp2((l[b] - top) * kLog2e);
      w += e;
      acc += e * x[b];
    }
    m = top;
    k += B;
  };
  // So many parts requested at once (one sequence of 16000 tokens, 33 parts:
  // 7.6 us, by fours 9.4).
  while (n - k > 4) step(Batch<8>{});
  if (k < n) step(Batch<4>{});
  const float inv = w == 0.f ? 0.f : 1.f / w;
  const size_t row = (size_t)t * a.num_q_heads + ((size_t)h << a.rep_shift) + (c & ((1 << a.rep_shift) - 1));
  acc *= inv;
  *reinterpret_cast<uint2*>(a.out + row * D + sub * 4) = make_uint2(pack_bf16x2(acc[0], acc[1]), pack_bf16x2(acc[2], acc[3]));
  if (a.lse != nullptr && sub == 0) a.lse[row] = w == 0.f ? -INFINITY : m + fast_log2(w) * kLn2;
}

template <int D, bool FP8>
hipError_t by_form(const TreeArgs& a, TreeForm form, unsigned blocks, hipStream_t st) {
  const dim3 grid(blocks), threads(64 * kWaves);
  switch (form) {
    case TreeForm::kSplit1: tree_split_kernel<D, FP8, 1><<<grid, threads, 0, st>>>(a); break;
    case TreeForm::kSplit2: tree_split_kernel<D, FP8, 2><<<grid, threads, 0, st>>>(a); break;
    case TreeForm::kSplit4: tree_split_kernel<D, FP8, 4><<<grid, threads, 0, st>>>(a); break;
    case TreeForm::kRows: tree_rows_kernel<D, FP8, 2><<<grid, threads, 0, st>>>(a); break;
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_tree_merge(const TreeArgs& a, int head_dim, hipStream_t stream) {
  const long long threads = (long long)a.num_drafts * a.num_q_heads * (head_dim / 4), blocks = (threads + 255) / 256;
  if (blocks <= 0) return hipSuccess;
  if (blocks > kMaxBlocks256) return hipErrorInvalidValue;
  if (head_dim == 128) tree_merge_kernel<128><<<(unsigned)blocks, 256, 0, stream>>>(a);
  else tree_merge_kernel<64><<<(unsigned)blocks, 256, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_tree_attn(const TreeArgs& a, int head_dim, bool fp8, TreeForm form, long long blocks,
                            hipStream_t stream) {
  if (blocks <= 0) return hipSuccess;
  if (blocks > kMaxBlocks256) return hipErrorInvalidValue;
  const unsigned n = (unsigned)blocks;
  if (head_dim == 128) return fp8 ? by_form<128, true>(a, form, n, stream) : by_form<128, false>(a, form, n, stream);
  if (head_dim == 64) return fp8 ? by_form<64, true>(a, form, n, stream) : by_form<64, false>(a, form, n, stream);
  return hipErrorInvalidValue;
}

}  // namespace rp
