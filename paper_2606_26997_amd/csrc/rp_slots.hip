// Writes into the paged cache by slot, and the tables that the slots come from.
//
// rp_kv_write_slots: row i of a list goes to slot page * 16 + row. bf16 pools
// copy. fp8 pools keep one scale per (page, kv-head) for K and for V, so the
// entries of a page are handled together: a run is a maximal stretch of the
// list whose slots follow each other inside one page, and one wave takes a run
// of one kv-head's K or V: amax over the run's rows, one scale, one rounding.
//
// rp_page_tables_resize: two exclusive prefix sums over the sequences (pages
// given back, pages taken) say where each page of a block table goes on, or
// comes from, the stack of free pages.
#include "rp_device.h"
#include "rp_internal.h"

#pragma clang fp contract(off)

namespace rp {
namespace {

constexpr int kWriteThreads = 256;

// Slot of list entry i and the row that goes there; false: nothing to write.
__device__ inline bool entry(const WriteArgs& a, long long i, int& slot, int& src) {
  slot = a.slot_map[i];
  src = a.src_rows != nullptr ? a.src_rows[i] : (int)i;
  return (unsigned)slot < (unsigned)a.num_slots && (unsigned)src < (unsigned)a.num_src;
}

template <int D>
__global__ __launch_bounds__(kWriteThreads) void write_bf16_kernel(const WriteArgs a) {
  constexpr int CPR = D / 8;  // 16-byte pieces per row
  const int per_token = 2 * a.num_kv_heads * CPR;
  const long long n = (long long)blockIdx.x * kWriteThreads + threadIdx.x;
  const long long i = n / per_token;
  if (i >= a.num_tokens) return;
  const int c = (int)(n - i * per_token);
  const int v = c / (per_token / 2), h = c % (per_token / 2) / CPR, col = c % CPR * 8;
  int slot, src;
  if (!entry(a, i, slot, src)) return;
  const uint16_t* from = static_cast<const uint16_t*>(v ? a.v_new : a.k_new);
  uint16_t* to = static_cast<uint16_t*>(v ? a.v_pages : a.k_pages);
  const uint4 w = *reinterpret_cast<const uint4*>(from + ((size_t)src * a.num_kv_heads + h) * D + col);
  *reinterpret_cast<uint4*>(to + (((size_t)(slot / kPage) * a.num_kv_heads + h) * kPage + slot % kPage) * D + col) = w;
}

// One wave: the runs that begin in `chunk` entries of the list, K or V of one
// kv-head. D / 8 lanes hold a row, 8 values each.
template <int D>
__global__ __launch_bounds__(64) void write_fp8_kernel(const WriteArgs a) {
  constexpr int LPR = D / 8, RPL = 64 / LPR, LOADS = kPage / RPL;  // lanes per row, rows per load, loads per run
  const int lane = threadIdx.x, Hkv = a.num_kv_heads;
  const int hv = blockIdx.x % (2 * Hkv), h = hv >> 1, v = hv & 1;
  const long long first = (long long)(blockIdx.x / (2 * Hkv)) * a.chunk;
  // Lane l holds entry first - 1 + l: the one before the chunk, the chunk, and
  // the 15 that a run from its last entry can reach.
  const long long mine = first - 1 + lane;
  int slot = -1, src = 0;
  const bool ok = mine >= 0 && mine < a.num_tokens && entry(a, mine, slot, src);
  const int before = __shfl_up(ok ? slot : -2, 1);
  const unsigned long long goes_on = __ballot(ok && lane > 0 && slot % kPage != 0 && before == slot - 1);
  const unsigned long long window = (2ull << a.chunk) - 2;  // the chunk's own entries
  unsigned long long heads = __ballot(ok) & ~goes_on & window;
  const uint16_t* from = static_cast<const uint16_t*>(v ? a.v_new : a.k_new);
  uint8_t* to = static_cast<uint8_t*>(v ? a.v_pages : a.k_pages);
  float* scales = v ? a.v_scale : a.k_scale;
  while (heads != 0) {
    const int at = __builtin_ctzll(heads);
    heads &= heads - 1;
    const int n = 1 + __builtin_ctzll(~(goes_on >> 1 >> at));
    const int slot0 = __builtin_amdgcn_readlane(slot, at);
    const int r0 = slot0 % kPage;
    const size_t block = (size_t)(slot0 / kPage) * Hkv + h;
    const float old = scales[block];
    uint4 w[LOADS];
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const int i = j * RPL + lane / LPR;
      const int row = __shfl(src, min(at + i, 63));
      w[j] = make_uint4(0, 0, 0, 0);
      if (i < n) w[j] = *reinterpret_cast<const uint4*>(from + ((size_t)row * Hkv + h) * D + lane % LPR * 8);
    }
    float amax = 0.f;
    bool plain = true;  // no NaN element
    float x[LOADS][8];
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const uint32_t u[4] = {w[j].x, w[j].y, w[j].z, w[j].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[j][2 * e] = bf16_lo(u[e]);
        x[j][2 * e + 1] = bf16_hi(u[e]);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        amax = fmaxf(amax, fabsf(x[j][e]));
        plain = plain && x[j][e] == x[j][e];
      }
    }
    amax = wave_max(amax);
    RequantJob job = {to + block * (kPage * D), old, old, 0};
    if (r0 == 0) {
      job.scale = amax > 0.f ? amax / 448.0f : 1.0f;
    } else if (!(amax <= 448.0f * old)) {
      job.scale = amax / 448.0f;
      job.rows = r0;
    }
    const float inv = 1.0f / job.scale;
    const bool scaled = plain && plain_scale(job.scale);
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const int i = j * RPL + lane / LPR;
      uint32_t codes[2];
      if (i < n) {
        e4m3_quotients(x[j], job.scale, inv, scaled, codes);
        *reinterpret_cast<uint2*>(job.blk + (size_t)(r0 + i) * D + lane % LPR * 8) = make_uint2(codes[0], codes[1]);
      }
    }
    if (lane == 0 && (r0 == 0 || job.rows > 0)) scales[block] = job.scale;
    requantise_fp8_rows<D>(job, lane == 0, lane);
  }
}

// ---- page tables --------------------------------------------------------------

constexpr int kTableThreads = 1024;

// Exclusive prefix sums over the sequences, the same in every workgroup.
struct Sums {
  int back[kTableMaxSeqs + 1];   // pages given back
  int take[kTableMaxSeqs + 1];   // pages taken
  int fresh[kTableMaxSeqs + 1];  // new tokens
  long long part[3][kTableThreads / 64];
  int bad, count;
};

__device__ inline void page_counts(int old_len, int new_len, int& back, int& take, int& fresh) {
  const int have = (old_len + kPage - 1) / kPage, want = (new_len + kPage - 1) / kPage;
  back = max(have - want, 0);
  take = max(want - have, 0);
  fresh = max(new_len - old_len, 0);
}

// Fills the sums and returns the call's status.
__device__ int sum_up(const TableArgs& a, Sums& m, long long (&total)[3]) {
  constexpr int PER = kTableMaxSeqs / kTableThreads;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (tid == 0) {
    m.bad = 0;
    m.count = *a.free_count;
  }
  __syncthreads();
  const int per = cdiv(a.num_seqs, kTableThreads);  // sequences per thread, consecutive ones
  const int cap = a.max_pages * kPage;
  int v[PER][3];
  long long x[3] = {0, 0, 0};
  bool bad = false;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int s = tid * per + i;
    v[i][0] = v[i][1] = v[i][2] = 0;
    if (i < per && s < a.num_seqs) {
      const int o = a.old_lens[s], n = a.new_lens[s];
      const bool fits = o >= 0 && o <= cap && n >= 0 && n <= cap;
      bad = bad || !fits;
      if (fits) page_counts(o, n, v[i][0], v[i][1], v[i][2]);
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) x[k] += v[i][k];
  }
  long long run[3];
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    long long y = x[k];
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const long long z = __shfl_up(y, o);
      y += lane >= o ? z : 0;
    }
    if (lane == 63) m.part[k][wave] = y;
    run[k] = y - x[k];
  }
  if (bad) m.bad = 1;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    total[k] = 0;
    for (int w = 0; w < kTableThreads / 64; ++w) {
      run[k] += w < wave ? m.part[k][w] : 0;
      total[k] += m.part[k][w];
    }
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int s = tid * per + i;
    if (i < per && s < a.num_seqs) {
      m.back[s] = (int)run[0];
      m.take[s] = (int)run[1];
      m.fresh[s] = (int)run[2];
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) run[k] += v[i][k];
  }
  if (tid == 0) {
    m.back[a.num_seqs] = (int)total[0];
    m.take[a.num_seqs] = (int)total[1];
    m.fresh[a.num_seqs] = (int)total[2];
  }
  __syncthreads();
  const long long count = m.count;
  if (m.bad) return RP_TABLES_BAD_LENGTH;
  if (count < 0 || count + total[0] > a.num_pages) return RP_TABLES_BAD_FREE_LIST;
  if (total[1] > count + total[0]) return RP_TABLES_NO_PAGES;
  if (total[2] >= (1ll << 31) || (a.slot_map != nullptr && total[2] > a.max_slots)) return RP_TABLES_NO_SLOTS;
  return RP_TABLES_OK;
}

// The sequence s with sums[s] <= rank < sums[s + 1].
__device__ inline int owner(const int* sums, int n, int rank) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (sums[mid] <= rank) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

__device__ inline int first_page(int len) { return (len + kPage - 1) / kPage; }

// Pages of rank `item`, `item` + `step` ...: given back, then taken. The page
// given back with rank f goes to place top - 1 - f of the stack, and the page
// taken with rank o comes from place top - 1 - o: for o below the number given
// back that is the page of rank o among those, which whoever gives it back
// hands over, so nothing that this call writes is read by it.
__device__ void move_pages(const TableArgs& a, const Sums& m, int item, int step) {
  const int S = a.num_seqs, F = m.back[S], N = m.take[S];
  const long long top = (long long)m.count + F;
  for (int f = item; f < F; f += step) {
    const int s = owner(m.back, S, f);
    int* at = a.block_table + (size_t)s * a.max_pages + first_page(a.new_lens[s]) + (f - m.back[s]);
    const int page = *at;
    *at = -1;
    a.free_pages[top - 1 - f] = page;
    if (f < N) {
      const int t = owner(m.take, S, f);
      a.block_table[(size_t)t * a.max_pages + first_page(a.old_lens[t]) + (f - m.take[t])] = page;
    }
  }
  for (int o = F + item; o < N; o += step) {
    const int s = owner(m.take, S, o);
    a.block_table[(size_t)s * a.max_pages + first_page(a.old_lens[s]) + (o - m.take[s])] = a.free_pages[top - 1 - o];
  }
}

__device__ void write_slots(const TableArgs& a, const int* fresh, int status, long long item, long long step) {
  const int total = status == RP_TABLES_OK ? fresh[a.num_seqs] : 0;
  for (long long t = item; t < a.max_slots; t += step) {
    int slot = -1;
    if (t < total) {
      const int s = owner(fresh, a.num_seqs, (int)t);
      const int pos = a.old_lens[s] + ((int)t - fresh[s]);
      slot = a.block_table[(size_t)s * a.max_pages + pos / kPage] * kPage + pos % kPage;
    }
    a.slot_map[t] = slot;
  }
}

__device__ void tell(const TableArgs& a, const Sums& m, int status, const long long (&total)[3]) {
  const int tid = threadIdx.x;
  if (a.slot_offs != nullptr)
    for (int s = tid; s <= a.num_seqs; s += kTableThreads) a.slot_offs[s] = status == RP_TABLES_OK ? m.fresh[s] : 0;
  if (tid == 0) {
    a.status[0] = status;
    a.status[1] = (int)total[1];
    a.status[2] = (int)total[0];
    a.status[3] = (int)min(total[2], (1ll << 31) - 1);
  }
}

// Everything in one workgroup.
__global__ __launch_bounds__(kTableThreads) void tables_one_kernel(const TableArgs a) {
  __shared__ Sums m;
  long long total[3];
  const int status = sum_up(a, m, total);
  tell(a, m, status, total);
  if (status == RP_TABLES_OK) {
    move_pages(a, m, threadIdx.x, kTableThreads);
    if (threadIdx.x == 0) *a.free_count = (int)(m.count + total[0] - total[1]);
  }
  __syncthreads();  // the tables are written
  if (a.slot_map != nullptr) write_slots(a, m.fresh, status, threadIdx.x, kTableThreads);
}

// The same in two launches of many workgroups: pages, then slots and the count
// of free pages, which every workgroup of the first one reads.
__global__ __launch_bounds__(kTableThreads) void tables_pages_kernel(const TableArgs a) {
  __shared__ Sums m;
  long long total[3];
  const int status = sum_up(a, m, total);
  if (blockIdx.x == 0) tell(a, m, status, total);
  if (status == RP_TABLES_OK)
    move_pages(a, m, blockIdx.x * kTableThreads + threadIdx.x, gridDim.x * kTableThreads);
}
__global__ __launch_bounds__(kTableThreads) void tables_slots_kernel(const TableArgs a) {
  __shared__ int fresh[kTableMaxSeqs + 1];
  const int status = a.status[0];
  if (blockIdx.x == 0 && threadIdx.x == 0 && status == RP_TABLES_OK) *a.free_count += a.status[2] - a.status[1];
  if (a.slot_map == nullptr) return;
  for (int s = threadIdx.x; s <= a.num_seqs; s += kTableThreads) fresh[s] = a.slot_offs[s];
  __syncthreads();
  write_slots(a, fresh, status, (long long)blockIdx.x * kTableThreads + threadIdx.x,
              (long long)gridDim.x * kTableThreads);
}

}  // namespace

hipError_t launch_write_slots(const WriteArgs& a, int head_dim, bool fp8, hipStream_t stream) {
  if (a.num_tokens <= 0) return hipSuccess;
  if (head_dim != 128 && head_dim != 64) return hipErrorInvalidValue;
  if (fp8) {
    const long long blocks = ((long long)a.num_tokens + a.chunk - 1) / a.chunk * 2 * a.num_kv_heads;
    if (a.chunk < 1 || a.chunk > 48 || blocks >= (1ll << 31)) return hipErrorInvalidValue;
    if (head_dim == 128) write_fp8_kernel<128><<<(unsigned)blocks, 64, 0, stream>>>(a);
    else write_fp8_kernel<64><<<(unsigned)blocks, 64, 0, stream>>>(a);
  } else {
    const long long pieces = (long long)a.num_tokens * 2 * a.num_kv_heads * (head_dim / 8);
    const long long blocks = (pieces + kWriteThreads - 1) / kWriteThreads;
    if (blocks >= (1ll << 31)) return hipErrorInvalidValue;
    if (head_dim == 128) write_bf16_kernel<128><<<(unsigned)blocks, kWriteThreads, 0, stream>>>(a);
    else write_bf16_kernel<64><<<(unsigned)blocks, kWriteThreads, 0, stream>>>(a);
  }
  return hipGetLastError();
}

hipError_t launch_page_tables(const TableArgs& a, int blocks, hipStream_t stream) {
  if (a.num_seqs > kTableMaxSeqs || blocks < 1) return hipErrorInvalidValue;
  if (blocks == 1) {
    tables_one_kernel<<<1, kTableThreads, 0, stream>>>(a);
    return hipGetLastError();
  }
  tables_pages_kernel<<<blocks, kTableThreads, 0, stream>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  tables_slots_kernel<<<blocks, kTableThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace rp
