// Writes into the paged cache by slot, and the tables that the slots come from.
//
// rp_kv_write_slots: row i of a list goes to slot page * 16 + row. bf16 pools
// copy. fp8 pools keep one scale per (page, kv-head) for K and for V, so the
// entries of a page are handled together: a run is a maximal stretch of the
// list, skipped entries left out, whose slots rise inside one page, and one wave
// takes a run of one kv-head's K or V: amax over the run's rows, one scale, one
// rounding.
//
// rp_page_tables_resize: two exclusive prefix sums over the sequences (pages
// given back, pages taken) say where each page of a block table goes on, or
// comes from, the stack of free pages.
#include <algorithm>

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

// A copy, 16 bytes per thread, K and V of an entry side by side: bound by
// memory, 64 prompts of 64 to 1024 tokens (Hkv 8, d 128) 285 MB in 55 us, 5.2
// TB/s read and written, what a large copy reaches; 4 tokens 1.7 us.
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

// Entries of the list without the skipped ones between them, for a wave that
// has some in sight: lane l holds the one before the wave's own entries (l = 0)
// or the l-th from those on, slot -1 behind the last; returns how many of the
// wave's own there are. In: entry first - 1 + lane, `live` and `own` as lane
// masks. The entry before is looked for among 64, those behind the wave's own
// among at least 64 for each: whatever a run of entries less than 64 places apart
// needs. Two more loads, side by side (256 sequences of 8 drafts, half of them
// accepted, Hkv 8, d 128: in place 11.0 us, gathered to half the entries 10.0).
__device__ inline int close_up(const WriteArgs& a, long long first, unsigned long long live, unsigned long long own,
                               int2 (&line)[64], int& slot, int& src) {
  const int lane = threadIdx.x;
  const long long back = first - 64 + lane, ahead = first + 63 + lane;
  int2 x = make_int2(-1, 0), y = x;
  const bool before = back >= 0 && entry(a, back, x.x, x.y);
  const bool behind = ahead < a.num_tokens && entry(a, ahead, y.x, y.y);
  const unsigned long long b = __ballot(before), c = __ballot(behind), lower = (1ull << lane) - 1, mine = live & ~1ull;
  line[lane] = make_int2(-1, 0);
  __syncthreads();
  if (mine >> lane & 1) line[1 + __popcll(mine & lower)] = make_int2(slot, src);
  const int at = 1 + __popcll(mine) + __popcll(c & lower);
  if (behind && at < 64) line[at] = y;
  if (before && (b & ~lower) >> 1 >> lane == 0) line[0] = x;
  __syncthreads();
  slot = line[lane].x;
  src = line[lane].y;
  return __popcll(live & own);
}

// One wave: the runs that begin in `chunk` entries of the list, K or V of one
// kv-head. D / 8 lanes hold a row, 8 values each. Whole pages are bound by
// memory: 32 prompts of 2048 to 4096 tokens (Hkv 8, d 128) 604 MB in 119 us,
// 5.1 TB/s; short runs by the chain slot, scale, row, requantised rows: 256 runs
// of 1 to 8 tokens 9 us a call.
template <int D>
__global__ __launch_bounds__(64) void write_fp8_kernel(const WriteArgs a) {
  constexpr int LPR = D / 8, RPL = 64 / LPR, LOADS = kPage / RPL;  // lanes per row, rows per load, loads per run
  const int lane = threadIdx.x, Hkv = a.num_kv_heads;
  const int hv = blockIdx.x % (2 * Hkv), h = hv >> 1, v = hv & 1;
  const long long first = (long long)(blockIdx.x / (2 * Hkv)) * a.chunk;
  __shared__ int2 line[64];
  // Lane l holds entry first - 1 + l: the one before the chunk, the chunk, and
  // the 15 that a run from its last entry can reach.
  const long long mine = first - 1 + lane;
  int slot = -1, src = 0;
  const bool listed = mine >= 0 && mine < a.num_tokens;
  if (listed && !entry(a, mine, slot, src)) slot = -1;
  const unsigned long long live = __ballot(slot >= 0);
  unsigned long long own = (2ull << a.chunk) - 2;  // the chunk's entries
  if ((live & own) == 0) return;
  if (live != __ballot(listed)) own = (2ull << close_up(a, first, live, own, line, slot, src)) - 2;
  const int before = __shfl_up(slot, 1);
  const unsigned long long goes_on =
      __ballot(lane > 0 && before >= 0 && before / kPage == slot / kPage && before < slot);
  unsigned long long heads = __ballot(slot >= 0) & ~goes_on & own;
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
    int to_row[LOADS];
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const int i = j * RPL + lane / LPR;
      const int row = __shfl(src, min(at + i, 63));
      to_row[j] = __shfl(slot, min(at + i, 63)) % kPage;
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
        *reinterpret_cast<uint2*>(job.blk + (size_t)to_row[j] * D + lane % LPR * 8) = make_uint2(codes[0], codes[1]);
      }
    }
    if (lane == 0 && (r0 == 0 || job.rows > 0)) scales[block] = job.scale;
    requantise_fp8_rows<D>(job, lane == 0, lane);
  }
}

// ---- page tables --------------------------------------------------------------

// Exclusive prefix sums over the sequences, the same in every workgroup.
struct Sums {
  int back[kTableMaxSeqs + 1];   // pages given back
  int take[kTableMaxSeqs + 1];   // pages taken
  int fresh[kTableMaxSeqs + 1];  // new tokens
  int old_len[kTableMaxSeqs], new_len[kTableMaxSeqs];
  long long part[3][16];
  int bad, count;
};

__device__ inline int pages_of(int len) { return (len + kPage - 1) / kPage; }

// Inclusive sum over the lanes of a wave.
__device__ inline int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, true);  // lane - 1, - 2, - 4, - 8 of a row of 16
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, true);  // the row before's last lane, into rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, true);  // lane 31, into rows 2 and 3
  return x;
}
__device__ inline long long wave_scan(long long x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const long long y = __shfl_up(x, o);
    x += lane >= o ? y : 0;
  }
  return x;
}

// Fills the sums and returns the call's status. Sum: the type that holds any
// sum of new tokens that the table could.
template <class Sum>
__device__ int sum_up(const TableArgs& a, Sums& m, long long (&total)[3]) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, waves = blockDim.x >> 6;
  if (tid == 0) {
    m.bad = 0;
    m.count = *a.free_count;
  }
  const int per = cdiv(a.num_seqs, (int)blockDim.x), s0 = tid * per;  // consecutive sequences of a thread
  const int cap = a.max_pages * kPage;
  Sum x[3] = {0, 0, 0};
  bool bad = false;
  for (int i = 0; i < per && s0 + i < a.num_seqs; ++i) {
    const int s = s0 + i, o = a.old_lens[s], n = a.new_lens[s];
    const bool fits = o >= 0 && o <= cap && n >= 0 && n <= cap;
    bad = bad || !fits;
    m.old_len[s] = fits ? o : 0;
    m.new_len[s] = fits ? n : 0;
    if (!fits) continue;
    const int d = pages_of(n) - pages_of(o);
    x[0] += max(-d, 0);
    x[1] += max(d, 0);
    x[2] += max(n - o, 0);
  }
  Sum run[3];
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    const Sum y = wave_scan(x[k]);
    if (lane == 63) m.part[k][wave] = y;
    run[k] = y - x[k];
  }
  __syncthreads();
  if (bad) m.bad = 1;
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    total[k] = 0;
    for (int w = 0; w < waves; ++w) {
      run[k] += w < wave ? (Sum)m.part[k][w] : 0;
      total[k] += m.part[k][w];
    }
  }
  for (int i = 0; i < per && s0 + i < a.num_seqs; ++i) {
    const int s = s0 + i, o = m.old_len[s], n = m.new_len[s], d = pages_of(n) - pages_of(o);
    m.back[s] = (int)run[0];
    m.take[s] = (int)run[1];
    m.fresh[s] = (int)run[2];
    run[0] += max(-d, 0);
    run[1] += max(d, 0);
    run[2] += max(n - o, 0);
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

// Table entry of the page given back, or taken, with rank r.
__device__ inline int* back_entry(const TableArgs& a, const Sums& m, int r) {
  const int s = owner(m.back, a.num_seqs, r);
  return a.block_table + (size_t)s * a.max_pages + pages_of(m.new_len[s]) + (r - m.back[s]);
}
__device__ inline int* take_entry(const TableArgs& a, const Sums& m, int r) {
  const int s = owner(m.take, a.num_seqs, r);
  return a.block_table + (size_t)s * a.max_pages + pages_of(m.old_len[s]) + (r - m.take[s]);
}

// Pages of rank `item`, `item` + `step` ...: given back, then taken. The page
// given back with rank f goes to place top - 1 - f of the stack, and the page
// taken with rank o comes from place top - 1 - o: for o below the number given
// back that is the page of rank o among those, which whoever gives it back
// hands over, so nothing that this call writes is read by it. between(): after
// the first of them have been read, before anything is written.
template <class F>
__device__ void move_pages(const TableArgs& a, const Sums& m, int item, int step, F between) {
  const int F_ = m.back[a.num_seqs], N = m.take[a.num_seqs];
  const long long top = (long long)m.count + F_;
  const int f0 = item, o0 = F_ + item;
  int *from = nullptr, *to = nullptr, given = 0, taken = 0;
  if (f0 < F_) {
    from = back_entry(a, m, f0);
    given = *from;
  }
  if (o0 < N) {
    to = take_entry(a, m, o0);
    taken = a.free_pages[top - 1 - o0];
  }
  between();
  for (int f = f0; f < F_; f += step) {
    if (f != f0) {
      from = back_entry(a, m, f);
      given = *from;
    }
    *from = -1;
    a.free_pages[top - 1 - f] = given;
    if (f < N) *take_entry(a, m, f) = given;
  }
  for (int o = o0; o < N; o += step) {
    if (o != o0) {
      to = take_entry(a, m, o);
      taken = a.free_pages[top - 1 - o];
    }
    *to = taken;
  }
}

// Slots t0, t0 + step ... of the new tokens; page(s, p): page p of sequence s.
template <class F>
__device__ void write_slots(const TableArgs& a, const int* fresh, const int* old_len, int total, long long t0,
                            long long step, F page) {
  for (long long t = t0; t < a.max_slots; t += step) {
    int slot = -1;
    if (t < total) {
      const int s = owner(fresh, a.num_seqs, (int)t);
      const int pos = old_len[s] + ((int)t - fresh[s]);
      slot = page(s, pos / kPage) * kPage + pos % kPage;
    }
    a.slot_map[t] = slot;
  }
}

__device__ void tell(const TableArgs& a, const Sums& m, int status, const long long (&total)[3]) {
  if (a.slot_offs != nullptr)
    for (int s = threadIdx.x; s <= a.num_seqs; s += blockDim.x) a.slot_offs[s] = status == RP_TABLES_OK ? m.fresh[s] : 0;
  if (threadIdx.x == 0) {
    a.status[0] = status;
    a.status[1] = (int)total[1];
    a.status[2] = (int)total[0];
    a.status[3] = (int)min(total[2], (1ll << 31) - 1);
  }
}

// Everything in one workgroup, which is latency: lengths, sums, table entries,
// slots, 3.8 us for 16 sequences and 136 new tokens. The slots come from what the
// tables hold before, with new pages by their rank, in the shadow of the first
// moves' loads.
__global__ __launch_bounds__(1024) void tables_one_kernel(const TableArgs a) {
  __shared__ Sums m;
  long long total[3];
  const int status = sum_up<int>(a, m, total);  // of at most 8192 pages
  const bool done = status == RP_TABLES_OK;
  const auto slots = [&]() {
    if (a.slot_map != nullptr) {
      const long long top = m.count + total[0];
      write_slots(a, m.fresh, m.old_len, done ? (int)total[2] : 0, threadIdx.x, blockDim.x, [&](int s, int p) {
        const int rank = m.take[s] + p - pages_of(m.old_len[s]);
        if (p < pages_of(m.old_len[s])) return a.block_table[(size_t)s * a.max_pages + p];
        return rank < total[0] ? *back_entry(a, m, rank) : a.free_pages[top - 1 - rank];
      });
    }
    __syncthreads();  // every read of what was there is done
  };
  if (done) {
    move_pages(a, m, threadIdx.x, blockDim.x, slots);
    if (threadIdx.x == 0) *a.free_count = (int)(m.count + total[0] - total[1]);
  } else {
    slots();
  }
  tell(a, m, status, total);
}

// The same in two launches of many workgroups: pages, then slots and the count
// of free pages, which every workgroup of the first one reads. Each sums up all
// lengths by itself: 6 to 7 us and 7.5 us for 1024 sequences.
template <class Sum>
__global__ __launch_bounds__(1024) void tables_pages_kernel(const TableArgs a) {
  __shared__ Sums m;
  long long total[3];
  const int status = sum_up<Sum>(a, m, total);
  if (blockIdx.x == 0) tell(a, m, status, total);
  if (status == RP_TABLES_OK)
    move_pages(a, m, blockIdx.x * blockDim.x + threadIdx.x, gridDim.x * blockDim.x, [] {});
}
__global__ __launch_bounds__(1024) void tables_slots_kernel(const TableArgs a) {
  __shared__ int fresh[kTableMaxSeqs + 1], old_len[kTableMaxSeqs];
  const int status = a.status[0];
  if (blockIdx.x == 0 && threadIdx.x == 0 && status == RP_TABLES_OK) *a.free_count += a.status[2] - a.status[1];
  if (a.slot_map == nullptr) return;
  for (int s = threadIdx.x; s <= a.num_seqs; s += blockDim.x) {
    fresh[s] = a.slot_offs[s];
    if (s < a.num_seqs) old_len[s] = a.old_lens[s];
  }
  __syncthreads();
  write_slots(a, fresh, old_len, status == RP_TABLES_OK ? fresh[a.num_seqs] : 0,
              (long long)blockIdx.x * blockDim.x + threadIdx.x, (long long)gridDim.x * blockDim.x,
              [&](int s, int p) { return a.block_table[(size_t)s * a.max_pages + p]; });
}

}  // namespace

hipError_t launch_write_slots(const WriteArgs& a, int head_dim, bool fp8, hipStream_t stream) {
  if (a.num_tokens <= 0) return hipSuccess;
  if (head_dim != 128 && head_dim != 64) return hipErrorInvalidValue;
  if (fp8) {
    const long long blocks = ((long long)a.num_tokens + a.chunk - 1) / a.chunk * 2 * a.num_kv_heads;
    if (a.chunk < 1 || a.chunk > 48 || blocks > 4 * kMaxBlocks256) return hipErrorInvalidValue;
    if (head_dim == 128) write_fp8_kernel<128><<<(unsigned)blocks, 64, 0, stream>>>(a);
    else write_fp8_kernel<64><<<(unsigned)blocks, 64, 0, stream>>>(a);
  } else {
    const long long pieces = (long long)a.num_tokens * 2 * a.num_kv_heads * (head_dim / 8);
    const long long blocks = (pieces + kWriteThreads - 1) / kWriteThreads;
    if (blocks > kMaxBlocks256) return hipErrorInvalidValue;
    if (head_dim == 128) write_bf16_kernel<128><<<(unsigned)blocks, kWriteThreads, 0, stream>>>(a);
    else write_bf16_kernel<64><<<(unsigned)blocks, kWriteThreads, 0, stream>>>(a);
  }
  return hipGetLastError();
}

hipError_t launch_page_tables(const TableArgs& a, hipStream_t stream) {
  if (a.num_seqs > kTableMaxSeqs) return hipErrorInvalidValue;
  // One workgroup where little can move, by the table and the slots: it takes
  // about 1 us for 1000 pages or slots, and the second launch about 5 us (16
  // sequences x 377 pages, 136 new tokens: one launch 3.8 us, two 8.9; 1024 x
  // 129, a quarter of them ending: one launch 150 us, two 14.4).
  const long long entries = (long long)a.num_seqs * a.max_pages, work = std::max<long long>(a.max_slots, entries);
  const int blocks = work <= 8192 ? 1 : (int)std::min(std::max(2ll, work / 1024), 256ll);
  const int threads = blocks > 1 || a.max_slots > 1024 || a.num_seqs > 256 ? 1024 : 256;
  if (blocks == 1) tables_one_kernel<<<1, threads, 0, stream>>>(a);
  else if (entries * kPage < (1ll << 31)) tables_pages_kernel<int><<<blocks, threads, 0, stream>>>(a);
  else tables_pages_kernel<long long><<<blocks, threads, 0, stream>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || blocks == 1) return e;
  tables_slots_kernel<<<blocks, threads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace rp
