// C-ABI entry points: argument validation, workspace layout and kernel
// launches on the caller's stream. No device allocation and no host sync on
// the hot path; rp_validate_layout is the one test utility that does both.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <mutex>

#include "rp.h"
#include "rp_internal.h"

namespace {

thread_local char g_err[512];

rp_status fail(rp_status st, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_err, sizeof(g_err), fmt, ap);
  va_end(ap);
  return st;
}

rp_status hip_fail(hipError_t e, const char* what) {
  return fail(RP_ERR_HIP, "%s: %s (%d)", what, hipGetErrorString(e), (int)e);
}

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

struct Shape {
  int S, G, Hq, Hkv, D, nrep, max_pp, max_rp, num_pages;
  bool fp8;
};

rp_status check_kv(const rp_paged_kv* kv) {
  if (kv == nullptr) return fail(RP_ERR_INVALID_ARG, "kv is NULL");
  if (kv->k_pages == nullptr || kv->v_pages == nullptr) return fail(RP_ERR_INVALID_ARG, "k_pages/v_pages is NULL");
  if (!aligned(kv->k_pages, 16) || !aligned(kv->v_pages, 16))
    return fail(RP_ERR_INVALID_ARG, "k_pages/v_pages must be 16-byte aligned");
  if (kv->num_pages < 1) return fail(RP_ERR_INVALID_ARG, "num_pages must be >= 1 (got %d)", kv->num_pages);
  if (kv->num_kv_heads < 1) return fail(RP_ERR_INVALID_ARG, "num_kv_heads must be >= 1");
  if (kv->page_size != rp::kPage) return fail(RP_ERR_UNSUPPORTED, "page_size %d unsupported (16 only)", kv->page_size);
  if (kv->head_dim != 64 && kv->head_dim != 128)
    return fail(RP_ERR_UNSUPPORTED, "head_dim %d unsupported (64 or 128)", kv->head_dim);
  const int dtype = rp::enum_bits(kv->kv_dtype);
  if (dtype == RP_KV_BF16) {
    if (kv->k_scale != nullptr || kv->v_scale != nullptr)
      return fail(RP_ERR_INVALID_ARG, "k_scale/v_scale must be NULL for bf16 KV");
  } else if (dtype == RP_KV_FP8_E4M3) {
    if (kv->k_scale == nullptr || kv->v_scale == nullptr)
      return fail(RP_ERR_INVALID_ARG, "k_scale/v_scale required for fp8 KV");
    if (!aligned(kv->k_scale, 4) || !aligned(kv->v_scale, 4))
      return fail(RP_ERR_INVALID_ARG, "k_scale/v_scale must be 4-byte aligned");
  } else {
    return fail(RP_ERR_UNSUPPORTED, "kv_dtype %d unsupported", dtype);
  }
  return RP_OK;
}

rp_status check_shape(const rp_paged_kv* kv, const rp_group_layout* l, Shape* sh) {
  rp_status st = check_kv(kv);
  if (st != RP_OK) return st;
  if (l == nullptr) return fail(RP_ERR_INVALID_ARG, "layout is NULL");
  if (l->num_seqs < 0) return fail(RP_ERR_INVALID_ARG, "num_seqs must be >= 0");
  if (l->num_q_heads < 1) return fail(RP_ERR_INVALID_ARG, "num_q_heads must be >= 1");
  if (l->num_q_heads % kv->num_kv_heads != 0)
    return fail(RP_ERR_INVALID_ARG, "num_q_heads %d not a multiple of num_kv_heads %d", l->num_q_heads,
                kv->num_kv_heads);
  const int nrep = l->num_q_heads / kv->num_kv_heads;
  if (nrep != 1 && nrep != 2 && nrep != 4 && nrep != 8)
    return fail(RP_ERR_UNSUPPORTED, "q/kv head ratio %d unsupported (1, 2, 4, 8)", nrep);
  if (l->max_prefix_pages < 0 || l->max_resp_pages < 0)
    return fail(RP_ERR_INVALID_ARG, "table widths must be >= 0");
  if (l->num_seqs > 0) {
    if (l->num_groups < 1) return fail(RP_ERR_INVALID_ARG, "num_groups must be >= 1");
    if (l->seq_to_group == nullptr || l->prefix_lens == nullptr || l->resp_lens == nullptr)
      return fail(RP_ERR_INVALID_ARG, "seq_to_group/prefix_lens/resp_lens is NULL");
    if (l->max_prefix_pages > 0 && l->prefix_block_table == nullptr)
      return fail(RP_ERR_INVALID_ARG, "prefix_block_table is NULL");
    if (l->max_resp_pages > 0 && l->resp_block_table == nullptr)
      return fail(RP_ERR_INVALID_ARG, "resp_block_table is NULL");
  }
  // Every index the kernels form stays below 2^31 elements per int32 table.
  const long long rows = (long long)l->num_seqs * l->num_q_heads;
  if (l->num_seqs > 0 && l->num_groups > rp::kPlanMaxGroups)
    return fail(RP_ERR_UNSUPPORTED, "num_groups %d above the planner's limit %d", l->num_groups, rp::kPlanMaxGroups);
  if ((long long)l->num_seqs * l->max_resp_pages >= (1ll << 31) ||
      (long long)l->num_groups * l->max_prefix_pages >= (1ll << 31) || rows >= (1ll << 31))
    return fail(RP_ERR_UNSUPPORTED, "layout too large for int32 indexing");
  sh->S = l->num_seqs;
  sh->G = l->num_groups;
  sh->Hq = l->num_q_heads;
  sh->Hkv = kv->num_kv_heads;
  sh->D = kv->head_dim;
  sh->nrep = nrep;
  sh->max_pp = l->max_prefix_pages;
  sh->max_rp = l->max_resp_pages;
  sh->num_pages = kv->num_pages;
  sh->fp8 = rp::enum_bits(kv->kv_dtype) == RP_KV_FP8_E4M3;
  return RP_OK;
}

// Workspace layout, 256-byte aligned sections.
struct WsLayout {
  size_t hdr, grp_off, members, pitems, ritems, seq_parts, part_o, part_lse, total;
  long long max_pitems, max_ritems, max_parts;
  int max_pc, max_rc;
};

size_t align_up(size_t x) { return (x + 255) & ~size_t(255); }

bool ws_layout(const Shape& sh, WsLayout* w) {
  w->max_pc = rp::cdiv(sh.max_pp, rp::kPrefixChunkPages);
  const bool small = (long long)sh.S * sh.max_rp * sh.Hkv <= rp::kSmallBatchPageHeads;
  w->max_rc = rp::cdiv(sh.max_rp, small ? rp::kRespChunkPagesSmall : rp::kRespChunkPagesMin);
  const long long groups_used = sh.G < sh.S ? sh.G : sh.S;
  w->max_pitems = groups_used * w->max_pc;
  w->max_ritems = (long long)sh.S * w->max_rc;
  w->max_parts = (long long)sh.S * sh.Hq * (w->max_pc + w->max_rc);
  if (w->max_parts >= (1ll << 31) || w->max_ritems * sh.Hkv >= (1ll << 31) ||
      w->max_pitems * sh.Hkv >= (1ll << 31))
    return false;
  size_t o = 0;
  w->hdr = o;       o = align_up(o + sizeof(int) * rp::kHdrSlots);
  w->grp_off = o;   o = align_up(o + sizeof(int) * ((size_t)sh.G + 1));
  w->members = o;   o = align_up(o + sizeof(int) * (size_t)sh.S);
  w->pitems = o;    o = align_up(o + sizeof(int2) * (size_t)w->max_pitems);
  w->ritems = o;    o = align_up(o + sizeof(int4) * (size_t)w->max_ritems);
  w->seq_parts = o; o = align_up(o + sizeof(int) * (size_t)sh.S);
  w->part_o = o;    o = align_up(o + sizeof(float) * (size_t)w->max_parts * sh.D);
  w->part_lse = o;  o = align_up(o + sizeof(float) * (size_t)w->max_parts);
  w->total = o;
  return true;
}

// Compute units of the current device, queried once per device (racing first
// calls store the same value; relaxed atomics keep that race defined).
rp_status device_cus(int* cus) {
  static std::atomic<int> cache[64];
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return hip_fail(e, "hipGetDevice");
  if (dev < 0 || dev >= 64) return fail(RP_ERR_UNSUPPORTED, "device %d out of range", dev);
  int n = cache[dev].load(std::memory_order_relaxed);
  if (n == 0) {
    e = hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev);
    if (e != hipSuccess) return hip_fail(e, "hipDeviceGetAttribute");
    cache[dev].store(n, std::memory_order_relaxed);
  }
  *cus = n;
  return RP_OK;
}

// Scratch of rp_group_decode_attn_noalloc: the work plan and partial results
// live in this device array instead of a caller workspace. Each GPU holds its
// own copy for the life of the process; its name is only a host-side handle,
// so host code uses the device address looked up once per device below.
__device__ __align__(256) static unsigned char scratch[RP_NOALLOC_SCRATCH_BYTES];

rp_status scratch_address(void** out) {
  static std::atomic<void*> addr[64];
  static std::mutex lookup;
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return hip_fail(e, "hipGetDevice");
  if (dev < 0 || dev >= 64) return fail(RP_ERR_UNSUPPORTED, "device %d out of range", dev);
  void* p = addr[dev].load(std::memory_order_acquire);
  if (p == nullptr) {
    std::lock_guard<std::mutex> lock(lookup);
    p = addr[dev].load(std::memory_order_relaxed);
    if (p == nullptr) {
      e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));  // with device `dev` current
      if (e != hipSuccess) return hip_fail(e, "hipGetSymbolAddress(scratch)");
      if (p == nullptr || !aligned(p, 256)) return fail(RP_ERR_HIP, "scratch has no usable device address");
      addr[dev].store(p, std::memory_order_release);
    }
  }
  *out = p;
  return RP_OK;
}

rp::PlanView plan_view(void* ws, const WsLayout& w) {
  char* b = static_cast<char*>(ws);
  rp::PlanView v;
  v.hdr = reinterpret_cast<int*>(b + w.hdr);
  v.grp_off = reinterpret_cast<int*>(b + w.grp_off);
  v.grp_members = reinterpret_cast<int*>(b + w.members);
  v.prefix_items = reinterpret_cast<int2*>(b + w.pitems);
  v.resp_items = reinterpret_cast<int4*>(b + w.ritems);
  v.seq_parts = reinterpret_cast<int*>(b + w.seq_parts);
  v.part_o = reinterpret_cast<float*>(b + w.part_o);
  v.part_lse = reinterpret_cast<float*>(b + w.part_lse);
  v.max_prefix_chunks = w.max_pc;
  v.max_resp_chunks = w.max_rc;
  v.parts_per_row = w.max_pc + w.max_rc;
  v.max_parts = (int)w.max_parts;
  v.max_prefix_items = (int)w.max_pitems;
  v.max_resp_items = (int)w.max_ritems;
  return v;
}

// Whether rp_group_decode_attn runs as one launch, a workgroup per (sequence,
// kv-head), instead of plan, parts and combine. Its seven shares of a
// sequence's pages (as many as the tables hold) take steps of 8 KiB of K and V
// one after the other; the three launches have more waves to share the pages
// but a longer chain of round trips, take one pass over a group's prefix for
// every 16 of its query rows, and slow down sooner as the batch's K and V grow.
// The line lies where the two are equal. Measured, three launches against one,
// in us at 4, 8, 10 and 16 steps (Hq / Hkv and d of the layer, sequences x
// kv-heads; 20-50% of the pages prefix):
//   2, 128 bf16, 1 x 1:  13.3 8.8, 14.6 12.9, 14.2 14.3, 15.2 20.9
//                16 x 8: 18.8 10.1, 19.8 14.8, 20.6 17.6, 25.0 24.8
//   2, 64 bf16,  1 x 1:  10.9 8.3, 11.6 11.9, 11.8 13.7, 12.3 19.6
//   2, 128 fp8,  1 x 1:  14.4 10.3, 14.8 15.0, 14.8 17.2, 16.0 23.7
//   2, 64 fp8,   1 x 1:  12.6 11.2, 13.2 17.9, 13.6 20.9, 14.2 30.4
//                16 x 8: 16.0 12.9, 20.3 19.7, 22.0 23.4, 28.7 33.5
//   4, 64 fp8,   16 x 2 (2 groups): 18.9 12.1, 19.5 18.9, 20.3 22.2, 21.6 32.3
//   8, 128 bf16, 16 x 2 (2 groups): 37.5 9.7, 41.1 14.2, 42.4 16.6, 42.9 23.6
// The batch's tables may span at most 128 MiB of K and V, since each member
// reads its group's prefix for itself, and the plan that the one launch leaves
// in the workspace is made by one wave (at most 64 sequences).
bool small_batch(const Shape& sh) {
  const long long page_bytes = 2ll * rp::kPage * sh.D * (sh.fp8 ? 1 : 2);  // K and V of a (page, kv-head)
  const long long pages = (long long)sh.max_pp + sh.max_rp, per_step = (rp::kSmallWaves - 1) * (8192 / page_bytes);
  const long long steps = (pages + per_step - 1) / per_step, kv_bytes = pages * sh.S * sh.Hkv * page_bytes;
  if (sh.S > rp::kSmallPlanMaxSeqs || steps > (sh.nrep >= 4 ? 20 : 10) || kv_bytes > (128ll << 20)) return false;
  const bool wide = sh.D == 128;
  // Passes over a group's prefix; several groups are seldom of one size, and
  // from four query rows a member on, one member more is often a pass more (4
  // sequences, 3 of them of one group, Hq 16, Hkv 2: three launches 24.0 us,
  // one 18.0).
  const int members = rp::cdiv(sh.S, sh.G) + (sh.G > 1 && sh.nrep >= 4 ? 1 : 0);
  const int passes = rp::cdiv(sh.nrep * members, 16);
  const double one_us = (double)steps * (!sh.fp8 ? 1.0 : wide ? 1.15 : 1.55);
  const double three_us = (!wide ? 8.0 : sh.fp8 ? 9.0 : 10.0) + 0.05 * (double)kv_bytes / (1 << 20) +
                          (passes - 1) * std::min(sh.max_pp, rp::kPrefixChunkPages) * (wide ? 0.45 : 0.25);
  return one_us <= three_us;  // both beyond what the shortest call takes
}

rp_status prepare(const rp_paged_kv* kv, const rp_group_layout* l, void* ws, size_t ws_bytes, Shape* sh,
                  WsLayout* w) {
  rp_status st = check_shape(kv, l, sh);
  if (st != RP_OK) return st;
  if (!ws_layout(*sh, w)) return fail(RP_ERR_UNSUPPORTED, "layout too large for the work plan");
  if (sh->S == 0) return RP_OK;
  if (ws == nullptr) return fail(RP_ERR_WORKSPACE, "workspace is NULL");
  if (!aligned(ws, 256)) return fail(RP_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  if (ws_bytes < w->total)
    return fail(RP_ERR_WORKSPACE, "workspace has %zu bytes, needs %zu", ws_bytes, w->total);
  return RP_OK;
}

rp::AttnArgs attn_args(const rp_paged_kv* kv, const rp_group_layout* l, const void* q, float scale,
                       const rp::PlanView& v) {
  rp::AttnArgs a;
  a.k_pages = kv->k_pages;
  a.v_pages = kv->v_pages;
  a.k_scale = kv->k_scale;
  a.v_scale = kv->v_scale;
  a.num_pages = kv->num_pages;
  a.num_kv_heads = kv->num_kv_heads;
  a.num_seqs = l->num_seqs;
  a.num_groups = l->num_groups;
  a.num_q_heads = l->num_q_heads;
  a.seq_to_group = l->seq_to_group;
  a.prefix_lens = l->prefix_lens;
  a.prefix_block_table = l->prefix_block_table;
  a.max_prefix_pages = l->max_prefix_pages;
  a.resp_lens = l->resp_lens;
  a.resp_block_table = l->resp_block_table;
  a.max_resp_pages = l->max_resp_pages;
  a.q = q;
  a.qk_scale = scale * rp::kLog2e;
  a.view = v;
  return a;
}

// The planner's arguments for a prepared batch (queries the device's compute
// units, which set the piece length).
rp_status plan_args(const Shape& sh, const rp_group_layout* l, void* ws, const WsLayout& w, int len_add,
                    rp::PlanArgs* a) {
  int cus = 0;
  rp_status st = device_cus(&cus);
  if (st != RP_OK) return st;
  a->num_seqs = sh.S;
  a->num_groups = sh.G;
  a->num_q_heads = sh.Hq;
  a->num_kv_heads = sh.Hkv;
  a->num_cus = cus;
  a->seq_to_group = l->seq_to_group;
  a->prefix_lens = l->prefix_lens;
  a->resp_lens = l->resp_lens;
  a->len_add = len_add;
  a->max_prefix_pages = sh.max_pp;
  a->max_resp_pages = sh.max_rp;
  a->view = plan_view(ws, w);
  return RP_OK;
}

// Checks and launch arguments of the decode step's q/k prep.
rp_status qk_prep_args(const rp_paged_kv* kv, const rp_group_layout* l, const Shape& sh, const void* q_in,
                       const void* k_in, const void* v_in, const void* q_norm_w, const void* k_norm_w,
                       double rms_eps, double rope_theta, void* q_out, void* k_out, rp::QkPrepArgs* a) {
  if (!(rms_eps >= 0.0) || !std::isfinite(rms_eps)) return fail(RP_ERR_INVALID_ARG, "rms_eps must be finite and >= 0");
  if (!(rope_theta > 0.0) || !std::isfinite(rope_theta))
    return fail(RP_ERR_INVALID_ARG, "rope_theta must be finite and > 0");
  if (sh.S == 0) return RP_OK;
  const void* in[] = {q_in, k_in, v_in, q_norm_w, k_norm_w, q_out};
  for (const void* p : in)
    if (p == nullptr || !aligned(p, 16))
      return fail(RP_ERR_INVALID_ARG, "q_in/k_in/v_in/q_norm_w/k_norm_w/q_out must be non-NULL and 16-byte aligned");
  if (k_out != nullptr && !aligned(k_out, 16)) return fail(RP_ERR_INVALID_ARG, "k_out must be 16-byte aligned");
  if (sh.max_rp < 1) return fail(RP_ERR_INVALID_ARG, "max_resp_pages must be >= 1 to append");
  a->k_pages = kv->k_pages;
  a->v_pages = kv->v_pages;
  a->k_scale = kv->k_scale;
  a->v_scale = kv->v_scale;
  a->num_pages = kv->num_pages;
  a->num_kv_heads = sh.Hkv;
  a->num_q_heads = sh.Hq;
  a->num_seqs = sh.S;
  a->num_groups = sh.G;
  a->seq_to_group = l->seq_to_group;
  a->prefix_lens = l->prefix_lens;
  a->resp_lens = l->resp_lens;
  a->resp_block_table = l->resp_block_table;
  a->max_resp_pages = sh.max_rp;
  a->q_in = static_cast<const uint16_t*>(q_in);
  a->k_in = static_cast<const uint16_t*>(k_in);
  a->v_in = static_cast<const uint16_t*>(v_in);
  a->q_norm_w = static_cast<const uint16_t*>(q_norm_w);
  a->k_norm_w = static_cast<const uint16_t*>(k_norm_w);
  a->rms_eps = rms_eps;
  // Rotary frequencies on the host in fp64 (libm pow), passed with the arguments.
  for (int i = 0; i < rp::kMaxHeadDim / 2; ++i)
    a->inv_freq[i] = i < sh.D / 2 ? std::pow(rope_theta, (-2.0 * i) / sh.D) : 0.0;
  a->q_out = static_cast<uint16_t*>(q_out);
  a->k_out = static_cast<uint16_t*>(k_out);
  a->blocks_per_seq = 0;
  return RP_OK;
}

// How a tree attention is divided. What depends on the lengths is decided on
// the device: the host has the tables' widths, which are often many times the
// lengths, and bounds from them.
//
// kTreeUnits units are two workgroups per compute unit of an MI355X, which read
// as fast as more of them and leave the shorter end. us a call with 256, 512,
// 1024 and 2048 of them (Hq 16, Hkv 8, d 128; sequences x drafts over tokens):
//   16 x 1-16 over 512 + U[0, 6016]:  45.3  45.1  53.0  53.1
//   16 x 32 over 512 + U[0, 6016]:    63.3  57.6  79.7  79.7
//   8 x 8 over 512 + U[0, 16000]:     52.9  54.9  56.9  64.1
//   16 x 8, fp8, the first's tokens:  38.3  31.1  39.3  39.5
//   64 x 8 over U[0, 7600]:           205   174   210   203
// A piece of fewer than 32 pages costs more in partial results than it gives,
// of more too few units for small calls (4 x 8 over 512 + U[0, 6016], 16, 32
// and 64 pages: 24.3 21.2 26.3).
//
// Forms, by the query rows of a (sequence, kv-head): one, two or four tiles of
// 16 with the keys split between waves up to 64 rows, keys shared by waves
// beyond. us with 1, 2, 4 tiles and shared keys (64 sequences, 8 kv-heads, d
// 64, 8192 tokens; bf16, then fp8):
//   16 rows   180 183 184 201   105 107 109 181
//   32 rows   264 190 188 205   149 113 115 183
//   64 rows   446 282 204 228   254 177 148 219
//   96 rows   634 388 308 254   363 253 259 234
//   128 rows  765 475 325 270   481 326 274 252
// and with d 128 (bf16 10240, fp8 20480 tokens) at 16 rows 440-456 against
// 430-460 with two tiles, at 32 441-473 against 610-640 with one, at 64 480 (fp8
// 592-615) against 506-520 (740) with shared keys, at 96 520 (815) with shared
// keys against 680 (1060) with four tiles.
//
// Prefixes are either units of their own, read once for all members, or part of
// every member's pages, read again from the caches: at about 14 TB/s, against
// the partial results that units of their own write and read (those of the
// prefix, and those of the pieces where these would be final), at about 1.8
// TB/s, and the second launch where nothing else needs it. us apart and read by
// each (8 kv-heads, d 128):
//   64 sequences, 512 tokens, 1, 8 and 16 drafts: 101 107, 108 106, 133 111
//   256 sequences, 512 tokens, 2 drafts, 1024 tokens, 8 drafts: 205 232, 251 297
//   64 sequences, 2048 tokens, 4 and 16 drafts: 40 66, 76 73
constexpr int kTreeLongPages = 480;
struct TreePlan {
  rp::TreeForm form;
  bool share;
  int longest_first, row_blocks, max_pc, repeats, seq_pieces, max_extra, slot_rows, least_pages;
  float piece_share;
  long long prefix_blocks, blocks, pieces_at;
  size_t parts, part_o, part_lse, total;  // total 0: every result is final
};

rp_status check_tree(const Shape& sh, const rp_draft_tree* t) {
  if (t == nullptr) return fail(RP_ERR_INVALID_ARG, "tree is NULL");
  if (t->num_drafts < 0) return fail(RP_ERR_INVALID_ARG, "num_drafts must be >= 0");
  if (t->max_drafts < 1) return fail(RP_ERR_INVALID_ARG, "max_drafts must be >= 1");
  if (t->max_drafts > rp::kTreeMaxDrafts)
    return fail(RP_ERR_UNSUPPORTED, "max_drafts %d above the limit %d", t->max_drafts, rp::kTreeMaxDrafts);
  if (sh.S == 0 || t->num_drafts == 0) return RP_OK;
  if (t->draft_offs == nullptr || !aligned(t->draft_offs, 4))
    return fail(RP_ERR_INVALID_ARG, "draft_offs must be a non-NULL int32 array");
  if (t->masks == nullptr || !aligned(t->masks, 8))
    return fail(RP_ERR_INVALID_ARG, "masks must be a non-NULL uint64 array");
  return RP_OK;
}

bool tree_plan(const Shape& sh, const rp_draft_tree* t, TreePlan* p) {
  using rp::TreeForm;
  const long long T = t->num_drafts, pairs = (long long)sh.S * sh.Hkv;
  const int rows = t->max_drafts * sh.nrep;
  p->form = rows <= 16   ? TreeForm::kSplit1
            : rows <= 32 ? TreeForm::kSplit2
            : rows <= 64 ? TreeForm::kSplit4
                         : TreeForm::kRows;
  const int cols = rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : 128, prefix_cols = rows <= 64 ? 64 : 128;
  p->row_blocks = rp::cdiv(rows, cols);
  // Pieces of each of `count` where they are the whole launch.
  const auto pieces_of = [](long long count) {
    return (int)(rp::kTreeUnits / std::min(std::max(count, 1ll), (long long)rp::kTreeUnits));
  };
  const long long base = pairs * p->row_blocks;
  const long long per_group = (T * sh.nrep + (long long)sh.G * prefix_cols - 1) / ((long long)sh.G * prefix_cols);
  p->repeats = (int)std::min(std::max(per_group, 1ll), 64ll);
  p->max_pc = std::min(rp::cdiv(sh.max_pp, rp::kTreeLeastPages), pieces_of((long long)sh.G * sh.Hkv * p->repeats));
  p->seq_pieces = pieces_of(base);
  // Up to half a round of units for the sequences' short pieces, and the whole
  // launch is one round; behind that, four fifths of a round and no pieces
  // below 480 pages (7680 tokens), which cost more in partial results (64 x 8
  // over U[0, 7600]: 173, from 240 pages on cut 184). us with
  // shares of 1, 1.25 and 2 places' pages (Hq 16, Hkv 8, d 128):
  //   16 x 1-16 over 512 + U[0, 6016]:  58 47 47 (1.14)
  //   32 x 8 over 512 + U[0, 6016]:     95 87 88 (1.33)
  //   32 x 8 over U[0, 30000]:          394 430 353 (1.33)
  //   64 x 1-32, fp8, over 256 + U[8192, 32768]:  563 549 590
  //   64 x 16, fp8, over U[0, 32768]:   430 390 426
  const double places = base <= rp::kTreeUnits / 2 ? rp::kTreeUnits - base / 2.0 : rp::kTreeUnits / 1.25;
  p->piece_share = (float)((double)sh.Hkv * p->row_blocks / places);
  p->least_pages = p->seq_pieces > 1 ? rp::kTreeLeastPages : kTreeLongPages;
  // The bound of find_piece's pieces besides the first ones.
  const auto extra = [&](int pages) -> int {
    if (sh.S > rp::kTreeOrderSeqs) return 0;
    const long long by_width = (long long)sh.S * (rp::cdiv(std::max(pages, 1), p->least_pages) - 1);
    const long long by_number = std::max((long long)sh.S * (p->seq_pieces - 1),
                                         rp::kTreeUnits / ((long long)sh.Hkv * p->row_blocks));
    return (int)std::min(by_width, by_number);
  };
  // Shared prefixes or not, in us.
  const int flat_pages = sh.max_pp + sh.max_rp;
  const double page_bytes = 2.0 * rp::kPage * sh.D * (sh.fp8 ? 1 : 2);
  const double again = (sh.S - std::min(sh.G, sh.S)) * (double)sh.max_pp * sh.Hkv * page_bytes / 14e6;
  const double parts = (double)T * sh.Hq * (p->max_pc + (p->seq_pieces == 1 ? 1 : 0)) * sh.D * 8 / 1.8e6 +
                       (extra(flat_pages) == 0 ? 6.0 : 0.0);
  p->share = again > parts;
  if (!p->share) p->max_pc = 0;
  const int pages = p->share ? sh.max_rp : flat_pages;
  p->max_extra = extra(pages);
  // The longest first; where one unit per sequence and kv-head fills the chip
  // once, two to a compute unit, the second one there has the shorter the
  // longer the first is (64 sequences of U[0, 7600] tokens, 8 kv-heads: as they
  // come 200 us, so 165; 32 of 1024 + U[0, 2048] with 64 drafts 135 and 119).
  p->longest_first = 0;
  if (sh.S <= rp::kTreeOrderSeqs && base > rp::kTreeUnits) p->longest_first = sh.S;
  if (sh.S <= rp::kTreeOrderSeqs && base <= rp::kTreeUnits && base > rp::kTreeUnits / 2 && pages >= 64)
    p->longest_first = (int)((sh.S * (rp::kTreeUnits / 2) + base - 1) / base);
  p->slot_rows = rows;
  p->pieces_at = p->share || p->max_extra > 0 ? T * sh.Hq * (p->max_pc + 1) : 0;
  const auto grid = [](long long units, long long repeats) { return (units + 7) / 8 * 8 * repeats; };
  p->prefix_blocks = p->share ? grid((long long)sh.G * p->max_pc * sh.Hkv, p->repeats) : 0;
  p->blocks = p->prefix_blocks + grid(((long long)sh.S + p->max_extra) * sh.Hkv, p->row_blocks);
  const long long partial = p->pieces_at + (long long)p->max_extra * sh.Hkv * rows;
  if (T * sh.Hq >= (1ll << 31) || partial >= (1ll << 31) || T * sh.Hq * (sh.D / 4) / 256 >= rp::kMaxBlocks256 ||
      p->blocks > rp::kMaxBlocks256)
    return false;
  size_t o = 0;
  p->parts = o;    o = align_up(o + (partial == 0 ? 0 : sizeof(int2) * (size_t)T));
  p->part_o = o;   o = align_up(o + sizeof(float) * (size_t)partial * sh.D);
  p->part_lse = o; o = align_up(o + sizeof(float) * (size_t)partial);
  p->total = o;
  return true;
}

}  // namespace

extern "C" {

const char* rp_status_string(rp_status status) {
  switch (rp::enum_bits(status)) {
    case RP_OK: return "RP_OK: success";
    case RP_ERR_INVALID_ARG: return "RP_ERR_INVALID_ARG: invalid argument";
    case RP_ERR_UNSUPPORTED: return "RP_ERR_UNSUPPORTED: unsupported configuration";
    case RP_ERR_WORKSPACE: return "RP_ERR_WORKSPACE: workspace missing or too small";
    case RP_ERR_HIP: return "RP_ERR_HIP: HIP runtime error";
    case RP_ERR_LAYOUT: return "RP_ERR_LAYOUT: layout entry out of range";
  }
  return "unknown rp_status";
}

const char* rp_last_error(void) { return g_err; }

rp_status rp_group_decode_attn_workspace_size(const rp_paged_kv* kv, const rp_group_layout* layout,
                                              size_t* bytes) {
  g_err[0] = 0;
  if (bytes == nullptr) return fail(RP_ERR_INVALID_ARG, "bytes is NULL");
  Shape sh;
  rp_status st = check_shape(kv, layout, &sh);
  if (st != RP_OK) return st;
  WsLayout w;
  if (!ws_layout(sh, &w)) return fail(RP_ERR_UNSUPPORTED, "layout too large for the work plan");
  *bytes = sh.S == 0 ? 0 : w.total;
  return RP_OK;
}

rp_status rp_plan(const rp_paged_kv* kv, const rp_group_layout* l, void* ws, size_t ws_bytes,
                  hipStream_t stream) {
  g_err[0] = 0;
  Shape sh;
  WsLayout w;
  rp_status st = prepare(kv, l, ws, ws_bytes, &sh, &w);
  if (st != RP_OK || sh.S == 0) return st;
  rp::PlanArgs a;
  st = plan_args(sh, l, ws, w, 0, &a);
  if (st != RP_OK) return st;
  hipError_t e = rp::launch_plan(a, stream);
  return e == hipSuccess ? RP_OK : hip_fail(e, "plan kernel launch");
}

rp_status rp_attn_parts(const rp_paged_kv* kv, const rp_group_layout* l, const void* q, float softmax_scale,
                        void* ws, size_t ws_bytes, hipStream_t stream) {
  g_err[0] = 0;
  Shape sh;
  WsLayout w;
  rp_status st = prepare(kv, l, ws, ws_bytes, &sh, &w);
  if (st != RP_OK || sh.S == 0) return st;
  if (q == nullptr || !aligned(q, 16)) return fail(RP_ERR_INVALID_ARG, "q must be non-NULL and 16-byte aligned");
  const rp::AttnArgs a = attn_args(kv, l, q, softmax_scale, plan_view(ws, w));
  hipError_t e = rp::launch_attn_parts(a, sh.D, sh.nrep, sh.fp8, w.max_pitems, w.max_ritems, stream);
  return e == hipSuccess ? RP_OK : hip_fail(e, "attention parts kernel launch");
}

rp_status rp_combine_parts(const rp_paged_kv* kv, const rp_group_layout* l, void* out, float* lse, void* ws,
                           size_t ws_bytes, hipStream_t stream) {
  g_err[0] = 0;
  Shape sh;
  WsLayout w;
  rp_status st = prepare(kv, l, ws, ws_bytes, &sh, &w);
  if (st != RP_OK || sh.S == 0) return st;
  if (out == nullptr || !aligned(out, 16)) return fail(RP_ERR_INVALID_ARG, "out must be non-NULL and 16-byte aligned");
  if (lse != nullptr && !aligned(lse, 4)) return fail(RP_ERR_INVALID_ARG, "lse must be 4-byte aligned");
  const rp::PlanView v = plan_view(ws, w);
  rp::CombineArgs c{};
  c.o_parts = v.part_o;
  c.lse_parts = v.part_lse;
  c.row_offs = nullptr;
  c.num_rows = sh.S * sh.Hq;
  c.out = out;
  c.lse = lse;
  c.seq_parts = v.seq_parts;
  c.num_q_heads = sh.Hq;
  c.parts_per_row = v.parts_per_row;
  hipError_t e = rp::launch_combine(c, sh.D, stream);
  return e == hipSuccess ? RP_OK : hip_fail(e, "combine kernel launch");
}

rp_status rp_group_decode_attn(const rp_paged_kv* kv, const rp_group_layout* l, const void* q,
                               float softmax_scale, void* out, float* lse, void* ws, size_t ws_bytes,
                               hipStream_t stream) {
  g_err[0] = 0;
  Shape sh;
  WsLayout w;
  rp_status st = prepare(kv, l, ws, ws_bytes, &sh, &w);
  if (st != RP_OK || sh.S == 0) return st;
  if (q == nullptr || !aligned(q, 16)) return fail(RP_ERR_INVALID_ARG, "q must be non-NULL and 16-byte aligned");
  if (out == nullptr || !aligned(out, 16)) return fail(RP_ERR_INVALID_ARG, "out must be non-NULL and 16-byte aligned");
  if (lse != nullptr && !aligned(lse, 4)) return fail(RP_ERR_INVALID_ARG, "lse must be 4-byte aligned");
  if (small_batch(sh)) {
    rp::PlanArgs p;
    st = plan_args(sh, l, ws, w, 0, &p);
    if (st != RP_OK) return st;
    const rp::AttnArgs a = attn_args(kv, l, q, softmax_scale, p.view);
    hipError_t e = rp::launch_attn_small(a, p, sh.D, sh.nrep, sh.fp8, out, lse, stream);
    return e == hipSuccess ? RP_OK : hip_fail(e, "small attention kernel launch");
  }
  st = rp_plan(kv, l, ws, ws_bytes, stream);
  if (st != RP_OK) return st;
  st = rp_attn_parts(kv, l, q, softmax_scale, ws, ws_bytes, stream);
  if (st != RP_OK) return st;
  return rp_combine_parts(kv, l, out, lse, ws, ws_bytes, stream);
}

rp_status rp_group_decode_attn_noalloc(const rp_paged_kv* kv, const rp_group_layout* l, const void* q,
                                       float softmax_scale, void* out, float* lse, hipStream_t stream) {
  g_err[0] = 0;
  Shape sh;
  rp_status st = check_shape(kv, l, &sh);
  if (st != RP_OK) return st;
  WsLayout w;
  if (!ws_layout(sh, &w)) return fail(RP_ERR_UNSUPPORTED, "layout too large for the work plan");
  if (sh.S == 0) return RP_OK;
  if (w.total > (size_t)RP_NOALLOC_SCRATCH_BYTES)
    return fail(RP_ERR_WORKSPACE,
                "this layout needs %zu bytes of scratch; the library's static scratch holds %zu "
                "(use rp_group_decode_attn with a workspace)",
                w.total, (size_t)RP_NOALLOC_SCRATCH_BYTES);
  void* ws = nullptr;
  st = scratch_address(&ws);
  if (st != RP_OK) return st;
  // The same launches as rp_group_decode_attn. The plan and the partial results
  // overwrite every entry that is read later, so nothing needs clearing.
  return rp_group_decode_attn(kv, l, q, softmax_scale, out, lse, ws, RP_NOALLOC_SCRATCH_BYTES, stream);
}

rp_status rp_lse_combine(const float* o_parts, const float* lse_parts, const int32_t* row_part_offsets,
                         int32_t num_rows, int32_t head_dim, void* out, float* lse_out, hipStream_t stream) {
  g_err[0] = 0;
  if (num_rows < 0) return fail(RP_ERR_INVALID_ARG, "num_rows must be >= 0");
  if (head_dim != 64 && head_dim != 128) return fail(RP_ERR_UNSUPPORTED, "head_dim %d unsupported", head_dim);
  if (num_rows == 0) return RP_OK;
  if (row_part_offsets == nullptr || out == nullptr)
    return fail(RP_ERR_INVALID_ARG, "row_part_offsets/out is NULL");
  if (!aligned(out, 8)) return fail(RP_ERR_INVALID_ARG, "out must be 8-byte aligned");
  if (lse_out != nullptr && !aligned(lse_out, 4)) return fail(RP_ERR_INVALID_ARG, "lse_out must be 4-byte aligned");
  if ((o_parts != nullptr && !aligned(o_parts, 16)) || (lse_parts != nullptr && !aligned(lse_parts, 4)))
    return fail(RP_ERR_INVALID_ARG, "o_parts must be 16-byte and lse_parts 4-byte aligned");
  rp::CombineArgs c{};
  c.o_parts = o_parts;
  c.lse_parts = lse_parts;
  c.row_offs = row_part_offsets;
  c.num_rows = num_rows;
  c.out = out;
  c.lse = lse_out;
  hipError_t e = rp::launch_combine(c, head_dim, stream);
  return e == hipSuccess ? RP_OK : hip_fail(e, "combine kernel launch");
}

rp_status rp_group_tree_attn_workspace_size(const rp_paged_kv* kv, const rp_group_layout* l, const rp_draft_tree* tree,
                                            size_t* bytes) {
  g_err[0] = 0;
  if (bytes == nullptr) return fail(RP_ERR_INVALID_ARG, "bytes is NULL");
  Shape sh;
  rp_status st = check_shape(kv, l, &sh);
  if (st == RP_OK) st = check_tree(sh, tree);
  if (st != RP_OK) return st;
  *bytes = 0;
  if (sh.S == 0 || tree->num_drafts == 0) return RP_OK;
  TreePlan p;
  if (!tree_plan(sh, tree, &p)) return fail(RP_ERR_UNSUPPORTED, "too many drafts for one call");
  *bytes = p.total;
  return RP_OK;
}

rp_status rp_group_tree_attn(const rp_paged_kv* kv, const rp_group_layout* l, const rp_draft_tree* tree, const void* q,
                             const void* k_draft, const void* v_draft, float softmax_scale, void* out, float* lse,
                             void* ws, size_t ws_bytes, hipStream_t stream) {
  g_err[0] = 0;
  Shape sh;
  rp_status st = check_shape(kv, l, &sh);
  if (st == RP_OK) st = check_tree(sh, tree);
  if (st != RP_OK) return st;
  if (!(softmax_scale > 0.f) || !std::isfinite(softmax_scale))
    return fail(RP_ERR_INVALID_ARG, "softmax_scale must be finite and > 0");
  if (sh.S == 0 || tree->num_drafts == 0) return RP_OK;
  TreePlan p;
  if (!tree_plan(sh, tree, &p)) return fail(RP_ERR_UNSUPPORTED, "too many drafts for one call");
  const void* in[] = {q, k_draft, v_draft, out};
  for (const void* x : in)
    if (x == nullptr || !aligned(x, 16))
      return fail(RP_ERR_INVALID_ARG, "q/k_draft/v_draft/out must be non-NULL and 16-byte aligned");
  if (lse != nullptr && !aligned(lse, 4)) return fail(RP_ERR_INVALID_ARG, "lse must be 4-byte aligned");
  if (p.total > 0) {
    if (ws == nullptr) return fail(RP_ERR_WORKSPACE, "workspace is NULL");
    if (!aligned(ws, 256)) return fail(RP_ERR_WORKSPACE, "workspace must be 256-byte aligned");
    if (ws_bytes < p.total) return fail(RP_ERR_WORKSPACE, "workspace has %zu bytes, needs %zu", ws_bytes, p.total);
  }
  rp::TreeArgs a{};
  a.k_pages = kv->k_pages;
  a.v_pages = kv->v_pages;
  a.k_scale = kv->k_scale;
  a.v_scale = kv->v_scale;
  a.num_pages = kv->num_pages;
  a.num_kv_heads = sh.Hkv;
  a.num_seqs = sh.S;
  a.num_groups = sh.G;
  a.num_q_heads = sh.Hq;
  a.rep_shift = sh.nrep == 1 ? 0 : sh.nrep == 2 ? 1 : sh.nrep == 4 ? 2 : 3;
  a.seq_to_group = l->seq_to_group;
  a.prefix_lens = l->prefix_lens;
  a.prefix_block_table = l->prefix_block_table;
  a.max_prefix_pages = sh.max_pp;
  a.resp_lens = l->resp_lens;
  a.resp_block_table = l->resp_block_table;
  a.max_resp_pages = sh.max_rp;
  a.num_drafts = tree->num_drafts;
  a.max_drafts = tree->max_drafts;
  a.draft_offs = tree->draft_offs;
  a.masks = reinterpret_cast<const unsigned long long*>(tree->masks);
  a.q = static_cast<const uint16_t*>(q);
  a.k_draft = static_cast<const uint16_t*>(k_draft);
  a.v_draft = static_cast<const uint16_t*>(v_draft);
  a.qk_scale = softmax_scale * rp::kLog2e;
  a.out = static_cast<uint16_t*>(out);
  a.lse = lse;
  char* b = static_cast<char*>(ws);
  if (p.total > 0) {
    a.token_parts = reinterpret_cast<int2*>(b + p.parts);
    a.part_o = reinterpret_cast<float*>(b + p.part_o);
    a.part_lse = reinterpret_cast<float*>(b + p.part_lse);
  }
  a.share = p.share ? 1 : 0;
  a.longest_first = p.longest_first;
  a.max_prefix_chunks = p.max_pc;
  a.prefix_repeats = p.repeats;
  a.prefix_blocks = (int)p.prefix_blocks;
  a.seq_pieces = p.seq_pieces;
  a.least_pages = p.least_pages;
  a.piece_share = p.piece_share;
  a.max_extra = p.max_extra;
  a.pieces_at = p.pieces_at;
  a.slot_rows = p.slot_rows;
  a.row_blocks = p.row_blocks;
  hipError_t e = rp::launch_tree_attn(a, sh.D, sh.fp8, p.form, p.blocks, stream);
  if (e != hipSuccess) return hip_fail(e, "tree attention kernel launch");
  if (p.total == 0) return RP_OK;
  e = rp::launch_tree_merge(a, sh.D, stream);
  return e == hipSuccess ? RP_OK : hip_fail(e, "tree merge kernel launch");
}

rp_status rp_kv_write_slots(const rp_paged_kv* kv, const int32_t* slot_map, int32_t num_tokens, const void* k_new,
                            const void* v_new, const int32_t* src_rows, int32_t num_src, hipStream_t stream) {
  g_err[0] = 0;
  rp_status st = check_kv(kv);
  if (st != RP_OK) return st;
  if (num_tokens < 0 || num_src < 0) return fail(RP_ERR_INVALID_ARG, "num_tokens/num_src must be >= 0");
  if (kv->num_pages >= (1 << 27)) return fail(RP_ERR_UNSUPPORTED, "slots of %d pages pass 32 bits", kv->num_pages);
  // A launch has fewer than 2^32 threads: 2 D / 8 for each row of bf16.
  if ((long long)num_tokens * kv->num_kv_heads * (kv->head_dim / 4) >= (1ll << 32) - 256)
    return fail(RP_ERR_UNSUPPORTED, "too many rows for one call");
  if (num_tokens == 0 || num_src == 0) return RP_OK;
  if (slot_map == nullptr || !aligned(slot_map, 4) || !aligned(src_rows, 4))
    return fail(RP_ERR_INVALID_ARG, "slot_map (non-NULL) and src_rows must be int32 arrays");
  if (k_new == nullptr || v_new == nullptr || !aligned(k_new, 16) || !aligned(v_new, 16))
    return fail(RP_ERR_INVALID_ARG, "k_new/v_new must be non-NULL and 16-byte aligned");
  rp::WriteArgs a;
  a.k_pages = kv->k_pages;
  a.v_pages = kv->v_pages;
  a.k_scale = kv->k_scale;
  a.v_scale = kv->v_scale;
  a.num_slots = kv->num_pages * rp::kPage;
  a.num_kv_heads = kv->num_kv_heads;
  a.num_tokens = num_tokens;
  a.num_src = num_src;
  a.slot_map = slot_map;
  a.src_rows = src_rows;
  a.k_new = k_new;
  a.v_new = v_new;
  // fp8: few entries per wave while there are few, so that no wave does many
  // runs one after the other, and 16 where the waves that begin no run would
  // count. us at 1, 4, 8, 16 entries (Hkv 8, d 128): 16 rows alone 8.2, 8.8, 13,
  // 21; 1024 alone 11.8, 13.3, 16, 24; 1024 runs of 8 36.8, 27.8, 20.4, 22.2; 64
  // prompts of 1024 234, 116, 98, 85.
  const long long waves = 2ll * num_tokens * kv->num_kv_heads;
  a.chunk = (int)std::min(std::max((waves + 12287) / 12288, 1ll), 16ll);
  hipError_t e = rp::launch_write_slots(a, kv->head_dim, rp::enum_bits(kv->kv_dtype) == RP_KV_FP8_E4M3, stream);
  return e == hipSuccess ? RP_OK : hip_fail(e, "slot write kernel launch");
}

rp_status rp_page_tables_resize(const rp_page_tables* t, const int32_t* old_lens, const int32_t* new_lens,
                                int32_t* status, int32_t* slot_offs, int32_t* slot_map, int32_t max_slots,
                                hipStream_t stream) {
  g_err[0] = 0;
  if (t == nullptr) return fail(RP_ERR_INVALID_ARG, "tables is NULL");
  if (t->num_seqs < 0 || t->max_pages < 0 || t->num_pages < 1 || max_slots < 0)
    return fail(RP_ERR_INVALID_ARG, "num_seqs/max_pages/max_slots must be >= 0 and num_pages >= 1");
  if (t->page_size != rp::kPage) return fail(RP_ERR_UNSUPPORTED, "page_size %d unsupported (16 only)", t->page_size);
  if (t->num_seqs > rp::kTableMaxSeqs)
    return fail(RP_ERR_UNSUPPORTED, "num_seqs %d above the limit %d", t->num_seqs, rp::kTableMaxSeqs);
  if (t->num_pages >= (1 << 27) || t->max_pages >= (1 << 27) || (long long)t->num_seqs * t->max_pages >= (1ll << 31))
    return fail(RP_ERR_UNSUPPORTED, "tables too large for int32 slots");
  if (status == nullptr || !aligned(status, 4)) return fail(RP_ERR_INVALID_ARG, "status must be a non-NULL int32 array");
  if (t->free_count == nullptr || t->free_pages == nullptr || !aligned(t->free_count, 4) || !aligned(t->free_pages, 4))
    return fail(RP_ERR_INVALID_ARG, "free_pages/free_count must be non-NULL int32 arrays");
  if (slot_map != nullptr && slot_offs == nullptr) return fail(RP_ERR_INVALID_ARG, "slot_map needs slot_offs");
  if (!aligned(slot_map, 4) || !aligned(slot_offs, 4))
    return fail(RP_ERR_INVALID_ARG, "slot_map/slot_offs must be int32 arrays");
  if (t->num_seqs > 0) {
    if (old_lens == nullptr || new_lens == nullptr || !aligned(old_lens, 4) || !aligned(new_lens, 4))
      return fail(RP_ERR_INVALID_ARG, "old_lens/new_lens must be non-NULL int32 arrays");
    if (t->max_pages > 0 && (t->block_table == nullptr || !aligned(t->block_table, 4)))
      return fail(RP_ERR_INVALID_ARG, "block_table must be a non-NULL int32 array");
  }
  rp::TableArgs a;
  a.num_seqs = t->num_seqs;
  a.max_pages = t->max_pages;
  a.num_pages = t->num_pages;
  a.max_slots = slot_map != nullptr ? max_slots : 0;
  a.block_table = t->block_table;
  a.free_pages = t->free_pages;
  a.free_count = t->free_count;
  a.old_lens = old_lens;
  a.new_lens = new_lens;
  a.slot_offs = slot_offs;
  a.slot_map = slot_map;
  a.status = status;
  hipError_t e = rp::launch_page_tables(a, stream);
  return e == hipSuccess ? RP_OK : hip_fail(e, "page table kernel launch");
}

rp_status rp_kv_append(const rp_paged_kv* kv, const rp_group_layout* l, const void* k_new, const void* v_new,
                       hipStream_t stream) {
  g_err[0] = 0;
  Shape sh;
  rp_status st = check_shape(kv, l, &sh);
  if (st != RP_OK) return st;
  if (sh.S == 0) return RP_OK;
  if (k_new == nullptr || v_new == nullptr || !aligned(k_new, 16) || !aligned(v_new, 16))
    return fail(RP_ERR_INVALID_ARG, "k_new/v_new must be non-NULL and 16-byte aligned");
  if (sh.max_rp < 1) return fail(RP_ERR_INVALID_ARG, "max_resp_pages must be >= 1 to append");
  rp::AppendArgs a;
  a.k_pages = kv->k_pages;
  a.v_pages = kv->v_pages;
  a.k_scale = kv->k_scale;
  a.v_scale = kv->v_scale;
  a.num_pages = kv->num_pages;
  a.num_kv_heads = kv->num_kv_heads;
  a.num_seqs = sh.S;
  a.resp_lens = l->resp_lens;
  a.resp_block_table = l->resp_block_table;
  a.max_resp_pages = sh.max_rp;
  a.k_new = k_new;
  a.v_new = v_new;
  hipError_t e = rp::launch_append(a, sh.D, sh.fp8, stream);
  return e == hipSuccess ? RP_OK : hip_fail(e, "append kernel launch");
}

rp_status rp_decode_qk_prep(const rp_paged_kv* kv, const rp_group_layout* l, const void* q_in, const void* k_in,
                            const void* v_in, const void* q_norm_w, const void* k_norm_w, double rms_eps,
                            double rope_theta, void* q_out, void* k_out, hipStream_t stream) {
  g_err[0] = 0;
  Shape sh;
  rp_status st = check_shape(kv, l, &sh);
  if (st != RP_OK) return st;
  rp::QkPrepArgs a;
  st = qk_prep_args(kv, l, sh, q_in, k_in, v_in, q_norm_w, k_norm_w, rms_eps, rope_theta, q_out, k_out, &a);
  if (st != RP_OK || sh.S == 0) return st;
  hipError_t e = rp::launch_qk_prep(a, sh.D, sh.fp8, stream);
  return e == hipSuccess ? RP_OK : hip_fail(e, "decode q/k prep kernel launch");
}

rp_status rp_decode_qk_prep_plan(const rp_paged_kv* kv, const rp_group_layout* l, const void* q_in,
                                 const void* k_in, const void* v_in, const void* q_norm_w, const void* k_norm_w,
                                 double rms_eps, double rope_theta, void* q_out, void* k_out, void* ws,
                                 size_t ws_bytes, hipStream_t stream) {
  g_err[0] = 0;
  Shape sh;
  WsLayout w;
  rp_status st = prepare(kv, l, ws, ws_bytes, &sh, &w);
  if (st != RP_OK) return st;
  rp::QkPrepArgs a;
  st = qk_prep_args(kv, l, sh, q_in, k_in, v_in, q_norm_w, k_norm_w, rms_eps, rope_theta, q_out, k_out, &a);
  if (st != RP_OK || sh.S == 0) return st;
  rp::PlanArgs p;
  st = plan_args(sh, l, ws, w, 1, &p);
  if (st != RP_OK) return st;
  hipError_t e;
  if (sh.S <= rp::kSmallPlanMaxSeqs && sh.G <= rp::kPlanMaxGroups) {
    e = rp::launch_qk_prep_plan(a, p, sh.D, sh.fp8, stream);
    return e == hipSuccess ? RP_OK : hip_fail(e, "decode q/k prep + plan kernel launch");
  }
  e = rp::launch_qk_prep(a, sh.D, sh.fp8, stream);
  if (e != hipSuccess) return hip_fail(e, "decode q/k prep kernel launch");
  e = rp::launch_plan(p, stream);
  return e == hipSuccess ? RP_OK : hip_fail(e, "plan kernel launch");
}

rp_status rp_grpo_advantage(const float* rewards, int32_t num_groups, int32_t group_size, double eps_std,
                            int32_t ddof, float* advantages, float* group_mean, float* group_std,
                            hipStream_t stream) {
  g_err[0] = 0;
  if (num_groups < 0 || group_size < 1)
    return fail(RP_ERR_INVALID_ARG, "num_groups must be >= 0 and group_size >= 1");
  if (ddof != 0 && ddof != 1) return fail(RP_ERR_INVALID_ARG, "ddof must be 0 or 1");
  if (!(eps_std >= 0.0) || !std::isfinite(eps_std)) return fail(RP_ERR_INVALID_ARG, "eps_std must be finite and >= 0");
  if ((long long)num_groups * group_size >= (1ll << 40)) return fail(RP_ERR_UNSUPPORTED, "too many rewards");
  if (num_groups == 0) return RP_OK;
  if (rewards == nullptr || advantages == nullptr || !aligned(rewards, 4) || !aligned(advantages, 4))
    return fail(RP_ERR_INVALID_ARG, "rewards/advantages must be non-NULL fp32 arrays");
  if ((group_mean != nullptr && !aligned(group_mean, 4)) || (group_std != nullptr && !aligned(group_std, 4)))
    return fail(RP_ERR_INVALID_ARG, "group_mean/group_std must be fp32 arrays");
  rp::GrpoArgs a;
  a.rewards = rewards;
  a.num_groups = num_groups;
  a.group_size = group_size;
  a.ddof = ddof;
  a.eps_std = eps_std;
  a.advantages = advantages;
  a.mean = group_mean;
  a.stdev = group_std;
  a.vector_ok = aligned(rewards, 16) && aligned(advantages, 16);
  hipError_t e = rp::launch_grpo(a, stream);
  return e == hipSuccess ? RP_OK : hip_fail(e, "GRPO advantage kernel launch");
}

// Shared checks of the prefill calls; fills a (pointers of the projections
// and outputs are checked by the callers).
static rp_status prefill_args(const rp_paged_kv* kv, const rp_prefill_layout* l, rp::PrefillArgs* a, int* n_rep) {
  rp_status st = check_kv(kv);
  if (st != RP_OK) return st;
  if (l == nullptr) return fail(RP_ERR_INVALID_ARG, "layout is NULL");
  if (l->num_groups < 0 || l->num_tokens < 0) return fail(RP_ERR_INVALID_ARG, "num_groups/num_tokens must be >= 0");
  if (l->num_q_heads < 1 || l->num_q_heads % kv->num_kv_heads != 0)
    return fail(RP_ERR_INVALID_ARG, "num_q_heads %d not a positive multiple of num_kv_heads %d", l->num_q_heads,
                kv->num_kv_heads);
  const int r = l->num_q_heads / kv->num_kv_heads;
  if (r != 1 && r != 2 && r != 4 && r != 8)
    return fail(RP_ERR_UNSUPPORTED, "q/kv head ratio %d unsupported (1, 2, 4, 8)", r);
  if (l->num_groups > 0) {
    if (l->prompt_offs == nullptr) return fail(RP_ERR_INVALID_ARG, "prompt_offs is NULL");
    if (l->max_prefix_pages < 1 || l->prefix_block_table == nullptr)
      return fail(RP_ERR_INVALID_ARG, "prefix_block_table must be non-NULL with max_prefix_pages >= 1");
  }
  // One prompt's K/V rows are addressed with 32-bit byte offsets.
  if ((long long)l->num_groups * l->max_prefix_pages * kv->num_kv_heads >= (1ll << 31) ||
      (long long)l->num_tokens * l->num_q_heads * kv->head_dim >= (1ll << 40) ||
      (long long)l->max_prefix_pages * rp::kPage * kv->num_kv_heads * kv->head_dim * 2 >= (1ll << 32))
    return fail(RP_ERR_UNSUPPORTED, "prefill too large");
  a->k_pages = kv->k_pages;
  a->v_pages = kv->v_pages;
  a->k_scale = kv->k_scale;
  a->v_scale = kv->v_scale;
  a->num_pages = kv->num_pages;
  a->num_kv_heads = kv->num_kv_heads;
  a->num_groups = l->num_groups;
  a->num_q_heads = l->num_q_heads;
  a->num_tokens = l->num_tokens;
  a->prompt_offs = l->prompt_offs;
  a->prefix_block_table = l->prefix_block_table;
  a->max_prefix_pages = l->max_prefix_pages;
  *n_rep = r;
  return RP_OK;
}

rp_status rp_prefill_kv_write(const rp_paged_kv* kv, const rp_prefill_layout* l, const void* k, const void* v,
                              hipStream_t stream) {
  g_err[0] = 0;
  rp::PrefillArgs a{};
  int n_rep = 0;
  rp_status st = prefill_args(kv, l, &a, &n_rep);
  if (st != RP_OK) return st;
  if (l->num_groups == 0 || l->num_tokens == 0) return RP_OK;
  if (k == nullptr || v == nullptr || !aligned(k, 16) || !aligned(v, 16))
    return fail(RP_ERR_INVALID_ARG, "k/v must be non-NULL and 16-byte aligned");
  a.k = k;
  a.v = v;
  hipError_t e = rp::launch_prefill_kv_write(a, kv->head_dim, rp::enum_bits(kv->kv_dtype) == RP_KV_FP8_E4M3, stream);
  return e == hipSuccess ? RP_OK : hip_fail(e, "prefill KV write kernel launch");
}

// Causal attention within each prompt; with `pages`, also the prompts' K/V
// page writes, in the same launch.
static rp_status prefill_impl(const rp_paged_kv* kv, const rp_prefill_layout* l, const void* q, const void* k,
                              const void* v, float softmax_scale, void* out, float* lse, bool pages,
                              hipStream_t stream) {
  g_err[0] = 0;
  rp::PrefillArgs a{};
  int n_rep = 0;
  rp_status st = prefill_args(kv, l, &a, &n_rep);
  if (st != RP_OK) return st;
  if (!(softmax_scale > 0.f) || !std::isfinite(softmax_scale))
    return fail(RP_ERR_INVALID_ARG, "softmax_scale must be finite and > 0");
  if (l->num_groups == 0 || l->num_tokens == 0) return RP_OK;
  if (q == nullptr || k == nullptr || v == nullptr || !aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16))
    return fail(RP_ERR_INVALID_ARG, "q/k/v must be non-NULL and 16-byte aligned");
  if (out == nullptr || !aligned(out, 16)) return fail(RP_ERR_INVALID_ARG, "out must be non-NULL and 16-byte aligned");
  if (lse != nullptr && !aligned(lse, 4)) return fail(RP_ERR_INVALID_ARG, "lse must be 4-byte aligned");
  a.q = q;
  a.k = k;
  a.v = v;
  a.qk_scale = softmax_scale * rp::kLog2e;
  a.out = out;
  a.lse = lse;
  a.write_pages = pages ? 1 : 0;
  hipError_t e = rp::launch_prefill_attn(a, kv->head_dim, n_rep, stream);
  return e == hipSuccess ? RP_OK : hip_fail(e, "prefill attention kernel launch");
}

rp_status rp_prefill_attn(const rp_paged_kv* kv, const rp_prefill_layout* l, const void* q, const void* k,
                          const void* v, float softmax_scale, void* out, float* lse, hipStream_t stream) {
  return prefill_impl(kv, l, q, k, v, softmax_scale, out, lse, false, stream);
}

rp_status rp_prefill(const rp_paged_kv* kv, const rp_prefill_layout* l, const void* q, const void* k, const void* v,
                     float softmax_scale, void* out, float* lse, hipStream_t stream) {
  return prefill_impl(kv, l, q, k, v, softmax_scale, out, lse, true, stream);
}

rp_status rp_plan_layout(const rp_paged_kv* kv, const rp_group_layout* l, rp_plan_info* info) {
  g_err[0] = 0;
  if (info == nullptr) return fail(RP_ERR_INVALID_ARG, "info is NULL");
  Shape sh;
  rp_status st = check_shape(kv, l, &sh);
  if (st != RP_OK) return st;
  WsLayout w;
  if (!ws_layout(sh, &w)) return fail(RP_ERR_UNSUPPORTED, "layout too large for the work plan");
  info->hdr = w.hdr;
  info->grp_off = w.grp_off;
  info->grp_members = w.members;
  info->prefix_items = w.pitems;
  info->resp_items = w.ritems;
  info->seq_parts = w.seq_parts;
  info->part_o = w.part_o;
  info->part_lse = w.part_lse;
  info->max_prefix_items = (int32_t)w.max_pitems;
  info->max_resp_items = (int32_t)w.max_ritems;
  info->parts_per_row = w.max_pc + w.max_rc;
  info->max_parts = (int32_t)w.max_parts;
  return RP_OK;
}

rp_status rp_validate_layout(const rp_paged_kv* kv, const rp_group_layout* l, hipStream_t stream) {
  g_err[0] = 0;
  Shape sh;
  rp_status st = check_shape(kv, l, &sh);
  if (st != RP_OK) return st;
  if (sh.S == 0) return RP_OK;
  int* dres = nullptr;
  hipError_t e = hipMalloc(&dres, 4 * sizeof(int));
  if (e != hipSuccess) return hip_fail(e, "hipMalloc");
  int hres[4] = {0, 0, 0, 0};
  e = hipMemcpyAsync(dres, hres, sizeof(hres), hipMemcpyHostToDevice, stream);
  if (e == hipSuccess) {
    rp::ValidateArgs a;
    a.num_pages = sh.num_pages;
    a.num_seqs = sh.S;
    a.num_groups = sh.G;
    a.seq_to_group = l->seq_to_group;
    a.prefix_lens = l->prefix_lens;
    a.prefix_block_table = l->prefix_block_table;
    a.max_prefix_pages = sh.max_pp;
    a.resp_lens = l->resp_lens;
    a.resp_block_table = l->resp_block_table;
    a.max_resp_pages = sh.max_rp;
    a.result = dres;
    e = rp::launch_validate(a, stream);
  }
  if (e == hipSuccess) e = hipMemcpyAsync(hres, dres, sizeof(hres), hipMemcpyDeviceToHost, stream);
  if (e == hipSuccess) e = hipStreamSynchronize(stream);
  hipError_t ef = hipFree(dres);
  if (e != hipSuccess) return hip_fail(e, "validate_layout");
  if (ef != hipSuccess) return hip_fail(ef, "hipFree");
  if (hres[0] != 0) {
    static const char* kinds[] = {"?", "seq_to_group", "prefix_lens", "resp_lens", "prefix_block_table",
                                  "resp_block_table"};
    const int k = (hres[1] >= 1 && hres[1] <= 5) ? hres[1] : 0;
    return fail(RP_ERR_LAYOUT, "%d bad entries; e.g. %s at index %d has value %d", hres[0], kinds[k], hres[2],
                hres[3]);
  }
  return RP_OK;
}

rp_status rp_selftest_mfma(int32_t shape, const void* a, const void* b, float* c, hipStream_t stream) {
  g_err[0] = 0;
  if (shape < RP_SELFTEST_MFMA_16X16X32 || shape > RP_SELFTEST_MFMA_16X16X32_LDS_TR)
    return fail(RP_ERR_UNSUPPORTED, "self-test shape %d unknown", shape);
  if (a == nullptr || b == nullptr || c == nullptr) return fail(RP_ERR_INVALID_ARG, "a/b/c is NULL");
  if (!aligned(a, 2) || !aligned(b, 2) || !aligned(c, 4))
    return fail(RP_ERR_INVALID_ARG, "a and b must be 2-byte and c 4-byte aligned");
  hipError_t e = rp::launch_selftest_mfma(shape, a, b, c, stream);
  return e == hipSuccess ? RP_OK : hip_fail(e, "self-test kernel launch");
}

rp_status rp_stream_read(const void* src, uint64_t bytes, uint32_t* sink, int32_t nontemporal, hipStream_t stream) {
  g_err[0] = 0;
  if (src == nullptr || sink == nullptr) return fail(RP_ERR_INVALID_ARG, "src/sink is NULL");
  if (!aligned(src, 16) || !aligned(sink, 4)) return fail(RP_ERR_INVALID_ARG, "src must be 16-byte and sink 4-byte aligned");
  if (bytes == 0 || bytes % 16 != 0) return fail(RP_ERR_INVALID_ARG, "bytes must be a positive multiple of 16");
  hipError_t e = rp::launch_stream_read(src, bytes, sink, nontemporal != 0, stream);
  return e == hipSuccess ? RP_OK : hip_fail(e, "stream-read kernel launch");
}

}  // extern "C"

namespace rp {
rp_status set_error(rp_status st, const char* msg) {
  snprintf(g_err, sizeof(g_err), "%s", msg);
  return st;
}
void clear_error() { g_err[0] = 0; }
}  // namespace rp
