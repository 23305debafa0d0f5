// Host/device interface between the C-ABI layer and the kernel launchers.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rp_device.h"
#include "rp_host.h"

namespace rp {

// Lengths and group ids are clamped into the table/pool bounds before use, so
// an invalid layout gives wrong numbers but never an out-of-bounds access.
__host__ __device__ inline int clamp_group(int g, int G) { return g < 0 ? 0 : (g >= G ? G - 1 : g); }
__host__ __device__ inline int clamp_len(int len, int max_pages) {
  const int cap = max_pages * kPage;
  return len < 0 ? 0 : (len > cap ? cap : len);
}
__host__ __device__ inline int prefix_chunks(int P, int max_prefix_pages, int max_chunks) {
  const int n = cdiv(cdiv(clamp_len(P, max_prefix_pages), kPage), kPrefixChunkPages);
  return n > max_chunks ? max_chunks : n;
}
__device__ inline int clamp_page(int p, int num_pages) {
  return (unsigned)p < (unsigned)num_pages ? p : 0;
}

struct PlanArgs {
  int num_seqs, num_groups, num_q_heads, num_kv_heads;
  int num_cus;  // compute units of the device the batch runs on (sets the piece length)
  const int* seq_to_group;
  const int* prefix_lens;
  const int* resp_lens;
  int len_add;  // the plan is for resp_lens[s] + len_add response tokens (1: after this step's append)
  int max_prefix_pages, max_resp_pages;
  PlanView view;
};

struct AttnArgs {
  const void* k_pages;
  const void* v_pages;
  const float* k_scale;
  const float* v_scale;
  int num_pages, num_kv_heads;
  int num_seqs, num_groups, num_q_heads;
  const int* seq_to_group;
  const int* prefix_lens;
  const int* prefix_block_table;
  int max_prefix_pages;
  const int* resp_lens;
  const int* resp_block_table;
  int max_resp_pages;
  const void* q;     // bf16 [S][Hq][D]
  float qk_scale;    // softmax_scale * log2(e)
  PlanView view;
};

// Combine input: either an explicit CSR (row_offs != null) or the planned
// fixed slots, whose part counts follow from the lengths.
struct CombineArgs {
  const float* o_parts;
  const float* lse_parts;
  const int* row_offs;   // CSR [num_rows + 1], or null for planned slots
  int num_rows;
  void* out;             // bf16 [rows][D]
  float* lse;            // [rows] or null
  // planned slots only: parts per query row of each sequence, from the plan
  const int* seq_parts;
  int num_q_heads, parts_per_row;
};

struct AppendArgs {
  void* k_pages;
  void* v_pages;
  float* k_scale;
  float* v_scale;
  int num_pages, num_kv_heads, num_seqs;
  const int* resp_lens;
  const int* resp_block_table;
  int max_resp_pages;
  const void* k_new;  // bf16 [S][Hkv][D]
  const void* v_new;
};

// GRPO advantages: rewards [num_groups][group_size] fp32.
struct GrpoArgs {
  const float* rewards;
  int num_groups, group_size, ddof;
  double eps_std;
  float* advantages;  // [num_groups][group_size]
  float* mean;        // [num_groups] or null
  float* stdev;       // [num_groups] or null
  bool vector_ok;     // rewards and advantages 16-byte aligned (group_size 4, 8 or 16 then loads float4)
};

constexpr int kMaxHeadDim = 128;

// Pre-attention side of a decode step: q/k RMS norm + rotary embedding,
// q written out, k and v appended at response slot resp_lens[s].
struct QkPrepArgs {
  void* k_pages;
  void* v_pages;
  float* k_scale;
  float* v_scale;
  int num_pages, num_kv_heads, num_q_heads, num_seqs, num_groups;
  const int* seq_to_group;
  const int* prefix_lens;
  const int* resp_lens;
  const int* resp_block_table;
  int max_resp_pages;
  const uint16_t* q_in;      // bf16 [S][Hq][D]
  const uint16_t* k_in;      // bf16 [S][Hkv][D]
  const uint16_t* v_in;
  const uint16_t* q_norm_w;  // bf16 [D]
  const uint16_t* k_norm_w;
  double rms_eps;
  double inv_freq[kMaxHeadDim / 2];  // rotary frequency of pair i: theta^(-2i/D)
  uint16_t* q_out;           // bf16 [S][Hq][D]
  uint16_t* k_out;           // bf16 [S][Hkv][D] or null
  int blocks_per_seq;        // set by the launcher
};

// Shared-prefix prefill: packed prompt tokens of every group (group g owns
// rows prompt_offs[g] .. prompt_offs[g+1]-1 of q/k/v/out), K/V written once
// into the group's prefix pages.
struct PrefillArgs {
  void* k_pages;
  void* v_pages;
  float* k_scale;
  float* v_scale;
  int num_pages, num_kv_heads, num_groups, num_q_heads, num_tokens;
  const int* prompt_offs;
  const int* prefix_block_table;
  int max_prefix_pages;
  const void* q;  // bf16 [T][Hq][D]
  const void* k;  // bf16 [T][Hkv][D]
  const void* v;
  float qk_scale;  // softmax_scale * log2(e)
  void* out;       // bf16 [T][Hq][D]
  float* lse;      // [T][Hq] or null
  int write_pages;  // attention kernel also writes the K/V pages (one launch for the whole prefill)
};

// A launch has fewer than 2^32 threads.
constexpr long long kMaxBlocks256 = (1ll << 24) - 1;

// Waves of a workgroup of the tree attention, and the forms of its units (keys
// split between waves of 1, 2 or 4 column tiles; row tiles over shared keys).
constexpr int kTreeWaves = 4;
enum class TreeForm { kSplit1, kSplit2, kSplit4, kRows };
// Units that fill the chip, two workgroups to a compute unit, and the fewest
// pages of a piece.
constexpr int kTreeUnits = 512, kTreeLeastPages = 32;
constexpr int kTreeMaxDrafts = 64;
// Most sequences that a launch orders by length.
constexpr int kTreeOrderSeqs = 1024;

// Attention of trees of drafted tokens over the cache.
struct TreeArgs {
  const void* k_pages;
  const void* v_pages;
  const float* k_scale;
  const float* v_scale;
  int num_pages, num_kv_heads;
  int num_seqs, num_groups, num_q_heads;
  int rep_shift;  // log2(num_q_heads / num_kv_heads)
  const int* seq_to_group;
  const int* prefix_lens;
  const int* prefix_block_table;
  int max_prefix_pages;
  const int* resp_lens;
  const int* resp_block_table;
  int max_resp_pages;
  int num_drafts, max_drafts;
  const int* draft_offs;             // [S + 1]
  const unsigned long long* masks;   // [T]
  const uint16_t* q;                 // bf16 [T][Hq][D]
  const uint16_t* k_draft;           // bf16 [T][Hkv][D]
  const uint16_t* v_draft;
  float qk_scale;                    // softmax_scale * log2(e)
  uint16_t* out;                     // bf16 [T][Hq][D]
  float* lse;                        // [T][Hq] or null
  // Partial results (null where every row has one unit), rows in the order of
  // (kv-head, token, query head of the kv-head): of max_prefix_chunks chunks of
  // prefixes and of the sequences' first pieces T * Hq rows each, then from row
  // pieces_at on max_drafts * (Hq / Hkv) = slot_rows rows per other piece and
  // kv-head.
  float* part_o;                     // [rows][D]
  float* part_lse;                   // [rows]
  // [T]: pieces of the token's sequence (0: its rows are stored already) and
  // the token's place in its tree << 16; chunks of its prefix and the first of
  // the other pieces << 16
  int2* token_parts;
  long long pieces_at;
  int slot_rows;
  // How the launch is divided.
  int share;                         // prefixes are units of their own, for all members at once
  int longest_first;                 // so many sequences by decreasing length, the others by increasing; 0: as they are
  int max_prefix_chunks, prefix_repeats, prefix_blocks;
  int seq_pieces, least_pages, max_extra, row_blocks;
  float piece_share;                 // pages of a piece over those of all sequences
};

// K/V rows into the cache by slot.
struct WriteArgs {
  void* k_pages;
  void* v_pages;
  float* k_scale;
  float* v_scale;
  int num_slots;          // num_pages * 16
  int num_kv_heads;
  int num_tokens, num_src;
  const int* slot_map;    // [num_tokens]
  const int* src_rows;    // [num_tokens] or null: row i
  const void* k_new;      // bf16 [num_src][Hkv][D]
  const void* v_new;
  int chunk;              // fp8: list entries per wave, at most 48
};

// Most sequences of a resize: their prefix sums stay in LDS.
constexpr int kTableMaxSeqs = 4096;

struct TableArgs {
  int num_seqs, max_pages, num_pages, max_slots;
  int* block_table;   // [S][max_pages]
  int* free_pages;    // [num_pages], a stack
  int* free_count;    // [1]
  const int* old_lens;
  const int* new_lens;
  int* slot_offs;     // [S + 1] or null
  int* slot_map;      // [max_slots] or null
  int* status;        // [4]
};

struct ValidateArgs {
  int num_pages, num_seqs, num_groups;
  const int* seq_to_group;
  const int* prefix_lens;
  const int* prefix_block_table;
  int max_prefix_pages;
  const int* resp_lens;
  const int* resp_block_table;
  int max_resp_pages;
  int* result;       // [4]: error count, first bad kind, first bad index, value
};

// Rows of logits, and what goes with each (rp.h states the meaning).
struct LogitArgs {
  const void* data;
  int rows, vocab;
  long long stride;  // elements
  int num_cus;       // compute units of the device
};

// Compute units of the current device.
rp_status device_cus(int* cus);

struct SampleArgs {
  LogitArgs logits;
  const float* temperature;
  const int* top_k;
  const float* top_p;
  const float* min_p;
  const float* u;
  int* tokens;
  float* logprobs;
  float* kept;
  void* workspace;  // sample_workspace bytes
};

struct LogprobArgs {
  LogitArgs logits;
  const int* tokens;
  double inv_t;  // 1 / temperature
  float* logprobs;
  float* entropy;
};

struct PolicyArgs {
  LogitArgs logits;
  const int* tokens;
  const float* old_logprobs;
  const float* ref_logprobs;  // null where kl_beta is 0
  const float* advantages;
  const int* row_seq;
  int num_advantages;
  const float* weights;
  double inv_t, clip_low, clip_high, kl_beta, entropy_coef;
  float* losses;
  float* logprobs;
  float* entropy;
  void* dlogits;
  long long dstride;
};

struct DistillArgs {
  LogitArgs logits;
  const int* ids;
  const float* values;
  int k, kind;
  const float* weights;
  double inv_t;
  float* losses;
  void* dlogits;
  long long dstride;
};

hipError_t launch_plan(const PlanArgs& a, hipStream_t stream);
// q/k prep and the plan of the attention after its append in one launch
// (batches of at most 64 sequences; the plan's len_add is 1).
hipError_t launch_qk_prep_plan(QkPrepArgs a, const PlanArgs& p, int head_dim, bool fp8, hipStream_t stream);
// Grid sizes are upper bounds from host scalars; idle waves exit at once.
hipError_t launch_attn_parts(const AttnArgs& a, int head_dim, int n_rep, bool fp8, long long max_prefix_items,
                             long long max_resp_items, hipStream_t stream);
// The whole attention of a small batch, and its plan, in one launch (at most
// 64 sequences).
hipError_t launch_attn_small(const AttnArgs& a, const PlanArgs& p, int head_dim, int n_rep, bool fp8, void* out,
                             float* lse, hipStream_t stream);
hipError_t launch_combine(const CombineArgs& a, int head_dim, hipStream_t stream);
// The second launch, where rows may have several units: merges the partial results.
hipError_t launch_tree_merge(const TreeArgs& a, int head_dim, hipStream_t stream);
hipError_t launch_tree_attn(const TreeArgs& a, int head_dim, bool fp8, TreeForm form, long long blocks,
                            hipStream_t stream);
hipError_t launch_write_slots(const WriteArgs& a, int head_dim, bool fp8, hipStream_t stream);
// One launch, or two where much moves.
hipError_t launch_page_tables(const TableArgs& a, hipStream_t stream);
hipError_t launch_append(const AppendArgs& a, int head_dim, bool fp8, hipStream_t stream);
hipError_t launch_prefill_kv_write(const PrefillArgs& a, int head_dim, bool fp8, hipStream_t stream);
hipError_t launch_prefill_attn(const PrefillArgs& a, int head_dim, int n_rep, hipStream_t stream);
hipError_t launch_qk_prep(QkPrepArgs a, int head_dim, bool fp8, hipStream_t stream);
hipError_t launch_grpo(const GrpoArgs& a, hipStream_t stream);
// Bytes of workspace that sampling takes (0 for many shapes).
size_t sample_workspace(int rows, int vocab, int dtype);
hipError_t launch_sample(const SampleArgs& a, int dtype, hipStream_t stream);
hipError_t launch_logprobs(const LogprobArgs& a, int dtype, hipStream_t stream);
hipError_t launch_policy(const PolicyArgs& a, int dtype, hipStream_t stream);
hipError_t launch_distill(const DistillArgs& a, int dtype, hipStream_t stream);
hipError_t launch_validate(const ValidateArgs& a, hipStream_t stream);
hipError_t launch_selftest_mfma(int shape, const void* a, const void* b, float* c, hipStream_t stream);
hipError_t launch_stream_read(const void* src, uint64_t bytes, uint32_t* sink, bool nontemporal,
                              hipStream_t stream);

}  // namespace rp
