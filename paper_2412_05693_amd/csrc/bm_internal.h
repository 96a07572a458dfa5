// Internal declarations shared by the C-ABI host code and the HIP kernel files.
// Not part of the public ABI (include/batchmax.h is).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "batchmax.h"
#include "bm_draft.h"
#include "bm_kv4.h"
#include "bm_probe.h"
#include "bm_synth.h"
#include "bm_window.h"

namespace bm {

// Prefill attention tiling (gfx950: 64-wide waves, 32x32 MFMA tiles).
// A workgroup has 4 waves; each wave owns 32 query rows of one query head, so a
// workgroup covers 128 / G consecutive block positions of one unit for all G
// heads of its group.  Keys stream through LDS in tiles of 64.
constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kRowsPerWave = 32;
constexpr int kKeyTile = 64;
constexpr int kMaxCap = 4096;          // cuts keep up to this many keys in registers
constexpr int kMaxCapAny = 1 << 16;    // slots per unit (larger cuts stream their keys)
constexpr int kMaxDecodeLen = 4097;    // entries one decode step attends to (LDS rows)
constexpr int kMaxBlock = 1024;
// MI355X's last-level (Infinity) cache: 256 MiB
constexpr size_t kLastLevelCacheBytes = (size_t)256 << 20;

// Ranking key of a cut packed with the position into 64 bits, (key bits << 32
// | pos); every key is >= 0 (scores are sums of probabilities), so the integer
// order is (key ascending, pos ascending): the smallest key goes first and, on
// an exact tie, the older entry.
//   BM_RANK_AVE:    ave = score / (curr_id + 1 - pos), correctly rounded fp32
//   BM_RANK_SUM:    score
//   BM_RANK_RECENT: pos alone (the oldest entry goes first)
//   BM_RANK_TOVA:   last, the last processed query's weight
__device__ __forceinline__ uint64_t rank_key(int rule, float score, float last, int pos,
                                             int curr_id) {
  if (rule == BM_RANK_RECENT) return (uint64_t)(uint32_t)pos;
  const float k = rule == BM_RANK_SUM    ? score
                  : rule == BM_RANK_TOVA ? last
                                         : score / (float)(curr_id + 1 - pos);
  return ((uint64_t)__float_as_uint(k) << 32) | (uint32_t)pos;
}

// slots a unit has in the planes of a 4-bit cache
inline int kv4_slots(int cap) { return (cap + 63) & ~63; }

inline int positions_per_wg(int group) { return kWaves * kRowsPerWave / group; }

// Workspace carve-up (all offsets 256-byte aligned).
struct Layout {
  int npt;              // prefill workgroups per unit for a full block
  size_t partial_off;   // float  [U][npt][cap]  per-workgroup score column sums
  size_t holes_off;     // int32  [U][cap]       evicted slots below kv_max, slot order
  size_t srcs_off;      // int32  [U][cap]       surviving slots at or above kv_max
  size_t mcount_off;    // int32  [U]            number of moves per unit
  size_t lastw_off;     // float  [U][cap]       last query's weights (TOVA key)
  size_t total;
};

Layout workspace_layout(const bm_dims& d);

struct PrefillArgs {
  const void* q;      // row t0 of [b, H, seq_ld, D]
  const void* kin;    // row t0 of [b, Hk, seq_ld, D]
  const void* vin;
  void* o;
  void* kc;           // cache [U, cap, D]
  void* vc;
  int32_t* pos;       // [U, cap]
  float* score;       // [U, cap]
  int32_t* len;       // [U]
  float* partial;     // [U, npt, cap]
  int64_t seq_ld;
  int n_heads, n_kv_heads, cap, len0, n_tok, t0, npt_used, npt_stride, units;
  int nsplit;         // workgroups per position tile (set by launch_prefill)
  int accumulate;     // 0: outputs only (no score sums; new entries get score 0)
  int append;         // 0: the block's rows are stored elsewhere, kc and vc are only read
  const int32_t* pad; // [b] left pad tokens per sample, or null
  float* lastw;       // [U, cap] weights of the block's last query, or null
  float scale_log2;   // sm_scale * log2(e)
};

struct EvictArgs {
  void* kc;
  void* vc;
  float* score;
  int32_t* pos;
  int32_t* len;
  int32_t* holes;
  int32_t* srcs;
  int32_t* mcount;
  int cap, n, kv_max, curr_id, units, head_dim, elem_bytes;
  int rule;           // bm_rank_rule
  float* lastw;       // [U, cap] last query's weights (moved with the entries), or null
  // a cache held in 4 bits: kc and vc are its code planes, these its scales, all of
  // `slots` slots a unit (bm_kv4.h)
  void* ks = nullptr;
  void* vs = nullptr;
  int slots = 0;
  int row_bytes() const { return ks ? head_dim / 2 : head_dim * elem_bytes; }
};

struct DecodeArgs {
  const void* q;      // [b, H, seq_ld, D] row of this step
  const void* kin;    // [b, Hk, seq_ld, D]
  const void* vin;
  void* o;
  void* kc;
  void* vc;
  float* score;
  int32_t* pos;
  int32_t* len;
  int64_t seq_ld;
  int n_heads, n_kv_heads, cap, len0, kv_max, cur_pos, units;   // kv_max: the decode bound
  int rule;           // bm_rank_rule
  const int32_t* pad; // [b] left pad tokens per sample, or null
  float* lastw;       // [U, cap] this step's weights are written here, or null
  float scale_log2;
};

struct LongDecodeArgs {
  const void* q;      // [b, H, seq_ld, D] row of this step
  const void* kin;    // [b, Hk, seq_ld, D]
  const void* vin;
  void* o;
  void* kc;
  void* vc;
  float* score;
  int32_t* pos;
  int32_t* len;
  float* part;        // [U][nsplit][G][D + 2] chunk partials (o, m, l)
  int64_t seq_ld;
  int n_heads, n_kv_heads, cap, len0, cur_pos, units, nsplit;
  const int32_t* pad; // [b] left pad tokens per sample, or null
  float scale_log2;
};

// A step over a cache held in 4 bits, scoring or split over key chunks.
struct Kv4DecodeArgs {
  const void* q;      // [b, H, seq_ld, D] row of this step
  const void* kin;    // [b, Hk, seq_ld, D]
  const void* vin;
  void* o;
  void* kq;           // the planes of bm_kv4.h, `slots` slots a unit
  void* vq;
  void* ks;
  void* vs;
  float* score;       // [U, cap]
  int32_t* pos;
  int32_t* len;
  float* part;        // [U][nsplit][G][D] partial outputs of a split step, then their [..][2] (m, l)
  int64_t seq_ld;
  int n_heads, n_kv_heads, cap, slots, len0, kv_max, cur_pos, units, nsplit;   // kv_max: the decode bound
  int rule;           // bm_rank_rule
  const int32_t* pad; // [b] left pad tokens per sample, or null
  float* lastw;       // [U, cap] this step's weights are written here, or null
  float scale_log2;
};

// Rows 0 .. n - 1 of [U, seq_ld, D] buffers to or from slots slot0 .. of a 4-bit cache.
struct Kv4RowsArgs {
  const void* k = nullptr;    // (a read writes through them)
  const void* v = nullptr;
  void* kq = nullptr;
  void* vq = nullptr;
  void* ks = nullptr;
  void* vs = nullptr;
  int64_t seq_ld = 0;
  int units = 0, slots = 0, slot0 = 0, n = 0;
};

// Tokens t0 .. t0 + n_tok - 1 through a window cache (bm_window.h).
struct PromptArgs {
  const void* q;      // row t0 of [b, H, seq_ld, D]
  const void* kin;    // row t0 of [b, Hk, seq_ld, D]
  const void* vin;
  void* o;
  void* kc;           // cache [U, window + sinks, D]
  void* vc;
  const int32_t* pad; // [b] left pad tokens per sample, or null
  int64_t seq_ld;
  float* part;        // scratch of prompt_work_bytes
  int n_heads, n_kv_heads, units, window, sinks, t0, n_tok;
  int nsplit;         // workgroups over the keys of a row block (set by launch_prompt)
  float scale_log2;
};

// tokens of a prompt that can be taken as the nodes of a chain (BM_DRAFT_MAX at most)
constexpr int kShortPrompt = 64;

// The n nodes of a tree (one: a token) over a cache: a bounded one of len0 entries
// (window 0) or a window cache.
struct NodesArgs {
  const void* q;      // [b, H, seq_ld, D] row 0
  const void* kin;    // [b, Hk, seq_ld, D]
  const void* vin;
  void* o;
  float* lse;         // [b, H, n] or null
  const int32_t* parent;   // [b, n], or null: every node is a root
  void* kc;           // cache [U, slots, D]
  void* vc;
  const int32_t* pos; // [U, slots] (bounded cache)
  const int32_t* pad; // [b] left pad tokens per sample, or null
  float* part;        // [U][nsplit][G n][D] partial outputs, then their [..][2] (m, l)
  int64_t seq_ld;
  int n_heads, n_kv_heads, units, slots, len0, n, next_pos, window, sinks;
  int nsplit;         // workgroups over a unit's entries (set by launch_nodes)
  int chain;          // each node hangs from the one before it (parent is null)
  int store;          // the node's rows go into the window cache (n == 1)
  float scale_log2;
};

// m of a tree's n nodes behind a cache.
struct AcceptArgs {
  const void* q;      // [b, H, seq_ld, D] row 0
  const void* kin;    // [b, Hk, seq_ld, D]
  const void* vin;
  const float* lse;   // [b, H, n], or null: no scores
  const int32_t* path;     // [b, m]
  const int32_t* count;    // [b] or null
  void* kc;           // cache [U, slots, D]
  void* vc;
  float* score;       // [U, slots] (bounded cache)
  int32_t* pos;
  int32_t* len;       // [U]
  float* lastw;       // [U, slots] weights of the last accepted query, or null
  int32_t* pad;       // [b], or null
  int64_t seq_ld;
  int n_heads, n_kv_heads, units, slots, len0, n, m, next_pos, window, sinks;
  float scale_log2;
};

struct SynthArgs {
  void* q;
  void* k;
  void* v;
  int b, n_heads, n_kv_heads, head_dim, dtype, layer, s, n_sinks, t0, n_rows;
  int64_t seq_ld;
  uint32_t seed, hh_threshold;
  float hh_scale, sink_scale, value_scale;
};

hipError_t launch_prefill(const PrefillArgs& a, int dtype, int head_dim, int group,
                          hipStream_t stream);
// workgroups per position tile of that launch
int prefill_split(const PrefillArgs& a, int row_bytes);
hipError_t launch_score_reduce(const PrefillArgs& a, hipStream_t stream);
hipError_t launch_select(const EvictArgs& a, hipStream_t stream);
hipError_t launch_fold_cut(const PrefillArgs& pa, const EvictArgs& a, int pt_positions,
                           hipStream_t stream);
// select and compaction of a.n <= kMaxCap entries in one launch
hipError_t launch_cut(const EvictArgs& a, hipStream_t stream);
hipError_t launch_compact(const EvictArgs& a, int max_moves, hipStream_t stream);
hipError_t launch_decode(const DecodeArgs& a, int dtype, int head_dim, int group,
                         hipStream_t stream);
int long_decode_splits(int len0);
hipError_t launch_decode_long(const LongDecodeArgs& a, int dtype, int head_dim, int group,
                              hipStream_t stream);
hipError_t launch_kv4_decode(const Kv4DecodeArgs& a, int dtype, int head_dim, int group,
                             hipStream_t stream);
int kv4_long_splits(int len0);
hipError_t launch_kv4_long(const Kv4DecodeArgs& a, int dtype, int head_dim, int group,
                           hipStream_t stream);
// read rows, then (independently: no slot and no row twice) write rows; either may have n = 0
hipError_t launch_kv4_rows(const Kv4RowsArgs& read, const Kv4RowsArgs& write, int dtype,
                           int head_dim, hipStream_t stream);
hipError_t launch_prompt(PromptArgs a, int dtype, int head_dim, int group, hipStream_t stream);
// whether a launch of that size can be made
bool prompt_fits(int units, int group, int n_tok);
// bytes of PromptArgs.part for calls of up to n tokens
size_t prompt_work_bytes(int units, int head_dim, int group, int n, bool bf16);
hipError_t launch_nodes(const NodesArgs& a, int dtype, int head_dim, int group, hipStream_t stream);
// bytes of NodesArgs.part for n nodes, whatever the cache holds
size_t nodes_work_bytes(int units, int head_dim, int group, int n);
// the join of launch_nodes alone: NodesArgs' o, part, seq_ld, units, heads, n and nsplit (> 1, 64 at most)
hipError_t launch_nodes_join(const NodesArgs& a, int dtype, int head_dim, hipStream_t stream);
hipError_t launch_accept(const AcceptArgs& a, int dtype, int head_dim, int group, hipStream_t stream);
hipError_t launch_reset(float* score, int32_t* len, size_t n_score, size_t n_len,
                        hipStream_t stream);
hipError_t launch_synth_qkv(const SynthArgs& a, hipStream_t stream);
hipError_t launch_philox(const uint32_t* in, uint32_t* out, int64_t n, hipStream_t stream);
hipError_t launch_probe_read(const void* src, size_t bytes, uint32_t* sink, int blocks, bool nt,
                             hipStream_t stream);
hipError_t launch_probe_mfma(int iters, float* sink, int blocks, hipStream_t stream);
// prefill timeline records (a BM_PREFILL_TIMELINE build; else hipErrorNotSupported)
bool timeline_enabled();
hipError_t read_timeline(uint64_t* dst, int n_records);

}  // namespace bm
