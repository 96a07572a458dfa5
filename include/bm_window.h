/*
 * bm_window.h -- attention with a sliding window and sinks (part of libbatchmax).
 *
 * The index of a token is its position less the left pad of its sample
 * (bm_set_left_padding).  The token at index i attends to the last `window` tokens,
 * its own included, and to the first `sinks` tokens of its sample:
 *
 *   key j is visible to query i  <=>  0 <= j <= i  and  (j < sinks or i - j < window)
 *
 * whatever the calls that brought the tokens: the mask is every query's own, where a
 * bounded cache cut by BM_RANK_RECENT shows all queries of a block the same entries.
 * There are no scores and no cuts.  Pad tokens (index below 0) are visible to no query
 * and give zeros; their rows are never read.
 *
 * A context made by bm_win_init or bm_win_resume drives such a cache through the calls
 * of batchmax.h: bm_prefill_block (and bm_prefill_block_cut, the same here) with up to
 * dims.block tokens a call, bm_decode_step, bm_set_left_padding, bm_set_split_event,
 * bm_evict_compact (never anything to cut) and bm_destroy, and those of bm_draft.h, with
 * the same arguments, order and errors.  The settings that concern scores and cuts
 * (bm_set_rank_rule, bm_set_decode_removal, bm_set_decode_bound and
 * bm_set_score_accumulation) return BM_ERR_UNSUPPORTED.  bm_ctx_len is the number of
 * slots that a sample without padding has filled.
 *
 * bfloat16: a prefill call of more than 64 tokens, or of more than 128 query rows a KV head
 * (tokens times query heads), rounds each softmax weight to bfloat16 before its product
 * with V, as bm_prefill_block over a bounded cache does; shorter calls, single tokens and
 * drafted ones carry weights to 2^-16.  So the last bits of an output depend on how its
 * prompt was cut into calls: 2.3e-3 and 1.6e-3 (relative, root mean square) from the exact
 * one, of which 1.6e-3 are the output's own rounding.  Float32 calls have no such step.
 *
 * bm_set_split_event's event is recorded behind a prefill call's launches.
 *
 * What a slot without a token holds is of no weight, NaN included, and so is what a
 * pad token's rows hold.  Rows of real tokens have to be finite: in a call's result a
 * NaN or infinity of a V row also reaches queries of the same call that do not see it.
 */
#ifndef BM_WINDOW_H
#define BM_WINDOW_H

#include "batchmax.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The cache, caller-owned device memory, C-contiguous, 16-byte aligned.
 *   k, v  [b, n_kv_heads, kv_max, head_dim] of dims.dtype: dims.kv_max = window + sinks
 *         slots a unit.  Token j < sinks lies in slot j, any other one in slot
 *         sinks + (j - sinks) mod window.
 *   work  bm_win_workspace_bytes(dims) bytes of scratch; contents need not survive
 *         between calls, so layers that run one after another can share it. */
typedef struct bm_win_cache {
  void* k;
  void* v;
  void* work;
  size_t work_bytes;
} bm_win_cache;

/* Bytes of bm_win_cache.work; 0 if dims are invalid. */
size_t bm_win_workspace_bytes(const bm_dims* dims);

/* Check dims and sinks alone.  dims.kv_max = window + sinks with window >= 1 and
 * sinks >= 0, at most 65535; dims.block (the most tokens of one prefill call) is not
 * bounded by the library; everything else as bm_validate_dims. */
int bm_win_validate(const bm_dims* dims, int32_t sinks);

/* A context over an empty window cache; no device work. */
int bm_win_init(const bm_dims* dims, int32_t sinks, const bm_win_cache* cache, bm_ctx** out);

/* A context over a cache that holds the rows of the tokens before next_pos.  Also how a turn
 * of several tokens follows generated ones, since a context prefills while its next
 * position is below dims.s and generates from there on: a new context over the same cache
 * at the same position, with dims.s past the turn (the other one is then destroyed). */
int bm_win_resume(const bm_dims* dims, int32_t sinks, const bm_win_cache* cache,
                  int32_t next_pos, bm_ctx** out);

#ifdef __cplusplus
}
#endif

#endif /* BM_WINDOW_H */
