/*
 * bm_draft.h -- drafted tokens over a cache: a tree's attention, and the acceptance of
 * a path (part of libbatchmax; speculative decoding).
 *
 * A draft model proposes a tree of n tokens behind the cache.  bm_draft_attend computes
 * every node's attention in one pass over the cache and changes nothing;
 * bm_draft_accept then appends the path that the program took.  Both work on contexts
 * of batchmax.h (a bounded cache) and of bm_window.h, after the prompt; a cache held in
 * 4 bits and Algorithm 1's literal removal (bm_set_decode_removal with p > 0) return
 * BM_ERR_UNSUPPORTED.
 *
 * Node a stands at position next_pos + depth(a), a root's depth being 0, and attends to
 * the cached entries, its ancestors and itself; over a window cache, to those of them
 * that the window shows it.  Left padding holds as in bm_decode_step.  K and V rows of
 * nodes that are no ancestor of a node are of no weight to it, NaN included.
 */
#ifndef BM_DRAFT_H
#define BM_DRAFT_H

#include "batchmax.h"
#include "bm_window.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Nodes of a tree, and tokens of an accepted path. */
#define BM_DRAFT_MAX 64

/* Bytes of scratch that bm_draft_attend needs for n nodes, whatever the cache holds; 0
 * for invalid dims or n.  Contents need not survive the call. */
size_t bm_draft_workspace_bytes(const bm_dims* dims, int32_t n);

/* The attention of a tree's nodes, 1 <= n <= BM_DRAFT_MAX.
 *   parent [b, n] int32: each node's parent, which comes before it; any value outside
 *          0 .. (the node's own number) - 1, usually -1, makes the node a root
 *   q, o   point at row 0 of [b, n_heads, seq_ld, head_dim] buffers, k, v at row 0 of
 *          [b, n_kv_heads, seq_ld, head_dim] buffers; seq_ld >= n.  o may be q itself;
 *          it must not overlap k or v.
 *   lse    [b, n_heads, n] float32 or null: log(sum_j exp(sm_scale q.k_j)) over the keys
 *          that a node sees (-infinity for a pad token)
 *   work   bm_draft_workspace_bytes(dims, n) bytes, 16-byte aligned
 * BM_ERR_ORDER before the prompt is processed or beyond s + max_gen.  A cache above the
 * decode bound is first cut to it, as by bm_decode_step. */
int bm_draft_attend(bm_ctx* ctx, int32_t n, const int32_t* parent, const void* q, const void* k,
                    const void* v, void* o, int32_t seq_ld, float* lse, void* work,
                    size_t work_bytes, hipStream_t stream);

/* Append m tokens of a tree of n nodes, 1 <= m <= n, and advance by m positions.
 *   path   [b, m] int32: node numbers, a root and then each one's child.  (A number
 *          outside 0 .. n - 1 is taken as the nearest one inside.)
 *   count  [b] int32 or null: sample j takes the first count[j] of them only (values are
 *          taken within 0 .. m).
 *   q, k, v, seq_ld and lse as bm_draft_attend had them and left them
 * A bounded cache takes them like a prefill block of m tokens: the entries' scores grow
 * by the probabilities that the m queries gave them, read from lse (needed unless score
 * accumulation is off, and then ignored: the new entries get score 0), and a cache of
 * more than the decode bound is cut back to it, ranked at the last token's position.
 * It needs free slots for them (m <= block does; else BM_ERR_CAPACITY).  lse has to be
 * that of the cache as it is: BM_ERR_ORDER if the cache is above the decode bound.
 * A window cache stores their rows (q and lse are not read and may be null).
 *
 * A sample that takes fewer falls behind by m - count[j] positions: its pad
 * (bm_set_left_padding, needed for count, else BM_ERR_ORDER) and the positions of its
 * entries grow by that much ON THE DEVICE, so that its next token again stands next to
 * its last, and in a bounded cache hidden entries of zeros, which leave at the next cut,
 * stand for the tokens that it did not take.  All that depends on ages or distances is
 * as if the sample had run by itself: its own next index is next_pos - pad[j].  So with
 * count each context (each layer's) needs a pad array of its own. */
int bm_draft_accept(bm_ctx* ctx, int32_t n, int32_t m, const int32_t* path, const int32_t* count,
                    const void* q, const void* k, const void* v, int32_t seq_ld, const float* lse,
                    hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* BM_DRAFT_H */
