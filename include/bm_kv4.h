/*
 * bm_kv4.h -- the bounded cache held in 4 bits (part of libbatchmax).
 *
 * Every K and V row of the cache is stored as 4-bit floats (e2m1: 0, .5, 1,
 * 1.5, 2, 3, 4, 6 and their negatives) with one power-of-two scale for each
 * group of 32 consecutive elements (the OCP microscaling format MXFP4): 4.25
 * bits an element, so the memory of bfloat16 rows holds 3.76 times as many (scores
 * and positions stay as they are).  Groups lie inside one row, so single entries
 * are written, evicted and moved without touching their neighbours.
 *
 *   E   = the smallest integer with max|x_i| <= 6 * 2^E, within [-119, 125]
 *   x^  = 2^E * e2m1(x_i / 2^E), rounded to nearest, ties to the even code
 *
 * The scale byte is E + 127.  Elements beyond 6 * 2^125 become +-6 * 2^125; a
 * group with an infinity or a NaN has the scale byte 255 and reads back as 32
 * NaN.  Every x^ is exact in bfloat16 and in float32, and a row that was read
 * back and is written again keeps its values.
 *
 * A context made by bm_kv4_init or bm_kv4_resume drives such a cache through
 * the calls of batchmax.h: bm_prefill_block, bm_prefill_block_cut,
 * bm_evict_compact, bm_decode_step, the bm_set_* calls and bm_destroy, with the
 * same arguments, checks, order and limits.  A call's own K and V rows are
 * attended to as given and stored in 4 bits; entries cached before the call
 * are attended to as they read back.  Weights of a prefill block's outputs are one
 * bfloat16 each over a bfloat16 batch, as over a cache of that type (outputs are off
 * by 1.9e-3 of their norm, where their own rounding gives 1.6e-3); a decode step
 * keeps two parts.  Scores, positions and lengths are those
 * of batchmax.h.
 *
 * A decode step gives hidden entries (left padding) and slots past the last
 * no weight whatever they hold, NaN included.  A prefill block needs finite
 * query, K and V rows at pad tokens, as bm_prefill_block does over a cache of
 * the element type.
 */
#ifndef BM_KV4_H
#define BM_KV4_H

#include "batchmax.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Elements that share one scale. */
#define BM_KV4_GROUP 32

/* The cache, caller-owned device memory, all C-contiguous; slots =
 * bm_kv4_slots(dims) is cap rounded up to a multiple of 64.  The layouts are what
 * the attention's lanes load 16 bytes at a time; bm_kv4_write and bm_kv4_read
 * convert rows, and a program need not know them.
 *   k        [b, n_kv_heads, slots, head_dim / 2] bytes: element 2i in the lower
 *            half of byte i, element 2i + 1 in the upper half
 *   v        [b, n_kv_heads, slots / 4, head_dim / 8, 4] words of 32 bits: eight
 *            codes each, lowest element first; four slots lie side by side
 *   k_scale  [b, n_kv_heads, slots / 64, head_dim / 32, 64] bytes: slot 16 t + i
 *            (t < 4, i < 16) of the 64 at byte 4 i + t
 *   v_scale  the same with slot 16 t + 4 h + r (t, h, r < 4) at 16 h + 4 t + r
 *   (these four 16-byte aligned)
 *   score, pos, len   as in bm_cache, of cap slots
 *   work              bm_kv4_workspace_bytes(dims) bytes of scratch, 16-byte
 *                     aligned; contents need not survive between calls (but
 *                     for BM_RANK_TOVA's weights, as in bm_cache) */
typedef struct bm_kv4_cache {
  void* k;
  void* v;
  void* k_scale;
  void* v_scale;
  float* score;
  int32_t* pos;
  int32_t* len;
  void* work;
  size_t work_bytes;
} bm_kv4_cache;

/* Slots a unit has in the planes of a 4-bit cache; -1 if dims are invalid. */
int32_t bm_kv4_slots(const bm_dims* dims);

/* Bytes of bm_kv4_cache.work; 0 if dims are invalid.  They hold
 * bm_workspace_bytes(dims) and one layer's cached rows in the element type of
 * dims.dtype, which a prefill block reads back once for all its queries;
 * layers that run one after another can share it.  Every context needs them, also
 * one that only decodes: a single layer with a workspace of its own takes more
 * memory than one of bfloat16 rows (64 samples, 8 heads, 768 slots of 128, blocks
 * of 256 and four query heads a KV head: 57 + 219 MB against 204 + 17); what 4 bits
 * save, they save over layers that share one. */
size_t bm_kv4_workspace_bytes(const bm_dims* dims);

/* bm_init over a 4-bit cache: enqueues the zeroing of len and score. */
int bm_kv4_init(const bm_dims* dims, const bm_kv4_cache* cache, hipStream_t stream, bm_ctx** out);

/* bm_resume over a 4-bit cache that already holds `len` entries per unit. */
int bm_kv4_resume(const bm_dims* dims, const bm_kv4_cache* cache, int32_t len, int32_t next_pos,
                  bm_ctx** out);

/* Store n rows of every unit in slots slot0 .. slot0 + n - 1 of the cache.
 *   k, v  point at row 0 of [b, n_kv_heads, seq_ld, head_dim] buffers of the
 *         element type of dims.dtype, 16-byte aligned; seq_ld >= n
 * Scores, positions and lengths are left as they are, the other slots too.
 * The cache's work, score, pos and len are not read and may be null.
 * BM_ERR_CAPACITY if slot0 + n exceeds cap; n = 0 is a no-op. */
int bm_kv4_write(const bm_dims* dims, const bm_kv4_cache* cache, int32_t slot0, int32_t n,
                 const void* k, const void* v, int32_t seq_ld, hipStream_t stream);

/* The inverse: slots slot0 .. slot0 + n - 1 of every unit into rows 0 .. n - 1
 * of k and v.  Rows from n on are left as they are.  BM_ERR_INVALID_ARG if a row of k
 * and one of v overlap. */
int bm_kv4_read(const bm_dims* dims, const bm_kv4_cache* cache, int32_t slot0, int32_t n, void* k,
                void* v, int32_t seq_ld, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* BM_KV4_H */
