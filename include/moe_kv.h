/*
 * moe_kv.h - C ABI of the operators around a paged cache of keys and values in 4 bits (B200, sm_100a).
 *
 * They are the other half of a served layer next to the MoE module of moe.h: page tables of a batch of
 * requests, rotary positions, storing keys and values in 4 bits, and attention over what is stored.
 * Status codes, dtypes and conventions are those of moe.h: every call is asynchronous on the stream it
 * is given, a plan serves one stream at a time, nothing of the caller's is kept after the call returns,
 * every function returns MOE_OK or a negative MOE_ERR_* code, nothing aborts.  Arrays lie on their type's
 * alignment (ALIGN otherwise) unless a call says more.  What only the device can
 * see (a page number outside the cache, a free list that is too short) skips the access and is kept in
 * the plan's status word, which moe_kv_device_status reads.
 *
 * THE CACHE.  cache[page][kv head][page_size/16] blocks of 16 tokens, dense, 16-byte aligned.  With
 * W = head_dim rounded up to 64, 128 or 256 a block has 18 W bytes:
 *
 *   offset 0     key codes     [16 tokens][W/2 bytes], dimension 2i in the low half of byte i
 *   offset 8 W   value codes   [8 stretches of W/8 dimensions][16 tokens][W/16 bytes]; the byte offset
 *                              token*(W/16) inside stretch r is XORed with 32*((r/2)%2), 64*(r%2) or
 *                              16*(r%2) for W = 64, 128, 256 (shared-memory banks of the attention)
 *   offset 16 W  key scales    [16 tokens][W/16]     one e4m3 byte for 16 dimensions
 *   offset 17 W  value scales  [W/16][16 tokens]
 *
 * A code is e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and the sign in its top bit); the number held is
 * code * scale * k_scale (v_scale for values), k_scale and v_scale being two fp32 numbers of the layer,
 * positive and normal.
 * For the 16 numbers x of a group: scale = e4m3(max|x| / (6 k_scale)), code = e2m1(x / (scale k_scale)),
 * both rounded to nearest even and held at their largest value.  A NaN is stored as 0, an infinity as
 * the largest value; either sets MOE_KV_STATUS_NONFINITE.
 */
#ifndef LEXI_MOE_KV_H_
#define LEXI_MOE_KV_H_

#include <stdint.h>

#include "moe.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Bits that moe_kv_device_status reports through *bits. */
enum {
    MOE_KV_STATUS_TIMEOUT   = 1,   /* a bounded device-side wait ran out                                  */
    MOE_KV_STATUS_BAD_INDEX = 2,   /* a page, slot, position or length outside its range; access skipped  */
    MOE_KV_STATUS_NO_PAGES  = 4,   /* the free list or the row of the block table was too short           */
    MOE_KV_STATUS_NONFINITE = 8    /* a NaN or an infinity was stored                                     */
};

typedef struct {
    int32_t n_heads;       /* query heads, a multiple of n_kv_heads                     */
    int32_t n_kv_heads;    /* key/value heads                                           */
    int32_t head_dim;      /* multiple of 8, 8..256                                     */
    int32_t page_size;     /* tokens a page: 16, 32, 64 or 128                          */
    int32_t max_requests;  /* largest number of requests of a call, 1..4096             */
    int32_t max_tokens;    /* largest number of new tokens of a call, >= 1; times n_heads at most 2^30 */
    int32_t dtype;         /* moe_dtype_t of queries, keys, values and outputs          */
} moe_kv_config_t;

/* Rows [tokens][heads][head_dim] with strides in elements; the dimensions of a head are neighbours. */
typedef struct {
    const void *data;
    int64_t token_stride;
    int64_t head_stride;
} moe_kv_rows_t;

/* How the angle of dimension pair i (of rope_dim/2) is stretched for contexts longer than the trained one. */
typedef enum {
    MOE_ROPE_PLAIN  = 0,   /* theta_i = base^(-2i/rope_dim)                                               */
    MOE_ROPE_LINEAR = 1,   /* theta_i / factor (positions interpolated)                                   */
    MOE_ROPE_BASE   = 2,   /* the base is raised to base * factor^(rope_dim/(rope_dim-2))                 */
    MOE_ROPE_PARTS  = 3,   /* pairs that turn more than `high` times over original_context keep theta_i, those
                              that turn less than `low` times get theta_i/factor, a straight ramp over the pair
                              index between (low < high; usually 1 and 32), ends rounded outwards to whole pairs;
                              magnitude 0 stands for 0.1 ln(factor) + 1                                    */
    MOE_ROPE_BANDS  = 4    /* the same ends (`low`, `high` turns over original_context; usually 1 and 4), the
                              ramp straight in the number of turns                                         */
} moe_rope_scaling_t;

typedef struct {
    int32_t rope_dim;          /* leading dimensions that turn: even, 2..head_dim      */
    int32_t scaling;           /* moe_rope_scaling_t                                   */
    double  base;              /* 10000 usually; > 0                                   */
    double  factor;            /* >= 1                                                 */
    double  low, high;         /* PARTS and BANDS                                      */
    double  original_context;  /* PARTS and BANDS: tokens of the trained context       */
    double  magnitude;         /* on cos and sin; 0 = 1 (PARTS: see there)             */
} moe_rope_config_t;

enum { MOE_ROPE_HALF = 0,      /* dimension i turns with i + rope_dim/2                */
       MOE_ROPE_PAIRS = 1 };   /* dimension 2i turns with 2i + 1                       */

typedef struct moe_kv_plan moe_kv_plan_t;

/* Validates the shapes and allocates the workspace (partial results of attention split over a long
 * context, counters, the status word) on the current device, the plan's.  Calls that launch are made with
 * that device current; reading the status word and destroying are not bound to it.  Synchronises.
 * Errors: INVALID_ARG, SHAPE, CUDA (no sm_100 device), WORKSPACE. */
int moe_kv_plan_create(const moe_kv_config_t *cfg, moe_kv_plan_t **out);
int moe_kv_plan_destroy(moe_kv_plan_t *plan);               /* synchronises the plan's device; NULL is accepted */
uint64_t moe_kv_plan_workspace_bytes(const moe_kv_plan_t *plan);
uint64_t moe_kv_plan_launch_count(const moe_kv_plan_t *plan);

/* Bytes of one page of the cache for this configuration (all key/value heads); 0 for a bad one. */
uint64_t moe_kv_page_bytes(const moe_kv_config_t *cfg);

/* Reads and clears the status word behind what is on the stream, one of the plan's device (NULL: its
 * default stream); synchronises the stream.  *bits (may be NULL) receives the
 * MOE_KV_STATUS_* bits.  Returns MOE_OK, MOE_ERR_TIMEOUT or MOE_ERR_DEVICE_CHECK. */
int moe_kv_device_status(moe_kv_plan_t *plan, int32_t *bits, void *cuda_stream);

/*
 * moe_kv_tables: the bookkeeping of one step, from lengths that are on the device.
 * Request i has ctx_len[i] tokens in the cache (its row of block_table names their pages) and new_len[i]
 * new ones.  With P = page_size it needs ceil((ctx+new)/P) - ceil(ctx/P) fresh pages; these are taken
 * from free_pages in order, request 0's first, and entered into its row of block_table [n_requests,
 * table_width], whose other entries stay.  For the new tokens, request after request:
 *   position[t] = ctx_len[i] + its number within the request,   slot[t] = page * P + position[t] % P,
 * cu_new [n_requests + 1] their running sum, kv_len[i] = ctx_len[i] + new_len[i], pages_taken[0] the
 * fresh pages that the step needs (more than n_free: NO_PAGES, and the entries and slots without a page
 * are -1).  n_tokens is the capacity of position and slot: entries behind the last new token get slot
 * -1 and position 0; new tokens behind the capacity set BAD_INDEX.  A negative length counts as 0 and
 * sets BAD_INDEX.  A position outside the row of the table gets slot -1 (NO_PAGES), one whose page is given
 * as a negative number too (BAD_INDEX).
 * ctx_len and the free list are not changed: kv_len is the next step's ctx_len, and the caller's free
 * list then begins pages_taken entries later.  Errors: INVALID_ARG, ALIGN, CUDA.
 */
int moe_kv_tables(moe_kv_plan_t *plan, const int32_t *ctx_len, const int32_t *new_len, int32_t n_requests,
                  const int32_t *free_pages, int32_t n_free, int32_t *block_table, int32_t table_width,
                  int32_t n_tokens, int32_t *kv_len, int32_t *cu_new, int32_t *position, int64_t *slot,
                  int32_t *pages_taken, void *cuda_stream);

/* Fills table [n_positions, rope_dim/2, 2] (fp32 cos, sin of position * theta_i, times the magnitude;
 * angles in 64 bits).  Errors: INVALID_ARG, ALIGN (8 bytes), CUDA. */
int moe_rope_table(const moe_rope_config_t *rope, int32_t n_positions, float *table, void *cuda_stream);

/*
 * moe_rope: y = x with the first rope_dim dimensions of every head turned by its token's position
 *   (u, w) -> (u cos - w sin, w cos + u sin),
 * in fp32, rounded once.  inverse = 1 turns back: the gradient with respect to x, given the one with
 * respect to y.  table as from moe_rope_table, n_positions its rows; a position outside sets BAD_INDEX
 * and leaves the token unturned.  y may be x with the same strides (in place) and must not overlap it
 * otherwise.  Any strides and any alignment of the type; rows on 16-byte boundaries are faster.
 * Errors: INVALID_ARG, SHAPE (odd rope_dim), ALIGN, CUDA.
 */
int moe_rope(moe_kv_plan_t *plan, const moe_kv_rows_t *x, int32_t n_tokens, int32_t n_heads,
             const int32_t *position, const float *table, int32_t n_positions, int32_t rope_dim,
             int32_t layout, int32_t inverse, void *y, int64_t y_token_stride, int64_t y_head_stride,
             void *cuda_stream);

/*
 * moe_kv_append: turns the new tokens' queries and keys (moe_rope) and stores keys and values at the
 * tokens' slots (slot -1: not stored; a slot outside the cache sets BAD_INDEX), all in one launch.
 * Keys are quantised from the turned fp32 numbers, without rounding in between.  q may be NULL (no
 * queries); q_out [n_tokens][n_heads][head_dim] dense, may be q itself if that is dense.  rope_dim = 0:
 * nothing turns (position and table may be NULL; with q given, q_out is its copy).
 * Two tokens of a call must not have the same slot.  Errors: INVALID_ARG, SHAPE, ALIGN, CUDA.
 */
int moe_kv_append(moe_kv_plan_t *plan, const moe_kv_rows_t *q, const moe_kv_rows_t *k, const moe_kv_rows_t *v,
                  int32_t n_tokens, const int32_t *position, const float *table, int32_t n_positions,
                  int32_t rope_dim, int32_t layout, const int64_t *slot, float k_scale, float v_scale,
                  void *q_out, void *cache, int32_t n_pages, void *cuda_stream);

/* moe_kv_read: the rows at n_tokens slots as the numbers they stand for, k and v [n_tokens][n_kv_heads]
 * [head_dim] dense, of the plan's dtype (bf16: rounded to nearest); either may be NULL.  Slot -1 gives
 * zeros, one outside the cache also sets BAD_INDEX.  Errors: INVALID_ARG, ALIGN, CUDA. */
int moe_kv_read(moe_kv_plan_t *plan, const void *cache, int32_t n_pages, const int64_t *slot, int32_t n_tokens,
                float k_scale, float v_scale, void *k, void *v, void *cuda_stream);

/*
 * moe_kv_attention: softmax attention of every new token over its request's cache.
 * Request i has kv_len[i] tokens in the cache, of which the last cu_new[i+1] - cu_new[i] are the new ones,
 * rows cu_new[i].. of q and out [n_tokens, n_heads, head_dim] (out dense).  With p the token's position,
 *   out = sum_j softmax_j(softmax_scale * q . k_j) v_j     over j <= p and, if window > 0,
 *                                                          p - j < window or j < sinks.
 * A row that sees no key (kv_len[i] = 0, or more new tokens than kv_len[i]) is 0; rows of q that belong
 * to no request are not written.  Query head h reads key/value head h / (n_heads / n_kv_heads).
 * max_new: the largest number of new tokens of a request, which only chooses the kernels; 0 = unknown.
 * Products in 16 bits with fp32 sums for bf16 (the stored numbers are exact there; queries are too, the
 * softmax weights have 11 bits); for fp32 queries and weights are split in two 16-bit parts.
 * A page number outside the cache sets BAD_INDEX and its keys count as absent.
 * Errors: INVALID_ARG, SHAPE (table_width * page_size above 2^30), ALIGN, CUDA.
 */
int moe_kv_attention(moe_kv_plan_t *plan, const moe_kv_rows_t *q, int32_t n_tokens, const int32_t *cu_new,
                     const int32_t *kv_len, int32_t n_requests, int32_t max_new, const int32_t *block_table,
                     int32_t table_width, const void *cache, int32_t n_pages, float softmax_scale,
                     float k_scale, float v_scale, int32_t window, int32_t sinks, void *out,
                     void *cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* LEXI_MOE_KV_H_ */
