/*
 * svfkv.h -- the paged key-value cache that the scheduler's budget counts:
 * append with rotary positions, attention over pages, eviction by weight.
 *
 * Part of libsvfsim.so.  The simulator (svfsim.h) counts a budget M of cache
 * slots and a step that advances every running request by one token; these
 * calls are that step's work on one layer's cache, so that a schedule can be
 * replayed on the hardware whose budget it plans.  A token of the model of
 * Section 3.1 is one slot; a running request that holds s + x tokens has all
 * of them read by its next step, so the slots read over its life are the
 * volume of Eq. 1.
 *
 * The cache of a layer is a pool of pages.  Slot j of sequence i is row
 * j % page_size of page page_table[i][j / page_size].  Pages may be handed out
 * in any order, and may be shared between sequences as long as nothing is
 * written to them (svf_kv_append, svf_kv_evict and the weights of
 * svf_kv_attend write).
 *
 * Conventions
 *   - Every pointer inside the structs is device memory; the structs
 *     themselves are host memory and are only read during the call.
 *   - Calls are asynchronous on hip_stream, allocate nothing, keep nothing
 *     and may be recorded into a graph.  The current device must be the
 *     stream's.
 *   - Sizes, strides, alignment and flags are checked on the host before
 *     anything is enqueued (SVF_EINVAL, text from svf_kv_last_error).  What lies in
 *     device memory cannot be: there, lengths are cut to [0, table_width *
 *     page_size], offsets to [0, num_tokens], and a slot whose page number is outside
 *     [0, num_pages) is not there (never written, invisible to attention,
 *     evicted before any with a weight).
 *   - A launch has fewer than 2^32 threads; sizes that need more are refused
 *     (some 2^26 tokens in svf_kv_append, 2^22 sequences times key heads in svf_kv_evict,
 *     2^31 rows or 2^24 sequences times key heads with chunks in svf_kv_attend).
 *   - Return codes are those of svfsim.h.
 */
#ifndef SVFKV_H
#define SVFKV_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of queries, keys, values and outputs. */
enum {
    SVF_KV_BF16 = 0,
    SVF_KV_F16 = 1
};

/* Which two of the rotated dimensions form a pair. */
enum {
    SVF_KV_ROPE_HALF = 0,        /* d and d + rot/2                           */
    SVF_KV_ROPE_INTERLEAVED = 1  /* 2d and 2d + 1                             */
};

/*
 * One layer's cache.  Element (page, head, row, d) of k is at
 * k[page * k_page_stride + head * k_head_stride + row * k_row_stride + d]; v
 * the same.  Strides are in elements, multiples of 8, those of pages and rows
 * below 2^31; k and v are aligned to 16 bytes.
 *   page_size  a power of two, 1 .. 65536;  num_pages * page_size < 2^31
 *   head_dim   64, 128 or 256
 *   weight     float [num_pages][kv_heads][page_size]: each slot's summed
 *              attention weight; NULL where it is not kept
 *   position   int32 [num_pages][kv_heads][page_size]: each slot's token
 *              position (heads evict different tokens); NULL where not kept
 */
typedef struct svf_kv_cache {
    void *k;
    void *v;
    float *weight;
    int32_t *position;
    int64_t k_page_stride, k_head_stride, k_row_stride;
    int64_t v_page_stride, v_head_stride, v_row_stride;
    int32_t num_pages, page_size, kv_heads, head_dim, dtype;
} svf_kv_cache;

/*
 * The sequences of one call.
 *   q_offsets   int32 [num_seqs + 1]: new tokens [q_offsets[i], q_offsets[i+1])
 *               belong to sequence i (nondecreasing, from 0 to num_tokens)
 *   kv_len      int32 [num_seqs]: slots of each sequence, its new tokens
 *               included: new token t of n has slot kv_len - n + t (none where
 *               that is negative)
 *   page_table  int32 [num_seqs][table_stride], table_width entries of each
 *               used, those behind kv_len never read
 *   max_q       no sequence has more new tokens than this (svf_kv_attend:
 *               the rows of a sequence that has more are NaN)
 * table_width * page_size < 2^31 - 2^16.
 */
typedef struct svf_kv_batch {
    const int32_t *q_offsets;
    const int32_t *kv_len;
    const int32_t *page_table;
    int64_t table_stride;
    int32_t num_seqs, num_tokens, table_width, max_q;
} svf_kv_batch;

/*
 * Rotary positions on new queries and keys, and the new tokens' slots.
 *   q, k, v     [num_tokens][heads or kv_heads][head_dim]; strides of token and
 *               head in elements, head_dim contiguous; any alignment
 *   q_out       the same shape as q; q itself with the same strides, or apart from it
 *   positions   int32 [num_tokens]
 *   rope        float [rope_rows][rot]: rot/2 cosines, then rot/2 sines, of
 *               each position; whatever stretches positions for long
 *               contexts (other frequencies, a factor) is in the table
 *   rot         even, 0 .. head_dim: the dimensions from 0 that are turned; the
 *               others are copied
 * For a pair (a, b) of token t, with c and s from row positions[t]:
 *   a' = a c - b s,   b' = b c + a s
 * in 32 bits, rounded once.  k rotated and v as it is go to the token's slot;
 * where the cache keeps them its weight is set to 0 and its position to
 * positions[t].  A token whose position is outside the table gets NaN for
 * every rotated element.
 */
typedef struct svf_kv_append_args {
    const void *q;
    const void *k;
    const void *v;
    void *q_out;
    const int32_t *positions;
    const float *rope;
    int64_t q_token_stride, q_head_stride;
    int64_t k_token_stride, k_head_stride;
    int64_t v_token_stride, v_head_stride;
    int64_t out_token_stride, out_head_stride;
    int32_t heads, rot, layout, rope_rows;
} svf_kv_append_args;

int svf_kv_append(const svf_kv_cache *cache, const svf_kv_batch *batch,
                  const svf_kv_append_args *args, void *hip_stream);

/*
 * The same for positions with several axes (time, height and width of an image's or a video's tokens): pair p
 * of a head turns by row positions[t][of_pair[p]] of the table, and its cosine and sine are columns p and
 * rot/2 + p of that row.  A position outside the table makes NaN of the pairs that turn by it and of no others.
 *   positions   (of svf_kv_append_args) element (t, axis) at positions[t * token_stride + axis * axis_stride]
 *   of_pair     the axis of each of the rot/2 pairs, below ``axes``
 *   kept        int32 [num_tokens]: what the cache's position is set to, for eviction goes by the order of
 *               the text; NULL: axis 0's position
 */
enum { SVF_KV_MOST_AXES = 4 };

typedef struct svf_kv_axes {
    const int32_t *kept;
    int64_t token_stride, axis_stride;
    int32_t axes;
    uint8_t of_pair[128];
} svf_kv_axes;

int svf_kv_append_axes(const svf_kv_cache *cache, const svf_kv_batch *batch,
                       const svf_kv_append_args *args, const svf_kv_axes *axes, void *hip_stream);

/*
 * Attention of the new tokens over their sequences' slots.  Query head h
 * reads key head h / (heads / kv_heads).  Row (t, h) of sequence i, whose own
 * slot is r = kv_len - n + t, sees slot j if
 *   0 <= j < kv_len,  j <= r when causal,  j > r - window when window > 0
 * (slots, not positions: a window means what it says only in a cache that was
 * never shrunk).  Over the slots it sees
 *   out = sum_j softmax_j(scale q.k_j) v_j,   lse = ln sum_j exp(scale q.k_j),
 * and a row that sees none, or only scores of -inf, has out = 0 and
 * lse = -inf.  What lies in slots that a row does not see, NaN and infinities
 * among it, has no effect on that row; an infinite or NaN element of a value that it
 * sees decides its output however small the slot's softmax is.
 *   scale       finite, below 2^127
 *   add_weight  1: weight[j] += the sum of slot j's softmax over the tokens and
 *               the query heads of its key head (in an order that is the same
 *               every time).  Each page at most once in the batch then.
 *   q           [num_tokens][heads][head_dim], as in svf_kv_append
 *   out         the same, contiguous heads not required, apart from q; 16-byte
 *               aligned, strides multiples of 8
 *   lse         float [num_tokens][heads]
 *   workspace   svf_kv_attend_workspace bytes, 256-byte aligned, nothing kept in it
 */
typedef struct svf_kv_attend_args {
    const void *q;
    void *out;
    float *lse;
    void *workspace;
    int64_t workspace_bytes;
    int64_t q_token_stride, q_head_stride;
    int64_t out_token_stride, out_head_stride;
    float scale;
    int32_t heads, causal, window, add_weight;
} svf_kv_attend_args;

int svf_kv_attend(const svf_kv_cache *cache, const svf_kv_batch *batch,
                  const svf_kv_attend_args *args, void *hip_stream);

/*
 * The same with first tokens that stay visible: row r also sees the slots j < first that its window
 * hides (0 <= j < kv_len, j <= r when causal).  Slots that no row sees are not read, and the pages that hold nothing
 * else may have been given back (no page there, a page number outside the pool).  Without a window, or where first is 0, it is
 * svf_kv_attend.
 *   workspace   (of svf_kv_attend_args) svf_kv_attend_first_workspace bytes
 */
int svf_kv_attend_first(const svf_kv_cache *cache, const svf_kv_batch *batch,
                        const svf_kv_attend_args *args, int32_t first, void *hip_stream);

int64_t svf_kv_attend_first_workspace(const svf_kv_cache *cache, const svf_kv_batch *batch,
                                      const svf_kv_attend_args *args, int32_t first);

/* Bytes of workspace that svf_kv_attend needs for these sizes (only sizes
 * and add_weight are read); negative: the code of an error. */
int64_t svf_kv_attend_workspace(const svf_kv_cache *cache, const svf_kv_batch *batch,
                                const svf_kv_attend_args *args);

/* Text of the calling thread's last error in one of these calls. */
const char *svf_kv_last_error(void);

/*
 * Shrink every sequence of more than ``budget`` slots to ``budget``, each key
 * head for itself.  Kept are the slots of the ``first`` lowest positions of the
 * text (position < first), of the ``recent`` newest tokens (position >=
 * next_position[i] - recent), and of the others those of largest weight; ties
 * go to the lower slot; NaN counts as less than any weight, a slot without a
 * page as NaN.  (first + recent
 * <= budget.  Should positions repeat, so that more are protected, the lower
 * slots of those stay.)  The kept slots at or above the budget, in rising
 * order, move into the slots below it that are not kept, in rising order: key,
 * value, weight and position (where the place has no page, they are lost).  Slots
 * at or above the budget keep what they held.  Each page at most once in the batch.
 *   next_position  int32 [num_seqs]: the position that the next token will have
 *   new_len        int32 [num_seqs]: min(kv_len, budget); not kv_len itself
 *   workspace      svf_kv_evict_workspace bytes, 256-byte aligned
 * Of the batch, q_offsets, num_tokens and max_q are not read.
 */
typedef struct svf_kv_evict_args {
    const int32_t *next_position;
    int32_t *new_len;
    void *workspace;
    int64_t workspace_bytes;
    int32_t budget, recent, first;
} svf_kv_evict_args;

int svf_kv_evict(const svf_kv_cache *cache, const svf_kv_batch *batch,
                 const svf_kv_evict_args *args, void *hip_stream);

int64_t svf_kv_evict_workspace(const svf_kv_cache *cache, const svf_kv_batch *batch,
                               const svf_kv_evict_args *args);

#ifdef __cplusplus
}
#endif

#endif /* SVFKV_H */
