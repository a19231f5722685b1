/*
 * hps_seq.h - operators of sequence models behind the embedding cache: a model that reads a user's
 * history takes the rows of the history's items as its tokens, keeps the keys and values of those
 * tokens in pages, and scores candidates against them.
 *
 *   hps_seq_extend      pages for the tokens that each request adds, and where every token goes
 *   hps_seq_release     the pages of finished requests go back to the free list
 *   hps_seq_rope_table  cosines and sines of rotary positions, plain or scaled for long contexts
 *   hps_seq_rope        queries and keys turned by their positions, and the gradient of that
 *   hps_seq_append      the same, with keys and values written to their pages
 *   hps_seq_attention   attention of every request's new tokens over the history that its group
 *                       shares (read once for all of them) and over the request's own tokens
 *
 * Pages: keys and values of tokens live in `n_blocks` blocks of `block_size` tokens (a power of two up to
 * 1024), one array each; a request's table lists its blocks in order, so token p of a request is
 * place p % block_size of block table[p / block_size], and its slot is block * block_size + place.
 * All layers of a model share one table; each layer has its own two arrays.
 *
 * Conventions for every call
 *   - Arrays are device memory on the current GPU; structures are read on the host during the call.
 *     Integer arrays are int32, 4-byte aligned.  Strides are in elements; the values of one head are
 *     adjacent.  Outputs must not overlap inputs unless a call says so.
 *   - Every call only enqueues kernels on `stream` (a hipStream_t passed as void*, NULL = the null
 *     stream) and may be captured into a HIP graph: lengths are read on the device, at each replay.
 *     hps_seq_attention_create, _destroy and _flags are the exceptions.
 *   - Status codes are those of hps_cache.h; nothing is thrown.  The message of the last failing call
 *     of this header on the calling thread is returned by hps_seq_last_error().
 *   - Lengths, block numbers, slots and positions are checked where they are used: bad ones never
 *     lead out of an array.  What they lead to instead stands at each call.
 */
#ifndef HPS_SEQ_H
#define HPS_SEQ_H

#include <stddef.h>
#include <stdint.h>

#include "hps_cache.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Types of queries, keys and values. */
#define HPS_SEQ_F32  0
#define HPS_SEQ_F16  1
#define HPS_SEQ_BF16 2

#define HPS_SEQ_MAX_BLOCK 1024u         /* most tokens of a block */

/*
 * Pages for new tokens.  Request r has past_lens[r] tokens and adds new_lens[r] (negative ones count as
 * 0).  Its first ceil(past / block_size) table entries are kept; every further block that its new
 * tokens need is taken from the end of the free list: the k-th new block of the call, counted by
 * request and then by place in the table, is free_blocks[*n_free - 1 - k].
 *   token_offsets  [n_requests + 1]  exclusive sums of new_lens: request r's new tokens are
 *                                    token_offsets[r] .. token_offsets[r + 1] of the call's tokens
 *   total_lens     [n_requests]      past + new: the next call's past_lens (not the array of this call's)
 *   slots          [max_tokens]      slot of each new token; -1 behind the last token
 *   positions      [max_tokens]      its position start[r] + place in the request; -1 behind the last
 *   info           [4]               blocks left in the free list, new tokens of the call, blocks that the
 *                                    free list lacked, tokens that did not fit their request's table
 * The new n_free is info[0], so a call may be given the previous call's info as n_free (another array
 * than its own info).  Lacking blocks: the table entry is -1 and so are the slots of its tokens.  A
 * request holds at most table_width * block_size tokens: total_lens stops there and slots are -1
 * beyond.  (hps_seq_attention takes a request's new tokens for the last of its length, so where tokens did not fit -
 * info[3] != 0, total_lens[r] < past + new - all rows of that request's new tokens are undefined in it, those of
 * tokens that did fit among them.  Other requests are as ever.)  Tokens beyond max_tokens are counted, and not
 * written.  Sums stop at 2^31 - 1.
 * n_requests == 0 is allowed.
 */
typedef struct {
    const int32_t *past_lens, *new_lens;
    const int32_t *start;               /* position of a request's first token, e.g. the length of a shared history; NULL = 0 */
    const int32_t *free_blocks;         /* [n_blocks], the first *n_free are free */
    const int32_t *n_free;
    int32_t *block_table;               /* [n_requests][table_width] */
    int32_t *token_offsets, *total_lens, *slots, *positions, *info;
    uint32_t n_requests, block_size, n_blocks, table_width, max_tokens;
} hps_seq_extend_args_t;

hps_status_t hps_seq_extend(const hps_seq_extend_args_t *args, void *stream);

/*
 * Blocks of finished requests.  For every r with finished[r] != 0 the first ceil(lens[r] / block_size)
 * entries of its table go to the end of the free list, in order, and become -1, and lens[r] becomes
 * 0.  Entries that are no block numbers are left out.  info[0] receives the new length of the free
 * list (n_free may be &info[0] here: one work-group does all of it), info[1] the blocks given back,
 * info[2] those for which the list, n_blocks long, had no room: blocks given back twice.
 */
hps_status_t hps_seq_release(int32_t *lens, const int32_t *finished, uint32_t n_requests, uint32_t block_size,
                             int32_t *block_table, uint32_t table_width, int32_t *free_blocks, uint32_t n_blocks,
                             const int32_t *n_free, int32_t *info, void *stream);

/*
 * Cosines and sines of the angles pos * w_i, i < rot_dim / 2, w_i = base^(-2i / rot_dim):
 * table [max_pos][rot_dim / 2][2] fp32, cosine first; angles are computed in 64 bits.
 *   scale HPS_SEQ_SCALE_NONE    w_i as it is
 *         HPS_SEQ_SCALE_LINEAR  w_i / factor
 *         HPS_SEQ_SCALE_PARTS   with n_i = original * w_i / (2 pi), the turns of pair i within the original
 *                               context, and g_i = clamp((n_i - low) / (high - low), 0, 1):
 *                               w_i * (g_i + (1 - g_i) / factor)
 * magnitude multiplies cosines and sines (1 = none).
 */
#define HPS_SEQ_SCALE_NONE   0
#define HPS_SEQ_SCALE_LINEAR 1
#define HPS_SEQ_SCALE_PARTS  2
hps_status_t hps_seq_rope_table(float *table, uint32_t max_pos, uint32_t rot_dim, double base, int scale, double factor,
                                double original, double low, double high, double magnitude, void *stream);

/* Heads of a run of tokens: element (t, h, d) is data[t * token_stride + h * head_stride + d]. */
typedef struct {
    void   *data;
    int64_t token_stride, head_stride;
} hps_seq_heads_t;

/*
 * Rotary positions.  Of each head the first rot_dim values (even, <= head_dim <= 512) are turned, pair by
 * pair: (a, b) becomes (a cos - b sin, a sin + b cos) with the table's row of the token's position;
 * pair i is (i, i + rot_dim / 2), or with interleaved != 0 (2i, 2i + 1).  The others are copied.
 * inverse != 0 turns the other way, which is the gradient with respect to the input.  Arithmetic is in
 * 32 bits, rounded once.  A tensor of 0 heads may have NULL data; an output may be its input, exactly.
 * A token with a negative position is passed over; at a position of max_pos or more the turned values
 * come out as NaN.
 */
typedef struct {
    hps_seq_heads_t q, k, q_out, k_out;
    const int32_t *positions;           /* [n_tokens] */
    const float   *table;               /* as hps_seq_rope_table writes it */
    uint32_t n_tokens, q_heads, k_heads, head_dim, rot_dim, max_pos;
    int32_t  dtype, interleaved, inverse;
} hps_seq_rope_args_t;

hps_status_t hps_seq_rope(const hps_seq_rope_args_t *args, void *stream);

/* Keys and values in pages: element (block, place, h, d) is data[block * block_stride + place * token_stride + h * head_stride + d]. */
typedef struct {
    void    *k, *v;
    int64_t  block_stride, token_stride, head_stride;   /* of both */
    uint32_t n_blocks, block_size;
} hps_seq_pages_t;

/*
 * hps_seq_rope for queries (to q_out) and keys, with the turned keys and the values (as they are) written
 * to their slots of the pages.  A token whose slot is outside 0 .. n_blocks * block_size - 1 has its
 * query turned and nothing stored.  Slots of one call must be different.  table NULL: nothing is turned
 * and positions is not read.  q_heads 0: keys and values alone.
 */
typedef struct {
    hps_seq_heads_t q, q_out, k, v;
    hps_seq_pages_t pages;
    const int32_t *slots, *positions;   /* [n_tokens] */
    const float   *table;
    uint32_t n_tokens, q_heads, kv_heads, head_dim, rot_dim, max_pos;
    int32_t  dtype, interleaved;
} hps_seq_append_args_t;

hps_status_t hps_seq_append(const hps_seq_append_args_t *args, void *stream);

/* ---- attention behind shared histories ------------------------------------------------- */

typedef struct hps_seq_attention_session hps_seq_attention_t;

/*
 * Scratch memory of hps_seq_attention for calls with up to max_rows = tokens * q_heads rows of up to
 * max_head_dim values: what parts of a long history leave behind before they are joined, about
 * (3 * max_rows + 65536) * (4 * max_head_dim + 8) bytes.  Calls on one session must not overlap (replays
 * of graphs captured from it included); different sessions are independent.
 */
hps_status_t hps_seq_attention_create(size_t max_rows, uint32_t max_head_dim, hps_seq_attention_t **out);

/* Waits for the device, then frees the session.  NULL is accepted. */
hps_status_t hps_seq_attention_destroy(hps_seq_attention_t *s);

/*
 * Attention with softmax over scale * (query . key).  The new tokens of request r are
 * token_offsets[r] .. token_offsets[r + 1]; the i-th of n attends to
 *   - the prefix_lens[g] tokens listed in row g of prefix_table, if group_offsets[g] <= r <
 *     group_offsets[g + 1] (groups are runs of requests; a request of no group has no history), and
 *   - the request's own tokens 0 .. lens[r] - n + i, listed in row r of block_table (its new tokens are the
 *     last n of them: append before attending; a length that hps_seq_extend had to cut does not fit this).
 * Offsets may go beyond n_tokens, as those of hps_seq_extend do beyond its max_tokens: the tokens there have no
 * query and no row, and count among the n.
 * Query head h reads key/value head h / (q_heads / kv_heads).  out receives the result in the queries'
 * type, lse [n_tokens][q_heads] fp32 (or NULL) the logarithm of the sum of exponentials.  A row that
 * attends to nothing, or whose scores are all minus infinity, gets 0, and minus infinity in lse.  Rows of
 * tokens in front of the first request's or behind the last one's are not written.  What lies in masked
 * places (behind a length, behind a query's own place) has no part in the result, whatever its value.  Sums,
 * maxima and weights are in 32 bits; weights are rounded to the values' type for the product with the
 * values (in f16 those above 2^-22 of a row's largest keep 11 bits, smaller ones fewer, and those below 2^-33
 * none), whose sums are formed before they are divided by the weights' (values up to 2^80 in size are
 * safe, whatever the scores).
 *
 * max_new, max_group, max_len, max_prefix bound the new tokens of a request, the new tokens of a
 * group, lens and prefix_lens: the host sizes the launch by them (the device reads the lengths
 * themselves), so bounds near the lengths pay: work-groups without rows come and go, but there are n_requests times
 * as many as max_new would fill (512 requests of a token, 32 / 8 heads: 18 us with max_new 1, 204 with 512; 8,192 requests
 * 163 us with 1, 18 ms with 8,192).  A longer one raises HPS_SEQ_FLAG_LENGTH and the rows concerned are undefined, and so does a
 * length that its table does not hold; a block number outside 0 .. n_blocks - 1 within a length raises
 * HPS_SEQ_FLAG_BLOCK and stands for a block of zeros.
 * Blocks of 16 tokens and more are read two to five times as fast as smaller ones.
 * dtype HPS_SEQ_F16 or HPS_SEQ_BF16; head_dim a multiple of 8 up to 256; q_heads a multiple of
 * kv_heads; all data and strides multiples of 16 bytes, the pages' not negative; scale finite and > 0.
 */
typedef struct {
    hps_seq_heads_t q, out;
    hps_seq_pages_t pages;
    const int32_t *prefix_table;        /* [n_groups][prefix_width] */
    const int32_t *prefix_lens;         /* [n_groups] */
    const int32_t *group_offsets;       /* [n_groups + 1] */
    const int32_t *block_table;         /* [n_requests][table_width] */
    const int32_t *lens;                /* [n_requests] */
    const int32_t *token_offsets;       /* [n_requests + 1] */
    float   *lse;
    uint32_t n_tokens, n_requests, n_groups, table_width, prefix_width;
    uint32_t max_new, max_group, max_len, max_prefix;
    uint32_t q_heads, kv_heads, head_dim;
    int32_t  dtype;
    float    scale;
} hps_seq_attention_args_t;

hps_status_t hps_seq_attention(hps_seq_attention_t *s, const hps_seq_attention_args_t *args, void *stream);

/* Flag word of a session, raised by kernels.  *flags [host] receives the bits; clear != 0 resets them.
 * Synchronous on the host; call it after synchronising the streams whose work is to be covered. */
#define HPS_SEQ_FLAG_LENGTH 1u
#define HPS_SEQ_FLAG_BLOCK  2u
hps_status_t hps_seq_attention_flags(hps_seq_attention_t *s, uint32_t *flags, int clear);

const char *hps_seq_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* HPS_SEQ_H */
