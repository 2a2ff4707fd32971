/*
 * santapp_serve.h — operators around the decode step (sm_100a): what a serving loop needs next to the
 * calls of santapp.h so that queries, keys, prompts and suffixes get there and stay in order.
 *
 *   santapp_rope_append         one new token per sequence: rotary positions on q and k, k and v
 *                               appended to the suffix the decode calls read
 *   santapp_rope_prompt         the rows of prompts: rotary positions on q and k, k and v laid out as
 *                               the builders and santapp_prompt_attn take them
 *   santapp_prompt_attn         attention of prompts: ragged, causal, optionally with a bidirectional
 *                               beginning, or of their last rows alone
 *   santapp_prefix_decode_attn  one decode step of sequences that share one long prompt: the prompt
 *                               is read once for the batch
 *   santapp_suffix_fork         suffixes copied, moved and freed when answers fork, move or end
 *
 * Conventions are those of santapp.h: device / host pointers of the current device, caller-owned
 * buffers, workspaces that need no initialisation, asynchronous on `stream`, nothing kept between
 * calls, negative santapp_status on error, argument errors found on the host before any launch.
 * Of santapp_geom the calls use n_seqs, the head counts, head_dim and elem_type (the parent fields
 * only have to be valid). Every call may be captured into a CUDA graph and replayed, and
 * santapp_last_launch_count tells how many kernels it launched.
 */
#ifndef SANTAPP_SERVE_H
#define SANTAPP_SERVE_H

#include "santapp.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Rotary positions (host struct, passed by value to the kernels: it may be changed or freed when a
 * call returns). Values a, b of a pair i at position p become
 *   amplitude * (a cos(p w_i) - b sin(p w_i)),  amplitude * (b cos(p w_i) + a sin(p w_i)),
 * w_i = inv_freq[i]; angles are reduced in 64 bits, so far positions lose nothing; the rotation is
 * fp32, rounded once. Values past rot_dim are copied. */
typedef struct santapp_rope {
    int32_t rot_dim;           /* rotated values of a head: a multiple of 16, 16..128               */
    int32_t interleaved;       /* 0: pair i is (i, i + rot_dim / 2); 1: (2 i, 2 i + 1)              */
    double amplitude;          /* 1, or what a long-context scaling multiplies the rotation by
                                  (finite in fp32)                                                  */
    double inv_freq[64];       /* radians per position of pairs 0 .. rot_dim / 2 - 1 (at most 1e6)  */
} santapp_rope;

/*
 * Fills rope->inv_freq from rope->rot_dim: f_i = theta^(-2 i / rot_dim), scaled for contexts `factor`
 * times as long (factor = 1: not scaled). original_len = 0 divides every f_i by factor (positions
 * interpolated). Otherwise, with r_i = original_len f_i / (2 pi) turns over the trained length and
 * g_i = clamp((r_i - low) / (high - low), 0, 1), the frequency is f_i (g_i + (1 - g_i) / factor):
 * pairs that turn more than `high` times keep theirs, pairs below `low` are interpolated.
 * Host arithmetic only; the other fields are left as they are.
 */
int santapp_rope_frequencies(santapp_rope *rope, double theta, double factor, double low, double high,
                             double original_len);

/*
 * One new token per sequence: with t = suffix_len[b], q and k of sequence b are rotated to position
 * base_pos[b] + t, k goes to row t of the sequence's suffix, v unchanged beside it.
 *   q, k, v           device [n_seqs][n_q_heads | n_kv_heads | n_kv_heads][d], rows of consecutive
 *                     heads; token b starts q_stride (k_stride, v_stride) elements behind token b - 1
 *                     (multiples of 8: slices of one fused projection work as they are)
 *   base_pos          device int32 [n_seqs]: position of the suffix's row 0 (the prompt's length)
 *   suffix_len        device int32 [n_seqs]: rows the suffix holds before the call
 *   q_out             device [n_seqs][n_q_heads][d], out; may be q itself when q_stride = n_q_heads * d
 *   k_suffix,v_suffix device [n_seqs][n_kv_heads][suffix_cap][d], one row per head written
 *   suffix_len_out    device int32 [n_seqs] or NULL, out: suffix_len + 1; may be suffix_len itself
 *                     (of several layers that share the lengths, the last one's call advances them),
 *                     must not overlap it otherwise, nor base_pos (refused)
 * A sequence whose suffix is full (suffix_len >= suffix_cap) or whose length is negative (a padded
 * slot) is left alone: nothing of it is written, its length is passed on as it is.
 */
int santapp_rope_append(const santapp_geom *geom, const santapp_rope *rope, const void *q, int64_t q_stride,
                        const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                        const int32_t *base_pos, const int32_t *suffix_len, void *q_out, void *k_suffix,
                        void *v_suffix, int32_t suffix_cap, int32_t *suffix_len_out, santapp_stream stream);

/*
 * n_rows prompt rows (of one or several sequences, or the next rows of one): row i is rotated to
 * positions[i], its keys and values go to row dst_row[i] of each KV head's plane.
 *   q, k, v, strides  as above, n_rows tokens
 *   positions         device int32 [n_rows], or NULL: position i
 *   dst_row           device int32 [n_rows], or NULL: row i. Rows outside [0, plane_rows) are not
 *                     written; two rows with one destination leave a mixture of the two
 *   q_out             device [n_rows][n_q_heads][d], out (may be q, as above)
 *   k_prompt,v_prompt device [n_kv_heads][plane_rows][d], out: the layout of santapp_build_teams
 * geom->n_seqs is not used.
 */
int santapp_rope_prompt(const santapp_geom *geom, const santapp_rope *rope, int64_t n_rows, const void *q,
                        int64_t q_stride, const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                        const int32_t *positions, const int32_t *dst_row, void *q_out, void *k_prompt,
                        void *v_prompt, int64_t plane_rows, santapp_stream stream);

/*
 * Slot b of the batch continues what slot src[b] held: rows [0, suffix_len[src[b]]) of both buffers
 * are copied, in place, as if every slot were read before any is written (permutations, a slot read
 * by several, chains). src[b] = b costs nothing; src[b] outside [0, n_seqs) frees the slot. Rows of a
 * slot behind its new length are left as they were.
 *   src               device int32 [n_seqs]
 *   suffix_len        device int32 [n_seqs], clamped to [0, suffix_cap]
 *   k_suffix,v_suffix device [n_seqs][n_kv_heads][suffix_cap][d], in and out
 *   suffix_len_out    device int32 [n_seqs] or NULL, out: suffix_len[src[b]], 0 for a freed slot; must
 *                     not overlap suffix_len (refused)
 * At most 4096 sequences (SANTAPP_ERR_UNSUPPORTED beyond).
 */
int santapp_suffix_fork(const santapp_geom *geom, const int32_t *src, const int32_t *suffix_len, void *k_suffix,
                        void *v_suffix, int32_t suffix_cap, int32_t *suffix_len_out, santapp_stream stream);

/* How a query scores a key (host struct): s = q.k * scale; with cap > 0, cap * tanh(s / cap); with
 * slopes, less slopes[h] * |position of the query - position of the key|. Both attention calls let a
 * weight grow to 2^24 before its sums are rescaled (bf16; fp16 keeps to its own range), so values of V
 * above 2^80 may overflow on the way. scale and cap times log2 e
 * have to be finite in fp32, scale / cap a normal number of it (SANTAPP_ERR_INVALID_ARG otherwise). */
typedef struct santapp_attn_opts {
    float scale;               /* 0: 1 / sqrt(d)                                                    */
    float cap;                 /* 0: none; else > 0                                                 */
    const float *slopes;       /* device fp32 [n_q_heads] or NULL                                   */
    int32_t *status;           /* device int32 [1] or NULL: bit 2 is raised when a bounded wait inside
                                  a kernel expired (never expected; the outputs are NaN then). The
                                  calls raise it only: the caller clears it                         */
} santapp_attn_opts;

/*
 * One decode step of a batch whose sequences share one prompt (several answers to it, or questions
 * about it): query heads of sequence b attend all prefix rows and the suffix_len[b] rows of their own
 * suffix; the prompt's rows are read once for the batch, not once per sequence. Equal to
 * santapp_dense_decode_attn on records that repeat the prompt for every sequence. The last bits of a
 * sequence's rows depend on the batch it is in: its size decides how the prompt is cut, and 32 rows that
 * a warp works on share the moments at which their sums are rescaled and the form of their tanh.
 *   k_prefix,v_prefix device [n_kv_heads] planes of prefix_len rows [d], plane_rows rows apart
 *                     (plane_rows >= prefix_len): a prompt in token order, or k_packed / v_packed of
 *                     records built for one sequence (attention does not depend on row order)
 *   prefix_len        host; 0: there is no prefix (the two pointers may be NULL)
 *   prefix_token      device int32 planes like the rows' (plane_rows apart): position of each row, in
 *                     [0, prefix_len); NULL: row i is at position i. Read only with slopes (row_token of
 *                     records)
 *   q                 device [n_seqs][n_q_heads][d], at position prefix_len + suffix_len[b] - 1
 *   k_suffix, v_suffix, suffix_len_dev, suffix_cap   as in santapp_decode_attn; suffix row i is at
 *                     position prefix_len + i
 *   opts              host or NULL (scale 1 / sqrt(d), no cap, no slopes)
 *   out               device fp32 [n_seqs][n_q_heads][d]; zero for a sequence without any row
 *   workspace         device, >= santapp_prefix_decode_workspace_bytes(...)
 */
size_t santapp_prefix_decode_workspace_bytes(const santapp_geom *geom, int64_t prefix_len, int32_t suffix_cap);
int santapp_prefix_decode_attn(const santapp_geom *geom, const void *k_prefix, const void *v_prefix,
                               int64_t prefix_len, int64_t plane_rows, const int32_t *prefix_token,
                               const void *q, const void *k_suffix, const void *v_suffix,
                               const int32_t *suffix_len_dev, int32_t suffix_cap, const santapp_attn_opts *opts,
                               float *out, void *workspace, size_t workspace_bytes, santapp_stream stream);

/*
 * Attention of the prompts of a ragged batch: the last new_len[b] rows of sequence b are queries
 * (all of them: a whole prompt; fewer: its next chunk, the rows before it being cached keys). A
 * query sees the rows of its own sequence up to itself, and in any case the first prefix_len[b] of
 * them (a bidirectional beginning).
 *   prompt_len_host   host int32 [n_seqs], each >= 1
 *   new_len_host      host int32 [n_seqs], 0..prompt_len[b], or NULL: all rows
 *   prefix_len_host   host int32 [n_seqs], 0..prompt_len[b], or NULL: 0
 *   q                 device [sum new_len][n_q_heads][d], sequences one after the other (q and out may
 *                     be NULL where that is no row: nothing is launched then)
 *   k_prompt,v_prompt device [n_kv_heads][sum prompt_len][d]: the layout of santapp_build_teams
 *   out               device [sum new_len][n_q_heads][d] of the element type: it feeds a 16-bit
 *                     product. Sums and softmax statistics are fp32; the weights are rounded to the
 *                     element type for their product with V (half a step each), the result once.
 *                     The tensor core cuts its sums to fp32 instead of rounding them, which shows
 *                     where very many keys weigh alike: 0.04 % too little at 2^20 keys, 2.4 % at 2^23
 * A value that is not finite in row i of V also reaches queries of the same sequence that see no further
 * than up to 254 rows before row i (127 where all rows are queries and none is bidirectional); other
 * sequences' rows and memory behind the last row reach nothing.
 */
int santapp_prompt_attn(const santapp_geom *geom, const int32_t *prompt_len_host, const int32_t *new_len_host,
                        const int32_t *prefix_len_host, const void *q, const void *k_prompt, const void *v_prompt,
                        const santapp_attn_opts *opts, void *out, santapp_stream stream);

#ifdef __cplusplus
}
#endif
#endif /* SANTAPP_SERVE_H */
