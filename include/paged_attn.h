/* paged_attn.h -- C ABI of the sampling phase on gfx950 / MI355X: rotary positions with several axes, a paged
 * cache of keys and values, and the attention of each sequence's newest tokens over its pages.
 *
 * The rollouts that the GRPO step of prefix_attn.h consumes are generated token by token (paper Sec. 4.2: G responses are
 * sampled for one question; Sec. 5.1: all of them share the video's cached embeddings).  A serving loop does per layer
 *
 *     paged_kv_append_rope   rotates the new tokens' queries and keys and stores keys and values in their pages,
 *     paged_attn_forward     attends the new tokens to everything their sequences hold,
 *
 * for one token of every rollout or for chunks of a prompt; rope_axes_forward / _backward are the same rotation for
 * the prefill and the training step, in front of prefix_attn_forward and behind prefix_attn_backward.
 *
 * Conventions are those of prefix_attn.h: status codes, no allocation and no synchronisation in the calls that enqueue
 * work, device pointers on the plan's device, which must be the current one (else PA_ERR_HIP).  What varies from step to
 * step (lengths, page tables, positions) is read on the device, so a captured call can be replayed on the next step's.
 */
#ifndef PAGED_ATTN_H_
#define PAGED_ATTN_H_

#include "prefix_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- rotary positions with several axes ---------------------------------------------------------------------------
 *
 * A head's first rotary_dim channels form rotary_dim / 2 pairs.  Pair i of token t is turned by the angle
 *     a = positions[pair_axis[i]][t] * inv_freq[i]:      y0 = x0 cos a - x1 sin a,   y1 = x1 cos a + x0 sin a;
 * the channels from rotary_dim on pass through.  A video token has a time, a height and a width; one axis gives
 * the ordinary rotary embedding.  The rotation is orthogonal, so its gradient is the rotation by -a. */
#define PA_ROPE_MAX_AXES 4
#define PA_ROPE_MAX_PAIRS 128

typedef enum {
  PA_ROPE_HALVES = 0, /* pair i is channels (i, i + rotary_dim / 2) */
  PA_ROPE_PAIRS = 1   /* pair i is channels (2 i, 2 i + 1) */
} pa_rope_layout_t;

typedef struct {
  int32_t head_dim;   /* D, 2 <= D <= 256 */
  int32_t rotary_dim; /* even, 2 <= rotary_dim <= D */
  int32_t layout;     /* pa_rope_layout_t */
  int32_t num_axes;   /* 1 <= num_axes <= PA_ROPE_MAX_AXES */
  uint8_t pair_axis[PA_ROPE_MAX_PAIRS]; /* the axis of pair i < rotary_dim / 2, < num_axes */
} rope_axes_desc_t;

/* Rotate the heads of num_tokens tokens, on the current device.
 *   q, q_out  [num_tokens, num_q_heads, D]   of dtype; heads contiguous, tokens q_stride (q_out_stride) elements apart:
 *             slices of a fused projection's output need no copy.  q_out may be q itself (in place), and must not
 *             overlap it otherwise.  Any alignment of whole elements.
 *   k, k_out  [num_tokens, num_k_heads, D]   likewise, with num_k_heads = 0 and NULL when there are none
 *   positions [num_axes, num_tokens] int32, any sign;  inv_freq [rotary_dim / 2] fp32 (radians per position)
 * num_tokens = 0 is valid and enqueues nothing.  The angle is exact until whole turns are off: sine
 * and cosine err by at most 4 units of 2^-24 at any position (angles up to 2^51 radians). */
int rope_axes_forward(const rope_axes_desc_t* desc, int32_t dtype, const void* q, int64_t q_stride, const void* k,
                      int64_t k_stride, int64_t num_tokens, int32_t num_q_heads, int32_t num_k_heads,
                      const int32_t* positions, const float* inv_freq, void* q_out, int64_t q_out_stride, void* k_out,
                      int64_t k_out_stride, void* hip_stream);

/* The gradient: q and k hold dL/d(q_out) and dL/d(k_out), and q_out and k_out receive dL/dq and dL/dk. */
int rope_axes_backward(const rope_axes_desc_t* desc, int32_t dtype, const void* q, int64_t q_stride, const void* k,
                       int64_t k_stride, int64_t num_tokens, int32_t num_q_heads, int32_t num_k_heads,
                       const int32_t* positions, const float* inv_freq, void* q_out, int64_t q_out_stride, void* k_out,
                       int64_t k_out_stride, void* hip_stream);

/* ---- paged cache ---------------------------------------------------------------------------------------------------
 *
 * k_cache, v_cache [num_pages, Hkv, page_size, D]: a page holds page_size consecutive tokens of one sequence, all
 * kv heads, a head's rows contiguous.  Sequence b names its pages in row b of page_table [num_seqs, max_pages_per_seq]
 * (token j is in page page_table[b][j / page_size]); tables may share pages.  seq_lens[b] counts ALL tokens of sequence b,
 * the new ones of this call included; its new tokens are the packed rows cu_new[b] .. cu_new[b + 1] - 1 (cu_new is
 * non-decreasing and starts at 0; a sequence without new tokens is skipped), at the positions
 * seq_lens[b] - n .. seq_lens[b] - 1.  Packed rows behind cu_new[num_seqs] are padding: nothing is computed for
 * them, and what is there stays.
 * These four arrays are int32 DEVICE memory and are checked by the kernels: no entry of them makes a call read or write
 * outside the caches and the packed rows (where cu_new falls, paged_attn_forward computes nothing). */
typedef struct paged_attn_plan paged_attn_plan_t; /* opaque, library-owned; host data only */

typedef struct {
  int32_t num_q_heads;       /* Hq >= 1 */
  int32_t num_kv_heads;      /* Hkv >= 1, Hq % Hkv == 0 */
  int32_t head_dim;          /* D in {64, 128} */
  int32_t page_size;         /* tokens per page: a power of two, 16 ... 1024 */
  int64_t num_pages;         /* pages of the cache, 1 ... 2^31 - 1 */
  int32_t max_pages_per_seq; /* columns of the page table; times page_size at most 2^30 tokens */
  int32_t max_seqs;          /* most sequences of a call, 1 ... 65,536 */
  int64_t max_tokens;        /* most packed rows of a call, 1 ... 2^24; times Hq below 2^31 */
  float softmax_scale;       /* finite and > 0 */
  int32_t dtype;             /* pa_dtype_t of q, k, v, the caches and out */
  int32_t device;            /* HIP device ordinal; -1 = host-only plan (validation and schedule only) */
} paged_attn_desc_t;

/* Validate `desc` and report the workspace that paged_attn_forward needs. */
int paged_attn_plan(const paged_attn_desc_t* desc, paged_attn_plan_t** plan_out, size_t* workspace_bytes_out);
void paged_attn_destroy(paged_attn_plan_t* plan);

/* Store the new tokens' keys and values: k, v [num_tokens, Hkv, D] (tokens k_stride, v_stride elements apart, any
 * alignment of whole elements).  A new token whose place has no page (a negative position, one behind the table, a table
 * entry outside [0, num_pages)) is not stored.  Two sequences must not store to the same page in one call. */
int paged_kv_append(const paged_attn_plan_t* plan, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                    void* k_cache, void* v_cache, const int32_t* page_table, const int32_t* seq_lens,
                    const int32_t* cu_new, int32_t num_seqs, int64_t num_tokens, void* hip_stream);

/* The same with the keys rotated (rope->head_dim = D), and the queries q [num_tokens, Hq, D] rotated into q_out
 * (which may be q; both NULL to store keys and values only). */
int paged_kv_append_rope(const paged_attn_plan_t* plan, const rope_axes_desc_t* rope, const void* q, int64_t q_stride,
                         const void* k, int64_t k_stride, const void* v, int64_t v_stride, const int32_t* positions,
                         const float* inv_freq, void* q_out, int64_t q_out_stride, void* k_cache, void* v_cache,
                         const int32_t* page_table, const int32_t* seq_lens, const int32_t* cu_new, int32_t num_seqs,
                         int64_t num_tokens, void* hip_stream);

/* Attention of the new tokens.  Row (t, h) of a token at position p of sequence b sees the keys j = 0 .. p of its pages:
 *     s_j = softmax_scale <q, k_j>,   LSE = ln sum_j e^{s_j},   out = sum_j e^{s_j - LSE} v_j.
 *   q          [num_tokens, Hq, D], tokens q_stride elements apart (a multiple of 16 bytes), 16-byte aligned
 *   out        [num_tokens, Hq, D] contiguous, of the plan's dtype
 *   lse_out    [Hq, num_tokens] fp32, or NULL
 *   shared_len NULL, or DEVICE int32: the first *shared_len tokens of every sequence with new tokens (rounded down to whole
 *              pages) are stored in the same pages, named by all their tables, and precede all new tokens: the
 *              video of G rollouts.  Calls of at most 56 rows a sequence on average (a token has Hq / Hkv rows)
 *              then read those pages once for every 64 rows (fp32: 32) that all sequences have together, instead of once for
 *              every sequence; other calls do not use it.  The result is that of the call without it; where the tables
 *              differ, it is unspecified.
 *   workspace  at least the planned size, 16-byte aligned; calls that may overlap need workspaces of their own
 * A row without a visible key (a position below 0) gets zeros and an LSE of minus infinity.  A row that sees a key without a
 * page (an entry outside [0, num_pages), a length beyond the table) gets NaN.  Keys and values that
 * no row of a sequence sees may hold anything; a value that is not finite reaches the rows that see it, and may reach
 * earlier new tokens of the same chunk.  Reproducible bit for bit for the same lengths and the same num_seqs and num_tokens. */
int paged_attn_forward(const paged_attn_plan_t* plan, const void* q, int64_t q_stride, const void* k_cache,
                       const void* v_cache, const int32_t* page_table, const int32_t* seq_lens, const int32_t* cu_new,
                       int32_t num_seqs, int64_t num_tokens, const int32_t* shared_len, void* out, float* lse_out,
                       void* workspace, size_t workspace_bytes, void* hip_stream);

/* ---- introspection of the schedule (host only; used by tests) ----
 *
 * The pieces of work that paged_attn_forward's workgroups take for these lengths (HOST arrays, as they would be on the device;
 * shared_len < 0: not given).  pieces_out [max_pieces][8] receives, in the order of the shares,
 *     {share, sequence (-1: the shared keys, with the rows of all sequences), kv head, first stacked row of the block (m = i * (Hq / Hkv) +
 *      h % (Hq / Hkv) over the sequence's new tokens), rows, first key, end of the keys, 1 if the piece is its whole block}.
 * Returns their number (also where it exceeds max_pieces), or minus a status code. */
int64_t paged_attn_schedule(const paged_attn_plan_t* plan, const int32_t* seq_lens, const int32_t* cu_new, int32_t num_seqs,
                            int64_t num_tokens, int32_t shared_len, int32_t* pieces_out, int64_t max_pieces);
/* The workgroups of such a call, the rows of a block and the keys of a tile. */
int paged_attn_schedule_shape(const paged_attn_plan_t* plan, int32_t num_seqs, int64_t num_tokens, int32_t with_shared,
                              int32_t* groups, int32_t* block_rows, int32_t* tile_keys);

#ifdef __cplusplus
}
#endif
#endif /* PAGED_ATTN_H_ */
