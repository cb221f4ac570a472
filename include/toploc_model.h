/*
 * toploc_model.h -- C ABI of the model-side operators for NVIDIA B200 (sm_100a).
 *
 * A proof (toploc.h) commits to the last hidden states of a model.  These are
 * the operators of the passes that produce those states: a provider plans
 * pages, writes keys and values to a paged cache and lets a chunk of new
 * tokens attend over it (Section 5.5: a proof per 32 new tokens); a validator
 * recomputes whole prompts in one packed pass (Section 5.1); both close every
 * layer with a residual addition and an RMS norm.
 *
 * The rules of toploc.h hold here: plain C, the caller owns every buffer,
 * nothing is allocated, work is only enqueued on the given stream, no kernel
 * traps, host-detected problems come back as TOPLOC_ERR_* and nothing is
 * enqueued then, per-sequence conditions come back as status bytes.  None of
 * these calls reads device memory from the host, so all can be captured into
 * a CUDA graph.
 */
#ifndef TOPLOC_MODEL_H_
#define TOPLOC_MODEL_H_

#include "toploc.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Per-sequence status bytes. */
#define TOPLOC_SEQ_OK 0
#define TOPLOC_SEQ_BAD_LENGTH 1 /* a negative length, or one beyond what the call was told it can be */
#define TOPLOC_SEQ_NO_PAGES 2   /* the free list ran out before this sequence's pages */
#define TOPLOC_SEQ_TABLE_FULL 3 /* more pages than a row of the block table holds */
#define TOPLOC_SEQ_BATCH_FULL 4 /* the sequence's tokens end beyond the token buffers */
#define TOPLOC_SEQ_BAD_PAGE 5   /* a block table entry outside the cache */
#define TOPLOC_SEQ_WAIT_EXPIRED 6 /* a wait inside the kernel ran out of its limit; rows that were not finished are NaN */

const char* toploc_sequence_status_string(int sequence_status);

/* ---- pages ------------------------------------------------------------ */

/*
 * Plans one step of a paged cache on the GPU.  Sequence i has c_i tokens in
 * the cache and brings t_i new ones; its tokens are rows
 * offset_i .. offset_i + t_i - 1 of the step's packed tensors,
 * offset_i = t_0 + .. + t_{i-1}.  It holds ceil(c_i / page_size) pages and
 * needs ceil((c_i + t_i) / page_size): the missing ones come off the free list
 * in sequence order, entry first_free + (pages taken by earlier sequences) on.
 *
 *   d_seq_offsets [num_seqs + 1]  offset_i, and the number of tokens
 *   d_kv_lens     [num_seqs]      c_i + t_i
 *   d_block_table [num_seqs, max_pages]  entries ceil(c_i / page_size) and on
 *                                 are written; the earlier ones are read
 *   d_slots       [max_tokens]    page * page_size + position in the page of
 *                                 every new token, -1 for rows without one
 *   d_positions   [max_tokens]    c_i + row - offset_i (rotary angle), 0 for
 *                                 rows past the last token
 *   d_next_free   [1]             first_free + pages taken: the next step's
 *                                 d_first_free (two buffers used in turn)
 *   d_status      [num_seqs]      TOPLOC_SEQ_*
 *
 * A sequence whose status is not OK takes no pages, gets kv_len 0 (attention
 * over it gives zeros) and slots -1; its rows stay in the packing.  The free
 * list runs out in order: the first sequence whose pages do not fit and all
 * later ones that need any get NO_PAGES (with a negative first_free: all that need any).  A sequence whose rows would end past
 * max_tokens gets BATCH_FULL and seq_offsets stop at max_tokens.  A negative
 * t_i counts as 0.  The same inputs give the same outputs, and a repeated call
 * changes nothing.
 *
 * All arrays DEVICE; int32 4-byte, int64 8-byte aligned.  What is written must
 * not lie in what is read (d_kv_lens is not d_cached_lens: two buffers used in
 * turn; refused), nor in another output.  page_size > 0,
 * table_stride >= max_pages (elements between rows of the table),
 * num_seqs and max_tokens >= 0, num_seqs <= 2^24, max_tokens < 2^31.
 */
int toploc_plan_pages(const int32_t* d_cached_lens, const int32_t* d_new_lens, int32_t num_seqs,
                      const int32_t* d_free_pages, int32_t num_free, const int32_t* d_first_free,
                      int32_t page_size, int32_t* d_block_table, int32_t max_pages, int64_t table_stride,
                      int32_t* d_seq_offsets, int32_t* d_kv_lens, int64_t* d_slots, int32_t* d_positions,
                      int64_t max_tokens, int32_t* d_next_free, uint8_t* d_status, void* cuda_stream);

/* Keys and values: a paged cache (both tensors may have any order of page,
 * token and head: strides in elements say which), or the packed rows of a
 * prompt (page_size 0; only the token and head strides count). */
typedef struct {
  int32_t page_size;    /* tokens per page */
  int32_t num_pages;    /* pages of the cache */
  int32_t max_pages;    /* columns of the block table */
  int32_t reserved;     /* 0 */
  int64_t table_stride; /* elements between rows of the block table */
  int64_t k_page_stride, k_token_stride, k_head_stride;
  int64_t v_page_stride, v_token_stride, v_head_stride;
} toploc_kv_layout;

/*
 * Writes the keys and values of new tokens to their slots of the cache.
 * d_k, d_v       DEVICE [num_tokens, kv_heads, head_dim], token and head
 *                strides in elements, the last dimension contiguous
 * d_slots        DEVICE [num_tokens]: page * page_size + position in the page;
 *                a negative one, or one past the cache, is skipped (distinct
 *                tokens have distinct slots)
 * d_k_cache, d_v_cache  DEVICE, as kv describes (table fields unused)
 * dtype          TOPLOC_DTYPE_* of all four
 * kv_heads * head_dim < 2^31.  Pointers aligned to the element; rows of whole
 * 16-byte vectors at 16-byte aligned places move as vectors, others element by
 * element.
 */
int toploc_cache_write(const void* d_k, const void* d_v, int64_t k_token_stride, int64_t k_head_stride,
                       int64_t v_token_stride, int64_t v_head_stride, const int64_t* d_slots, int64_t num_tokens,
                       int32_t dtype, int32_t kv_heads, int32_t head_dim, void* d_k_cache, void* d_v_cache,
                       const toploc_kv_layout* kv, void* cuda_stream);

/* ---- attention -------------------------------------------------------- */

/* The batch of an attention call: packed new tokens, grouped heads (query
 * heads h * q_heads / kv_heads and on, q_heads / kv_heads of them, share key
 * head h). */
typedef struct {
  int32_t dtype;          /* TOPLOC_DTYPE_*: q, k, v and out */
  int32_t head_dim;       /* a multiple of 8, at most 256 */
  int32_t q_heads;        /* a multiple of kv_heads, at most 128 per key head */
  int32_t kv_heads;
  int32_t num_seqs;       /* >= 0 */
  int32_t max_new_tokens; /* no sequence brings more (a bound; it sizes the launch) */
  int64_t total_tokens;   /* rows of q, out and lse */
  float scale;            /* > 0, finite; 1 / sqrt(head_dim) as a rule */
  int32_t wait_tries;     /* 0; else the tries (4 us each) after which a wait inside the kernel gives up, by default
                             8 s in all (see TOPLOC_SEQ_WAIT_EXPIRED) */
  int64_t q_token_stride, q_head_stride;     /* elements; the last dimension is contiguous */
  int64_t out_token_stride, out_head_stride;
} toploc_attention_layout;

/*
 * Attention of new tokens over a paged cache that already holds them
 * (toploc_cache_write), causal: row r of sequence i (r = 0 .. t_i - 1,
 * t_i = seq_offsets[i + 1] - seq_offsets[i]) sees keys
 * j <= kv_lens[i] - t_i + r,
 *   out = sum_j p_j v_j / sum_j p_j,   p_j = exp(scale * q . k_j - max),
 *   lse = log sum_j exp(scale * q . k_j).
 * t_i = 1 is a decode step, t_i = 32 the proof interval, t_i = kv_lens[i] a
 * whole prompt.  A row that sees no key gets out 0 and lse -inf.  What lies in
 * the cache past kv_lens[i], NaN included, has no influence on any result; nor
 * has a key that the mask hides from a row on that row.
 *
 * Scores, maxima, sums and outputs are accumulated in fp32 (the outputs' sums
 * with weights up to 2^8, so values up to about 2^120 / keys are safe); bf16 inputs take
 * the weights p_j rounded to bf16 into the second product (8 bits, as v_j has;
 * the sum in the denominator uses them unrounded).
 *
 * d_q            DEVICE [total_tokens, q_heads, head_dim]
 * d_k_cache, d_v_cache, kv  DEVICE / HOST, the cache
 * d_block_table  DEVICE [num_seqs, max_pages] int32
 * d_seq_offsets  DEVICE [num_seqs + 1] int32, ascending from 0
 * d_kv_lens      DEVICE [num_seqs] int32
 * d_out          DEVICE out [total_tokens, q_heads, head_dim]; rows of no
 *                sequence are left as they are
 * d_lse_opt      DEVICE out, NULL or [total_tokens, q_heads] fp32
 * d_status_opt   DEVICE in/out, NULL or [num_seqs] bytes: set to TOPLOC_SEQ_*
 *                where a sequence is not as promised (BAD_LENGTH: t_i over
 *                max_new_tokens or kv_lens[i] over the table, counted as the
 *                largest possible; BAD_PAGE; WAIT_EXPIRED), else left as it is;
 *                nothing outside the cache is read in any case.  With NULL the
 *                first two have no sign, and WAIT_EXPIRED only the NaN rows
 * d_workspace    DEVICE toploc_attention_workspace_bytes, 32-byte aligned:
 *                partial results of rows whose keys are split over blocks
 *                (always joined in the same order); contents are undefined
 *                afterwards, and calls that can overlap need one each
 * Asynchronous, deterministic.
 *
 * Variants, by a rule on types and layout: bf16 with head_dim 64 or 128, rows
 * and strides of 16-byte multiples, and a page_size that is a multiple of 8 and
 * divides 128 (or a multiple of 128) takes the tensor cores, all else (fp32
 * among it) a kernel on the fp32 units.  On the tensor cores, calls whose
 * max_new_tokens * q_heads / kv_heads is at most 8 (single tokens, as a rule) take
 * a kernel of their own that holds keys instead of rows along a product.
 */
size_t toploc_attention_workspace_bytes(const toploc_attention_layout* lay, const toploc_kv_layout* kv);
int toploc_attention_paged(const void* d_q, const void* d_k_cache, const void* d_v_cache,
                           const toploc_attention_layout* lay, const toploc_kv_layout* kv,
                           const int32_t* d_block_table, const int32_t* d_seq_offsets, const int32_t* d_kv_lens,
                           void* d_out, float* d_lse_opt, uint8_t* d_status_opt, void* d_workspace,
                           size_t workspace_bytes, void* cuda_stream);

/*
 * Causal attention over whole prompts of different lengths, packed: sequence
 * i is rows seq_offsets[i] .. seq_offsets[i + 1] - 1 of q, k and v, and a row
 * sees its own sequence's rows up to itself.  Everything else as above, with
 * d_k, d_v DEVICE [total_tokens, kv_heads, head_dim] (views of one tensor are
 * fine: strides), and kv with page_size 0.
 */
int toploc_attention_prompt(const void* d_q, const void* d_k, const void* d_v, const toploc_attention_layout* lay,
                            const toploc_kv_layout* kv, const int32_t* d_seq_offsets, void* d_out, float* d_lse_opt,
                            uint8_t* d_status_opt, void* d_workspace, size_t workspace_bytes, void* cuda_stream);

/* ---- norm ------------------------------------------------------------- */

#define TOPLOC_NORM_OUT_SAME 0 /* y has the input's type */
#define TOPLOC_NORM_OUT_E4M3 1 /* y is 8-bit e4m3 with fp32 scales */

typedef struct {
  int32_t dtype;    /* TOPLOC_DTYPE_* of x, residual, weight and residual_out */
  int32_t out_kind; /* TOPLOC_NORM_OUT_* */
  int32_t group;    /* e4m3: channels per scale (a last group may be shorter); 0 = one scale per row */
  int32_t hidden;   /* > 0, at most 49152 */
  int64_t rows;     /* >= 0 */
  int64_t x_stride, residual_stride, residual_out_stride, y_stride; /* elements between rows */
} toploc_norm_layout;

/*
 * The seam between two sub-layers of a decoder: the residual stream takes a
 * sub-layer's output, and its RMS norm feeds the next product,
 *   h = x + residual,  residual_out = h rounded to dtype,
 *   y = h * rsqrt(mean(h^2) + eps) * weight
 * with fp32 arithmetic on the unrounded h.  With TOPLOC_NORM_OUT_E4M3 each group
 * of channels is scaled to the type's range,
 *   scale = max(max |y| / 448, 2^-126),  stored = y / scale rounded to nearest even
 * (a zero group stores zeros), scales [rows, ceil(hidden / group)] fp32.  Both
 * quotients are products with a reciprocal in fp32, off by a rounding or two, as
 * y is: a value next to the middle of two e4m3 numbers may go to the other one.
 *
 * d_residual_opt     NULL: no addition, h = x
 * d_residual_out_opt NULL: not written; may be d_residual itself
 * d_scales_opt       required with E4M3, ignored else
 * Pointers aligned to their elements; rows at 16-byte aligned places with
 * hidden a multiple of 16 bytes (of 8 elements) move as vectors.  Asynchronous.
 */
int toploc_rmsnorm_residual(const void* d_x, const void* d_residual_opt, const void* d_weight, float eps,
                            const toploc_norm_layout* lay, void* d_residual_out_opt, void* d_y, float* d_scales_opt,
                            void* cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* TOPLOC_MODEL_H_ */
