/*
 * toploc_model.h -- C ABI of the model-side operators for NVIDIA B200 (sm_100a).
 *
 * A proof (toploc.h) commits to the last hidden states of a model.  These are
 * the operators of the passes that produce those states: a provider plans
 * pages, norms and turns queries and keys, writes keys and values to a paged
 * cache and lets a chunk of new tokens attend over it (Section 5.5: a proof per
 * 32 new tokens); a validator recomputes whole prompts in one packed pass
 * (Section 5.1); both close every layer with a residual addition and an RMS
 * norm and read log probabilities off the logits; sequences are forked, end and
 * give their pages back.
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
#define TOPLOC_SEQ_BAD_PARENT 7   /* a fork of a sequence that does not exist, or that is forked from another itself */
#define TOPLOC_SEQ_IN_USE 8       /* a fork into a sequence that holds tokens */
#define TOPLOC_SEQ_NO_ROOM 9      /* the free list has no room for all pages that came back */

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

/* ---- pages that sequences share, give back or move ---------------------- */

/*
 * Sequences that begin with the same tokens (samples of one prompt) can hold the
 * same pages.  d_shares [num_pages] says how many sequences hold a page beyond
 * the first: zeros for a pool whose pages have one holder each, as
 * toploc_plan_pages hands them out (it needs no shares).  Only whole pages are
 * shared, and new tokens go behind them, so a shared page is never written.
 *
 * Outputs of the three planners below are apart from inputs (shares and
 * lengths: two buffers used in turn), so that a repeated call gives the same,
 * but for a compaction of the table in place; refused where they overlap.  The
 * same inputs give the same outputs.  All arrays DEVICE; int32 4-byte aligned.
 * page_size > 0, num_seqs <= 2^24, num_pages <= 2^30, max_pages >= 0,
 * table_stride >= max_pages.
 */

/*
 * Forks sequences: sequence i with d_parents[i] >= 0 begins as a copy of that
 * one, length l = d_kv_lens[d_parents[i]].  It shares the parent's
 * floor(l / page_size) whole pages; where tokens are left over it gets a page of
 * its own off the free list (entry first_free + pages taken by earlier children
 * on), and the pair goes to the list of copies that toploc_copy_pages works off.
 *
 *   d_parents     [num_seqs]   -1: the sequence stays as it is
 *   d_kv_lens     [num_seqs]   tokens held; a child's must be 0
 *   d_block_table [num_seqs, max_pages]  children's rows are written, entries
 *                              0 .. ceil(l / page_size) - 1; parents' are read
 *   d_kv_lens_out [num_seqs]   l for children that were forked, else d_kv_lens
 *   d_shares_out  [num_pages]  shares with the children counted
 *   d_copy_from, d_copy_to [num_seqs]  the pages to copy, in order of children,
 *                              -1 behind the last
 *   d_num_copies  [1]          how many
 *   d_next_free   [1]          first_free + pages taken
 *   d_status      [num_seqs]   TOPLOC_SEQ_*
 *
 * A child whose status is not OK stays as it was (its row's contents do not
 * count): BAD_PARENT, IN_USE, BAD_LENGTH (the parent's is negative or beyond
 * its row), BAD_PAGE (an entry of the parent's row, or of the free list, is
 * outside the pool; a page off the list is used up all the same and its pair is
 * -1), NO_PAGES (in order, as in toploc_plan_pages).
 */
int toploc_fork_pages(const int32_t* d_parents, const int32_t* d_kv_lens, int32_t num_seqs, const int32_t* d_shares,
                      int32_t num_pages, const int32_t* d_free_pages, int32_t num_free, const int32_t* d_first_free,
                      int32_t page_size, int32_t* d_block_table, int32_t max_pages, int64_t table_stride,
                      int32_t* d_kv_lens_out, int32_t* d_shares_out, int32_t* d_copy_from, int32_t* d_copy_to,
                      int32_t* d_num_copies, int32_t* d_next_free, uint8_t* d_status, void* cuda_stream);

/*
 * Releases sequences: those with d_release[i] != 0 let go of their
 * ceil(d_kv_lens[i] / page_size) pages.  A page that nobody holds any longer
 * goes back to the free list, in front of its head: the pages, in ascending
 * order, become entries next_free .. first_free - 1.
 *
 *   d_release     [num_seqs]   bytes
 *   d_free_pages  [num_free]   in/out, entries in front of first_free (which
 *                              earlier steps have taken) are written
 *   d_kv_lens_out [num_seqs]   0 for released sequences, else d_kv_lens
 *   d_shares_out  [num_pages]  shares without the released holders
 *   d_next_free   [1]          first_free - pages that came back
 *   d_status      [num_seqs]   TOPLOC_SEQ_*: of released sequences, BAD_LENGTH (a
 *                              negative one counts as 0, one beyond the row as
 *                              the row), BAD_PAGE (an entry outside the pool,
 *                              passed over), NO_ROOM (first_free is smaller than
 *                              the pages that came back, so the pages were never
 *                              all taken off this list: the highest ones that do
 *                              not fit are left out)
 *
 * A first_free outside 0 .. num_free counts as the nearest of the two for the
 * room that there is.  A page released more often than it is held comes back
 * once.
 */
int toploc_release_pages(const uint8_t* d_release, const int32_t* d_kv_lens, int32_t num_seqs,
                         const int32_t* d_block_table, int32_t max_pages, int64_t table_stride, const int32_t* d_shares,
                         int32_t num_pages, int32_t page_size, int32_t* d_free_pages, int32_t num_free,
                         const int32_t* d_first_free, int32_t* d_kv_lens_out, int32_t* d_shares_out,
                         int32_t* d_next_free, uint8_t* d_status, void* cuda_stream);

/*
 * Compacts a pool: its n pages in use (those that a sequence holds) become pages
 * 0 .. n - 1, so that the memory behind them can be given up or the pool's
 * tail cut off.  Pages below n stay where they are; the others go to the unused
 * places below n, both in ascending order.
 *
 *   d_block_table_out [num_seqs, max_pages]  entries of held pages are written,
 *                              others left as they are; may be d_block_table
 *                              itself (with the same stride).  A call in
 *                              place leaves new page numbers, which d_shares
 *                              does not go by: it is not to be repeated or
 *                              replayed before d_shares holds what
 *                              d_shares_out got
 *   d_shares_out  [num_pages]  at the pages' new places, 0 behind them
 *   d_free_pages_out [num_free]  the unused pages n .. num_pages - 1 in its last
 *                              num_pages - n entries, next_free and on; entries
 *                              in front are left as they are.  num_free >=
 *                              num_pages
 *   d_copy_from, d_copy_to [num_pages]  the pages to copy, -1 behind the last; no
 *                              page is in both
 *   d_num_copies  [1]
 *   d_next_free   [1]          num_free - (num_pages - n)
 *   d_status      [num_seqs]   TOPLOC_SEQ_*: BAD_LENGTH and BAD_PAGE as in
 *                              toploc_release_pages (the entry stays as it is)
 *
 * Lengths do not change.  Pages that no sequence holds and that were lost to the
 * free list are found again.
 */
int toploc_compact_pages(const int32_t* d_kv_lens, int32_t num_seqs, const int32_t* d_block_table, int32_t max_pages,
                         int64_t table_stride, const int32_t* d_shares, int32_t num_pages, int32_t page_size,
                         int32_t* d_block_table_out, int64_t table_out_stride, int32_t* d_shares_out,
                         int32_t* d_free_pages_out, int32_t num_free, int32_t* d_copy_from, int32_t* d_copy_to,
                         int32_t* d_num_copies, int32_t* d_next_free, uint8_t* d_status, void* cuda_stream);

/* Caches that share a block table (keys and values of all layers): one layout for all of them. */
typedef struct {
  int32_t dtype;      /* TOPLOC_DTYPE_* */
  int32_t num_pages, page_size, kv_heads, head_dim;
  int32_t num_caches; /* >= 0 */
  int64_t page_stride, token_stride, head_stride; /* elements */
} toploc_pool_layout;

/*
 * Copies pages inside every one of the caches: page d_copy_from[c] to page
 * d_copy_to[c], c < d_num_copies[0] (at most max_copies).  Pairs with a page
 * outside the caches are skipped.  No page may be written twice, or written and
 * read.
 *
 * h_caches       HOST array of num_caches DEVICE pointers (read before the call
 *                returns), aligned to the element
 */
int toploc_copy_pages(void* const* h_caches, const toploc_pool_layout* lay, const int32_t* d_copy_from,
                      const int32_t* d_copy_to, const int32_t* d_num_copies, int32_t max_copies, void* cuda_stream);

/* ---- queries and keys between projection and attention ------------------ */

#define TOPLOC_ROTARY_HALVES 0     /* channel c turns with channel c + rotary_dim / 2 */
#define TOPLOC_ROTARY_NEIGHBOURS 1 /* channel 2c turns with channel 2c + 1 */

typedef struct {
  int32_t dtype;      /* TOPLOC_DTYPE_* of all tensors and weights */
  int32_t head_dim;   /* 1 .. 256 */
  int32_t q_heads;    /* 1 .. 16384 */
  int32_t kv_heads;   /* 1 .. 16384 */
  int32_t rotary_dim; /* even, 0 .. head_dim: the first channels of a head turn, the rest stay */
  int32_t pairing;    /* TOPLOC_ROTARY_* */
  int64_t num_tokens; /* 0 .. 2^31 - 1 */
  float eps;          /* >= 0 */
  int32_t reserved;   /* 0 */
  int64_t q_token_stride, q_head_stride, k_token_stride, k_head_stride, v_token_stride, v_head_stride; /* elements */
  int64_t q_out_token_stride, q_out_head_stride, k_out_token_stride, k_out_head_stride;
} toploc_rotary_layout;

/*
 * The RMS norm of every head of the queries and keys, and the rotation by
 * position behind it, in one pass:
 *   y = x * rsqrt(mean over the head's channels(x^2) + eps) * weight
 *   (a, b) <- (a cos t - b sin t, a sin t + b cos t),  t = position * inv_freq[c]
 * for the pairs (a, b) = channels (c, c + rotary_dim / 2) or (2c, 2c + 1) of y,
 * c < rotary_dim / 2.  fp32 arithmetic with one rounding at the end (a head's sum
 * of squares has to fit fp32); t is formed and brought into one turn in 64 bits
 * with remainders, so that far positions are as exact as near ones, up to
 * |position * inv_freq| = 2^64.
 *
 * d_q, d_k       DEVICE [num_tokens, heads, head_dim], the last dimension
 *                contiguous (views of one projection are fine)
 * d_positions    DEVICE [num_tokens] int32 (as toploc_plan_pages writes them)
 * d_inv_freq     DEVICE [rotary_dim / 2] fp32
 * d_q_weight_opt, d_k_weight_opt  DEVICE [head_dim], NULL: no norm of that one
 * d_q_out, d_k_out  DEVICE; each may be its input (with the same strides), else
 *                they share no memory with the inputs or each other (refused,
 *                but not looked for where both have gaps of different lengths)
 * Pointers aligned to the element; heads at places of 16 (8) bytes, less than
 * 2^26 elements apart, whose channels and turned channels are whole vectors of
 * that size move as vectors, others element by element.  Asynchronous.
 */
int toploc_norm_rotary_prompt(const void* d_q, const void* d_k, const int32_t* d_positions, const float* d_inv_freq,
                              const void* d_q_weight_opt, const void* d_k_weight_opt, const toploc_rotary_layout* lay,
                              void* d_q_out, void* d_k_out, void* cuda_stream);

/*
 * The same, with keys and values [num_tokens, kv_heads, head_dim] written
 * straight to their slots of the paged cache (as toploc_cache_write does it:
 * negative slots and slots past the cache are skipped, distinct tokens have
 * distinct slots; values are copied as they are).  The k_out strides are not
 * used.
 */
int toploc_norm_rotary_paged(const void* d_q, const void* d_k, const void* d_v, const int32_t* d_positions,
                             const int64_t* d_slots, const float* d_inv_freq, const void* d_q_weight_opt,
                             const void* d_k_weight_opt, const toploc_rotary_layout* lay, void* d_q_out,
                             void* d_k_cache, void* d_v_cache, const toploc_kv_layout* kv, void* cuda_stream);

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

/* ---- log probabilities -------------------------------------------------- */

#define TOPLOC_MAX_ALTERNATIVES 32

typedef struct {
  int32_t dtype;      /* TOPLOC_DTYPE_* of the logits */
  int32_t vocab;      /* 1 .. 2^20 */
  int32_t top;        /* alternatives a row, 0 .. TOPLOC_MAX_ALTERNATIVES */
  int32_t reserved;   /* 0 */
  int64_t rows;       /* 0 .. 2^31 - 1 */
  int64_t row_stride; /* elements, >= vocab (columns past the vocabulary are not read) */
} toploc_logprob_layout;

/*
 * What a sampler or a validator reads off rows of logits x, in one pass over
 * them:
 *   logprob  = x[token] - lse,             lse = log sum_j exp(x_j)
 *   entropy  = -sum_j p_j log p_j,         p_j = exp(x_j - lse)
 *   top      = the `top` likeliest tokens, ordered by logit, equal ones by
 *              index (the first is the greedy token), and their log
 *              probabilities
 * in fp32, log probabilities at most 0, entropies at least 0.  A logit of -inf
 * is an impossible token: it has no part in entropy, its log probability is
 * -inf, and it is no alternative; places that no token is left for get id -1 and
 * -inf.  A row with nothing above -inf gets logprob -inf and entropy 0.  A row
 * with a NaN or +inf gets NaN for all but the ids (which pass over NaN).
 *
 * d_logits           DEVICE [rows, vocab], row_stride
 * d_tokens_opt       DEVICE [rows] int64, or NULL: no logprob; one outside the
 *                    vocabulary gets NaN
 * d_logprobs_opt     DEVICE [rows] fp32, NULL exactly where d_tokens is
 * d_entropy_opt      DEVICE [rows] fp32 or NULL
 * d_top_ids, d_top_logprobs  DEVICE [rows, top] int64 / fp32, NULL with top 0
 * Pointers aligned to their elements.  Asynchronous.  The same call gives the same
 * bits.  How a row is summed goes by the number of rows too, so the same row in a
 * call of another size can differ in the last bits of its log probabilities and
 * its entropy (not in its ids): a provider's and a validator's numbers are
 * compared with a tolerance.
 */
int toploc_token_logprobs(const void* d_logits, const toploc_logprob_layout* lay, const int64_t* d_tokens_opt,
                          float* d_logprobs_opt, float* d_entropy_opt, int64_t* d_top_ids, float* d_top_logprobs,
                          void* cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* TOPLOC_MODEL_H_ */
