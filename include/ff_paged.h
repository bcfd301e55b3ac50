/*
 * ff_paged.h - C ABI of libff's paged key-value cache: appending new tokens of many
 * sequences to a pool of pages, and attention over it.
 *
 * The renderer cache of ff.h holds one clip: rings of equal chunks, whose lengths the
 * host knows.  Here one pool is shared by any number of sequences of unequal lengths
 * (streams of different ages, the text model that writes their prompts), whose lengths
 * and pages live in device memory, so that a captured graph can be replayed while the
 * sequences grow.
 *
 *   ff_paged_append     rotates K (and Q) of the new tokens by their positions and writes
 *                       K and V into the sequences' pages: ff_rope3d and ff_kv_publish in
 *                       one pass
 *   ff_paged_attention  attention of the new tokens over their sequences: one new token
 *                       each (decoding), a few, or whole prompts and renderer chunks
 *
 * The conventions of ff.h hold (memory, streams, errors, ff_status, ff_last_error()).  Calls
 * keep no state: two may run at once on two streams unless one writes what the other
 * reads or writes.  The device that the pointers and the stream belong to must be the
 * current one.
 *
 * The pool.  k_pages and v_pages are [num_pages][num_kv_heads][page_tokens][head_dim]
 *   arrays of dtype, one pair per layer, 16-byte aligned.  Sequence s holds kv_len[s]
 *   tokens; its token j is in page page_table[s * table_stride + j / page_tokens], slot j %
 *   page_tokens.
 * Holes.  A table entry outside [0, num_pages) is a hole: its tokens are not written, not
 *   read, and count as masked (a program that drops old pages writes -1 there).  So do
 *   tokens behind the table (j >= max_pages * page_tokens).
 * New tokens.  Rows q_start[s] .. q_start[s + 1] - 1 of a call's tensors belong to the last
 *   tokens of sequence s: with n = q_start[s + 1] - q_start[s], row q_start[s] + tau is token
 *   i = kv_len[s] - n + tau.  kv_len counts the new tokens, and may be 0.  Rows that belong
 *   to no sequence (behind q_start[n_seqs], say) are left as they are, and so are rows of
 *   tokens with i < 0 by ff_paged_append; ff_paged_attention gives those a zero row unless
 *   `block` lets them see something.  q_start must not decrease.
 * Pages shared by sequences may be read by all of them; the tokens that one ff_paged_append
 *   call writes must lie in different slots.
 */
#ifndef FF_PAGED_H_
#define FF_PAGED_H_

#include "ff.h"

#ifdef __cplusplus
extern "C" {
#endif

#define FF_MAX_PAGED_SEQS 1024   /* sequences per call */
#define FF_MIN_PAGE_TOKENS 16
#define FF_MAX_PAGE_TOKENS 256

/* Shape and plan of one call.
 *   num_pages        pages of the pool, >= 1
 *   page_tokens      tokens per page: 16, 32, 64, 128 or 256
 *   num_q_heads      a multiple of num_kv_heads; query head h reads kv head
 *                    h / (num_q_heads / num_kv_heads)
 *   head_dim         64 or 128
 *   dtype            ff_dtype of every tensor and of the pool
 *   n_seqs           sequences, 0 .. FF_MAX_PAGED_SEQS (0: nothing is done)
 *   n_tokens         rows of q, k, v and out, >= 0 (new tokens and rows behind them)
 *   max_pages        columns of page_table, >= 1; max_pages * page_tokens <= 2^30
 *   min_new, max_new bounds of a sequence's new tokens, 0 and 0: not known.  They choose
 *                    kernels: the results hold whatever they say.  max_new 1 for
 *                    decoding steps, min_new for batches of long prompts only.  max_pages
 *                    chooses too, since lengths are on the device: a table no wider than
 *                    the sequences need is the fastest for short ones
 *   table_stride     elements between rows of page_table (>= max_pages)
 *   q_start          device, n_seqs + 1 values
 *   kv_len           device, n_seqs values
 *   page_table       device, n_seqs rows                                             */
typedef struct {
  int32_t num_pages;
  int32_t page_tokens;
  int32_t num_q_heads;
  int32_t num_kv_heads;
  int32_t head_dim;
  int32_t dtype;
  int32_t n_seqs;
  int32_t n_tokens;
  int32_t max_pages;
  int32_t min_new;
  int32_t max_new;
  int32_t reserved;
  int64_t table_stride;
  const int32_t* q_start;
  const int32_t* kv_len;
  const int32_t* page_table;
} ff_paged_desc;

/* Rotation of ff_paged_append: the convention of ff_rope3d, rope_pairs_* and theta as in
 * ff_cache_desc (pairs all 0: the default split; (head_dim / 2, 0, 0): one axis). */
typedef struct {
  int32_t rope_pairs_t;
  int32_t rope_pairs_h;
  int32_t rope_pairs_w;
  int32_t reserved;
  double rope_theta;
} ff_paged_rope;

/* Append: K of every new token rotated by its position and V, written to the token's
 * page; q, when given, rotated into q_out ([n_tokens][num_q_heads][head_dim]; q_out may be
 * q itself when q is dense).  q, k and v are rows of heads, [head][head_dim] dense inside a
 * row, rows *_stride elements apart (a multiple of 16 bytes, at least a row: slices of one
 * projection's output can be passed as they are).  positions (device, [n_tokens][3], or
 * NULL) are the t, h and w positions of each row; NULL turns every axis by the token's
 * index i (text).  Angles, cosines, sines and the rotation are evaluated in float64 and
 * rounded once to dtype (nearest even); V is copied bit for bit.  The tensors must not
 * overlap the pool.  One kernel launch of at most 2^24 - 1 rows. */
ff_status ff_paged_append(const ff_paged_desc* desc, const ff_paged_rope* rope, const void* q,
                          const void* k, const void* v, int64_t q_stride, int64_t k_stride,
                          int64_t v_stride, const int32_t* positions, void* q_out, void* k_pages,
                          void* v_pages, void* stream);

/* Device workspace bytes that ff_paged_attention needs for `desc` (0 where it needs none;
 * 0 and an error for an invalid desc).  It depends on sizes only, never on the
 * device arrays. */
size_t ff_paged_attention_workspace(const ff_paged_desc* desc);

/* Attention of the new tokens.  Row i of sequence s (its token index, see above) attends to
 * the sequence's tokens j with
 *   block = 0 (causal)  j <= i         and (j >= i - window        or j < anchor_tokens)
 *   block = 1           j < kv_len[s]  and (j >= first - window    or j < anchor_tokens),
 * first being the index of the sequence's first new token (the renderer's read set:
 * anchors, a window of history, the chunk itself, bidirectional).  window -1: no bound;
 * window 0: the token (causal) or the new tokens (block) alone.  Per query head out =
 * softmax(softmax_scale * q K^T) V over those keys; a row that sees none is zero.  What
 * masked places of the pool hold does not matter (stale values, infinities, NaN).
 * q rows are q_stride elements apart as in ff_paged_append; out is dense, [n_tokens]
 * [num_q_heads][head_dim].  lse (optional, device, [n_tokens][num_q_heads] float) receives
 * the base-2 log-sum-exp of each row's scaled scores, -inf for a row that sees none.
 * Arithmetic as ff_chunk_attention: bf16 products on the matrix cores with float32
 * accumulation, softmax in float32, output rounded to bf16 (nearest even); f32 float32
 * throughout.  A bf16 probability enters the second product as two bf16 (2^-17) in the kernel
 * of few rows, and as one (2^-8) in the kernel of many.  Which one a sequence meets, how its keys
 * are split, and with both the last bits of a row, follow from the sizes of the whole batch,
 * the table's columns and the hints among them; asking for the log-sum-exp may change them too.
 * The same call gives the same bits.  Values of up to 2^127 give finite results, however many
 * keys weigh alike.  One to four kernel launches, by the sizes in `desc`.
 * workspace (device, 16-byte aligned, ff_paged_attention_workspace() bytes) is the call's
 * until its work is done: calls that may overlap, graphs among them, need one each.  out
 * and lse must not overlap anything else. */
ff_status ff_paged_attention(const ff_paged_desc* desc, const void* q, int64_t q_stride,
                             const void* k_pages, const void* v_pages, void* out, float* lse,
                             float softmax_scale, int32_t block, int32_t window,
                             int32_t anchor_tokens, void* workspace, size_t workspace_bytes,
                             void* stream);

#ifdef __cplusplus
}
#endif

#endif /* FF_PAGED_H_ */
