/*
 * aj_kv — the key-value cache around the verify-and-judge cycle, on one B200 (sm_100a).
 *
 * aj_verify starts from the hidden states of a window of K + 1 rows.  These operators are the attention side
 * of the model pass that produces them, and of the draft model's single-token steps and the prompts before
 * them: write new tokens into a paged cache, attend against it, measure how much attention each cached token
 * receives, and drop the tokens that receive least.  They are part of the same library and use the status
 * values, storage types and conventions of aj_verify.h (nothing throws, aborts or synchronises unless stated).
 *
 * The cache of one layer.  k_pages and v_pages are [n_pages, Hkv, page_size, D], contiguous.  Slot j of
 * sequence b lies in page block_table[b, j / page_size], row j % page_size.  seq_lens[b] counts the slots in
 * use INCLUDING the new tokens of the call, so the same array serves aj_kv_append and aj_kv_attend of a step;
 * a rejected draft is taken back by lowering it.  Page numbers outside [0, n_pages) are read as page 0 and never
 * written; lengths outside [0, table_width * page_size] are clamped.  Slots past a sequence's length are never
 * used, whatever they hold (NaN included).  Sequences may share pages that are only read (a common beginning); a page that a
 * call writes, to append a token or to move one in an eviction, must belong to one sequence.  Outputs must not overlap
 * inputs but where a call says so.
 *
 * New tokens.  A call brings, for each of B sequences, n_q tokens (rows b * n_q + t of q, k, v, out); or, with
 * q_start [B + 1] (int32, device), a ragged number of at most n_q: rows q_start[b] .. q_start[b + 1] - 1.  Token t
 * of nq new tokens sits in slot seq_lens[b] - nq + t.  Query head i reads key head i / (Hq / Hkv).
 * Row strides (in elements) let q, k and v be slices of one projection's output; heads lie D apart.
 */
#ifndef AJ_KV_H
#define AJ_KV_H

#include "aj_verify.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct aj_kv_s *aj_kv;

/* Comparison switches for tests and measurements: keep aj_kv_attend and aj_kv_weigh on the CUDA-core kernels; let
 * aj_kv_attend_shared attend the shared slots together even where that is slower. */
enum { AJ_KV_FLAG_FORCE_SIMT = 1u, AJ_KV_FLAG_FORCE_SHARED = 4u };

/*
 * Create a handle for fixed head counts on CUDA device `device`.
 *   max_B, max_q  largest batch and number of new tokens per sequence a later call may use (max_B <= 4096)
 *   Hq, Hkv       query and key-value heads, Hq a multiple of Hkv
 *   D             head size: a multiple of 8, at most 256.  64 and 128 with AJ_BF16 run on the tensor cores
 *   page_size     slots per page: 16, 32, 64 or 128
 *   dtype         storage of q, k, v, out and the pages
 * The handle owns a device workspace for the partial results of attention that is split over the cache's
 * length; calls on one handle share it, so calls that overlap on the GPU race.  It is ready for any stream on return.  One
 * handle serves every layer of these sizes; making one takes 0.6 ms.
 * Errors: AJ_ERR_INVALID_ARG, AJ_ERR_UNSUPPORTED, AJ_ERR_CUDA, AJ_ERR_NOT_SM100.
 */
aj_status aj_kv_create(aj_kv *out, int device, int max_B, int max_q, int Hq, int Hkv, int D, int page_size,
                       aj_dtype dtype, unsigned flags);
aj_status aj_kv_destroy(aj_kv h);

/*
 * Norms of queries and keys per head, position rotation and the write into the cache, in one pass.
 *   y = x * rsqrt(mean(x^2) + eps) * w      where q_norm / k_norm [D] f32 are given (NULL: y = x)
 *   (a, b) -> (a cos - b sin, b cos + a sin) on the first rot_dim elements: pairs (i, i + rot_dim / 2), or
 *   (2i, 2i + 1) with interleaved != 0; rot_dim even, 0 <= rot_dim <= D (0: no rotation, cos_sin may be NULL)
 *   cos_sin [n_pos, rot_dim] f32: rot_dim / 2 cosines, then rot_dim / 2 sines of a position
 *   positions [rows] int32: each new token's position; NULL: its slot.  Clamped to [0, n_pos)
 *   q -> q_out (may be q itself), k and v -> their slots.  32-bit arithmetic, one rounding on the store
 *   slot_pos [B, Hkv, cap] int32, weight [B, Hkv, cap] f32, cap = table_width * page_size: optional state for
 *   aj_kv_weigh / aj_kv_evict; the new slots get the token's position and weight zero
 * New tokens whose slot would be negative (more new tokens than seq_lens) are rotated but not cached.
 * Errors: AJ_ERR_INVALID_ARG, AJ_ERR_WORKSPACE (B or n_q above the handle's), AJ_ERR_UNSUPPORTED (alignment: pages
 * and rows start on 16 bytes), AJ_ERR_CUDA.  The same for all calls below.
 */
aj_status aj_kv_append(aj_kv h, const void *q, long long q_stride, const void *k, long long k_stride, const void *v,
                       long long v_stride, const float *q_norm, const float *k_norm, float eps, const float *cos_sin,
                       int n_pos, int rot_dim, int interleaved, const int32_t *positions, void *k_pages, void *v_pages,
                       int n_pages, const int32_t *block_table, int table_width, const int32_t *seq_lens,
                       const int32_t *q_start, int B, int n_q, void *q_out, long long q_out_stride,
                       int32_t *slot_pos, float *weight, void *cuda_stream);

/*
 * Attention of the new tokens over the cache: out = softmax(scale * q K^T) V over the visible slots.
 * The token in slot p sees slot j iff j <= p and (window == 0, or j > p - window, or j < sinks).
 *   out [rows, Hq * D] (row stride out_stride), lse [rows, Hq] f32 optional: log of the sum of exponentials
 * A row that sees nothing, or whose visible scores are all -inf, gets zeros and lse = -inf.  A NaN or +infinite score makes its
 * row NaN, lse too.  Keys that a row does not see never reach it whatever they hold; a non-finite VALUE in a slot that other
 * rows of the call see may reach it.
 * Scores, maximum, sum and output accumulate in 32 bits.  On the tensor cores the weights exp(s - max) are rounded to bf16
 * before they meet V, and above 16 rows a quarter of the exponentials are a polynomial with a relative error below 4e-6: lse
 * is off by less than that (by 1e-6 where many slots share the weight).
 * Two runs on the same inputs give the same bits.
 * More than 16 rows (new tokens x query heads per key head) go to the tensor cores only where k_pages and v_pages start on
 * 128 bytes, as an allocation does, and Hq / Hkv <= 128; else the CUDA cores take them, many times slower: about the time
 * of plain matrix products in 32 bits, as for f32 and for head sizes other than 64 and 128.  Rows of q on 128 bytes (pointer and
 * stride) are loaded fastest.
 */
aj_status aj_kv_attend(aj_kv h, const void *q, long long q_stride, const void *k_pages, const void *v_pages, int n_pages,
                       const int32_t *block_table, int table_width, const int32_t *seq_lens, const int32_t *q_start,
                       int B, int n_q, float scale, int window, int sinks, void *out, long long out_stride, float *lse,
                       void *cuda_stream);

/*
 * Attention of a batch whose sequences share their first slots (few-shot examples, a system prompt, a document), which are
 * attended once for all of them instead of once for each, where that pays.  The result is that of aj_kv_attend with window 0, up to the order in
 * which the sums are added:
 *   m = max(m1, m2),  out = (e^(m1 - m) O1 + e^(m2 - m) O2) / (e^(m1 - m) l1 + e^(m2 - m) l2)
 * with O, l, m the weighted values, their sum and the maximum over the shared slots (1) and over a sequence's others (2), f32.
 * As in aj_kv_attend the weights are rounded to bf16 before they meet the values.
 *   shared        slots 0 .. shared - 1 of the sequences hold the same tokens (whole tiles of 128 of them are used together)
 *   shared_table  [shared / page_size, rounded up] int32: their pages
 * A sequence with at least `shared` slots before its new tokens is taken to share them.  Any other (a shorter one, one
 * of a padded batch) is attended by its own table alone; block_table names every page of a sequence, the shared ones too.
 * aj_kv_reserve_shared(h, max_rows) sets aside a workspace for max_rows new tokens of a call (2 * (D + 2) * Hq * 4 bytes each, and 20 to 60 MB
 * however few they are) unless the handle has as much; a larger one takes the place of a smaller, and 0 frees it.  It allocates and may wait for the device: call it
 * outside of captures, and before capturing calls that use the workspace.  Sequences of a ragged call whose tokens lie past max_rows are attended alone.
 * f32, head sizes other than 64 and 128, Hq / Hkv > 128, pages off 128 bytes, one sequence, or less than 128 shared
 * slots: aj_kv_attend's kernels do the whole call, nothing is shared and nothing need be reserved.
 * Errors: as aj_kv_attend; AJ_ERR_WORKSPACE also for B * n_q rows above max_rows, whether or not sharing would pay.
 */
aj_status aj_kv_reserve_shared(aj_kv h, int max_rows);
aj_status aj_kv_attend_shared(aj_kv h, const void *q, long long q_stride, const void *k_pages, const void *v_pages, int n_pages,
                              const int32_t *shared_table, int shared, const int32_t *block_table, int table_width,
                              const int32_t *seq_lens, const int32_t *q_start, int B, int n_q, float scale, void *out,
                              long long out_stride, float *lse, void *cuda_stream);

/*
 * Accumulated attention weight: weight_out[b, h, j] = weight[b, h, j] + sum over the counted new tokens t that see
 * slot j, and the query heads of key head h, of exp(scale * q k_j - lse).
 *   lse [rows, Hq]: what aj_kv_attend gave for the same q, window and sinks
 *   n_rows [B] int32 optional: only the first n_rows[b] new tokens of a sequence count (accept_len + 1 after a
 *   verification: a rejected draft's attention must not); NULL: all
 *   weight, weight_out [B, Hkv, cap] f32, may be the same.  Slots past the length are not written.
 */
aj_status aj_kv_weigh(aj_kv h, const void *q, long long q_stride, const float *lse, const void *k_pages, int n_pages,
                      const int32_t *block_table, int table_width, const int32_t *seq_lens, const int32_t *q_start,
                      const int32_t *n_rows, int B, int n_q, float scale, int window, int sinks, const float *weight,
                      float *weight_out, void *cuda_stream);

/*
 * Cut every (sequence, key head) whose length exceeds `keep` to `keep` slots.
 * Kept: tokens at a position below `sinks` and the `recent` newest positions, then the largest weights; the lower
 * slot wins ties, NaN counts as the lowest weight.  (sinks + recent <= keep.)  In place: the r-th kept slot past
 * `keep` (ascending) moves into the r-th dropped slot below it, keys, values, weight and position, so nothing else
 * moves and the pages past `keep` are free afterwards.  The order of slots changes; attention without a window
 * does not depend on it, and rotated keys carry their position.
 *   lens_out [B] = min(seq_lens, keep) (may be seq_lens); weight_out, slot_pos_out [B, Hkv, cap] may be the
 *   inputs; only slots below lens_out are written.
 */
aj_status aj_kv_evict(aj_kv h, void *k_pages, void *v_pages, int n_pages, const int32_t *block_table, int table_width,
                      const int32_t *seq_lens, int B, int keep, int sinks, int recent, const float *weight,
                      const int32_t *slot_pos, int32_t *lens_out, float *weight_out, int32_t *slot_pos_out,
                      void *cuda_stream);

/* AJ_OK, or AJ_ERR_TIMEOUT if a bounded wait of a kernel on this handle ran out since the last call of this
 * function (outputs since then are invalid; after this call the handle is as new).  Synchronises the device. */
aj_status aj_kv_last_status(aj_kv h);
/* Kernels launched by the last call on this handle, and the name of the path the last attend / weigh took. */
int aj_kv_last_launch_count(aj_kv h);
const char *aj_kv_last_path(aj_kv h);

#ifdef __cplusplus
}
#endif
#endif
