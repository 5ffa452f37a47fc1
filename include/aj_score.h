/*
 * aj_score — the last norm of a model pass and what is read off its hidden states, on one B200 (sm_100a).
 *
 * aj_verify answers which draft tokens stay.  These operators sit beside it on the same hidden states: aj_add_norm makes
 * them (and the inputs of the layers in between), aj_score_tokens gives, through the same LM head, the log probabilities of
 * given tokens, each row's entropy and its most likely alternatives.  They are part of the same library and use the status
 * values and conventions of aj_verify.h (nothing throws, aborts or synchronises unless stated).
 */
#ifndef AJ_SCORE_H
#define AJ_SCORE_H

#include "aj_verify.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct aj_score_s *aj_score;

/* Storage in 8 bits with scales (sign, 4 exponent and 3 mantissa bits, largest value 448), beside aj_dtype's values. */
enum { AJ_E4M3 = 2 };

/* Comparison switch for tests and measurements: keep aj_score_tokens on the CUDA-core kernel. */
enum { AJ_SCORE_FLAG_FORCE_SIMT = 1u };

/* Most alternatives and given tokens per row. */
enum { AJ_SCORE_MAX_TOP = 32, AJ_SCORE_MAX_TOKENS = 1024 };

/*
 * Residual addition and root-mean-square norm of each row, output in the storage type, in 8 bits, or both.
 *   s = x + residual;  y = s * rsqrt(mean(s^2) + eps) * weight        in 32 bits
 *   residual_out = s, out = y, each rounded once to the storage type; y comes from the unrounded s
 *   scale8 = max |y| / 448;  out8 = y / scale8 rounded to e4m3        the largest value of a row becomes 448
 *   x, residual, residual_out, out [rows, d], dtype AJ_BF16 or AJ_F32, on `device`; row strides in elements
 *   residual, residual_out NULL: no addition, the sum is not wanted
 *   weight [d] f32; out8 [rows, d] bytes, scale8 [rows] f32: both or neither; at least one of out and out8
 * residual_out may be x or residual, out may be x or residual (with the same strides); other overlaps are not allowed.
 * A row of zeros gets scale 0 and zeros, with eps = 0 too.  A scale below 2^-126 has fewer bits, and below 2^-150 it is 0, with zeros;
 * out8 goes by the scale as it is stored.  A row with a NaN, or whose square sum leaves f32's range, has no meaningful numbers;
 * its scale is then NaN if a y is.  rows may be 0.
 * d <= 32768.  Rows and weight on 16 bytes, 8-bit rows on 8 bytes, and d a multiple of 8 are fastest; all else goes element by element.
 * Errors: AJ_ERR_INVALID_ARG, AJ_ERR_UNSUPPORTED (d), AJ_ERR_CUDA.
 */
aj_status aj_add_norm(int device, const void *x, long long x_stride, const void *residual, long long residual_stride, const float *weight,
                      float eps, long long rows, int d, aj_dtype dtype, void *residual_out, long long residual_out_stride, void *out,
                      long long out_stride, void *out8, long long out8_stride, float *scale8, void *cuda_stream);

/* The same with its arguments in one structure, for bindings whose calls cost by the argument (18 of them 1.6 us through ctypes). */
typedef struct {
    int64_t device;
    const void *x;
    int64_t x_stride;
    const void *residual;
    int64_t residual_stride;
    const float *weight;
    double eps;
    int64_t rows, d, dtype;
    void *residual_out;
    int64_t residual_out_stride;
    void *out;
    int64_t out_stride;
    void *out8;
    int64_t out8_stride;
    float *scale8;
    void *cuda_stream;
} aj_norm_args;
aj_status aj_add_norm_call(const aj_norm_args *args);

/*
 * Create a handle for scoring through an LM head of V entries of width d on CUDA device `device`.
 *   max_rows   rows of hidden states a later call may bring
 *   dtype      storage of the hidden states and of W: AJ_BF16, AJ_F32 or AJ_E4M3
 *   max_top    alternatives a later call may ask for (0 .. AJ_SCORE_MAX_TOP)
 * The handle owns a device workspace: logits of up to 2560 rows at a time (4 bytes each, about 2 GB at most) and per-tile
 * sums; more rows are worked off in groups.  For 2112 rows of 128,256 entries it is 1.1 GB, of which a call with 5 alternatives writes an
 * eighth (only tiles that can matter are stored).  Creation takes 0.2 to 3 ms.  Calls on one handle share it, so calls that overlap on the GPU race.  Ready for any stream on return.
 * Errors: AJ_ERR_INVALID_ARG, AJ_ERR_UNSUPPORTED (d > 65536, V > 2^21), AJ_ERR_CUDA, AJ_ERR_NOT_SM100.
 */
aj_status aj_score_create(aj_score *out, int device, int max_rows, int d, int V, int dtype, int max_top, unsigned flags);
aj_status aj_score_destroy(aj_score h);

/*
 * Log probabilities of given tokens, entropy and the most likely alternatives of each row of hidden states.
 *   logit[m, v] = sum_k h[m, k] W[v, k]              AJ_E4M3: times h_scale[m], times w_scale[v]; f32
 *   z = inv_temperature * logit (inv_temperature > 0);  lse[m] = log sum_v exp z[m, v]
 *   logprob[m, i] = z[m, tokens[m, i]] - lse[m];  NaN for a token outside [0, V)
 *   entropy[m] = - sum_v p log p,  p = exp(z - lse)
 *   top_id[m, j], top_logprob[m, j]: the n_top entries with the largest logits, in order, the lowest entry first among equals
 *   (a zero's sign does not count)
 *   h [rows, d] row stride h_stride (elements); W [V, d] contiguous; h_scale [rows], w_scale [V] f32 (AJ_E4M3 only, else NULL)
 *   tokens [rows, n_tok] int32, logprob [rows, n_tok] f32 (n_tok 0: both NULL), lse [rows], entropy [rows] f32 optional,
 *   top_id [rows, n_top] int32, top_logprob [rows, n_top] f32 (n_top 0: both NULL; top_logprob optional)
 * Logits, maxima and sums are in 32 bits.  A row with a NaN or an infinite largest logit gets NaN in every f32 output, and
 * alternatives in [0, V) of no meaning.  Two runs on the same inputs give the same bits.  rows may be 0.
 * The tensor cores take AJ_BF16 and AJ_E4M3 where h, W and w_scale start on 16 bytes and rows are whole 16-byte pieces; all else
 * goes to the CUDA cores, many times slower.
 * Errors: AJ_ERR_INVALID_ARG, AJ_ERR_WORKSPACE (rows or n_top above the handle's), AJ_ERR_CUDA.
 */
aj_status aj_score_tokens(aj_score h, const void *hidden, long long h_stride, const float *h_scale, const void *W, const float *w_scale,
                          const int32_t *tokens, int n_tok, int rows, int n_top, float inv_temperature, float *logprob, float *lse,
                          float *entropy, int32_t *top_id, float *top_logprob, void *cuda_stream);

/* The same with its arguments in one structure. */
typedef struct {
    const void *hidden;
    int64_t h_stride;
    const float *h_scale;
    const void *W;
    const float *w_scale;
    const int32_t *tokens;
    int64_t n_tok, rows, n_top;
    double inv_temperature;
    float *logprob, *lse, *entropy;
    int32_t *top_id;
    float *top_logprob;
    void *cuda_stream;
} aj_score_args;
aj_status aj_score_call(aj_score h, const aj_score_args *args);

/* AJ_OK, or AJ_ERR_TIMEOUT if a bounded wait of a kernel on this handle ran out since the last call of this
 * function (outputs since then are invalid).  Synchronises the device. */
aj_status aj_score_last_status(aj_score h);
/* Kernels launched by the last call on this handle, and the name of the path it took. */
int aj_score_last_launch_count(aj_score h);
const char *aj_score_last_path(aj_score h);

#ifdef __cplusplus
}
#endif
#endif
