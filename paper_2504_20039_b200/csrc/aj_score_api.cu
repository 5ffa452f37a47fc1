// Host side of aj_score.h: argument checks, the handle's workspace, choice of kernel, launches.
// No call synchronises or allocates but aj_score_create, aj_score_destroy and aj_score_last_status.
#include "../../include/aj_score.h"

#include <new>

#include "aj_norm.cuh"
#include "aj_score.cuh"

using namespace aj;

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                  const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
typedef CUresult (*ReplaceAddressFn)(CUtensorMap *, void *);

struct aj_score_s {
    int device = 0, num_sms = 0, max_pairs = 0;
    int max_rows = 0, group = 0, d = 0, V = 0, dtype = 0, max_top = 0;
    unsigned flags = 0;
    int tile = 0;            // entries per tile of the one-SM kernel
    bool tensor = false;     // a type and a width that the tensor-core kernels take
    EncodeTiledFn encode = nullptr;
    ReplaceAddressFn replace = nullptr;
    // tensor maps of W for tiles of both kernels, and of the last call's shape of h: a call puts its addresses in
    CUtensorMap w_one = {}, w_pair = {}, rows = {};
    long long rows_stride = -1;
    int rows_n = 0, rows_box = 0;
    float *logits = nullptr;
    float4 *parts = nullptr;
    unsigned *slots = nullptr;
    int *status = nullptr;
    int last_launches = 0;
    const char *last_path = "none";
};

namespace {

class Guard {  // a device for the duration of a call
   public:
    explicit Guard(int dev) {
        if (cudaGetDevice(&prev_) != cudaSuccess) prev_ = -1;
        if (prev_ != dev) ok_ = cudaSetDevice(dev) == cudaSuccess;
        changed_ = ok_ && prev_ != dev;
        if (!ok_) cudaGetLastError();
    }
    ~Guard() {
        if (changed_ && prev_ >= 0) cudaSetDevice(prev_);
    }
    bool ok() const { return ok_; }

   private:
    int prev_ = -1;
    bool ok_ = true, changed_ = false;
};

bool off(const void *p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) != 0; }

aj_status done(cudaError_t e) {
    if (e == cudaSuccess) return AJ_OK;
    cudaGetLastError();
    return AJ_ERR_CUDA;
}

// A tensor map of n rows of the handle's width, boxes of 128 bytes x box rows, 128-byte swizzle; zeros past the last row and column.
bool encode(aj_score h, CUtensorMap *m, void *any, long long n, long long stride, int box_rows) {
    const int e = h->dtype == AJ_BF16 ? 2 : 1;
    const cuuint64_t dims[2] = {(cuuint64_t)h->d, (cuuint64_t)n};
    const cuuint64_t strides[1] = {(cuuint64_t)stride * e};
    const cuuint32_t box[2] = {(cuuint32_t)(128 / e), (cuuint32_t)box_rows}, one[2] = {1, 1};
    return h->encode(m, e == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, any, dims, strides, box, one,
                     CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool at_address(aj_score h, CUtensorMap *m, const CUtensorMap &from, const void *p) {
    *m = from;
    return h->replace(m, const_cast<void *>(p)) == CUDA_SUCCESS;
}

template <typename F> bool driver_entry(const char *name, F *out) {
    void *fn = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion(name, &fn, 12000, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess || !fn) return false;
    *out = reinterpret_cast<F>(fn);
    return true;
}

bool fits_int(int64_t x) { return x >= -0x7fffffffll && x <= 0x7fffffffll; }

int elem(int dtype) { return dtype == AJ_BF16 ? 2 : dtype == AJ_F32 ? 4 : 1; }

}  // namespace

extern "C" {

aj_status aj_add_norm(int device, const void *x, long long x_stride, const void *residual, long long residual_stride, const float *weight,
                      float eps, long long rows, int d, aj_dtype dtype, void *residual_out, long long residual_out_stride, void *out,
                      long long out_stride, void *out8, long long out8_stride, float *scale8, void *cuda_stream) {
    if (device < 0 || rows < 0 || d < 1 || (dtype != AJ_BF16 && dtype != AJ_F32) || !(eps >= 0.0f) || !(eps < 1e30f)) return AJ_ERR_INVALID_ARG;
    if (rows == 0) return d > norm::MAX_D ? AJ_ERR_UNSUPPORTED : AJ_OK;  // (tensors without rows have no address)
    if ((!out && !out8) || !out8 != !scale8 || (out && out == residual_out)) return AJ_ERR_INVALID_ARG;
    if (d > norm::MAX_D || rows > 0x7fffffffll) return AJ_ERR_UNSUPPORTED;
    if (!x || !weight) return AJ_ERR_INVALID_ARG;
    // a single row needs no stride
    auto short_rows = [&](const void *p, long long stride) { return p && rows > 1 && stride < d; };
    if (short_rows(x, x_stride) || short_rows(residual, residual_stride) || short_rows(residual_out, residual_out_stride) || short_rows(out, out_stride) ||
        short_rows(out8, out8_stride))
        return AJ_ERR_INVALID_ARG;
    const int e = elem(dtype);
    if (off(x, e) || off(residual, e) || off(residual_out, e) || off(out, e) || off(weight, 4) || off(scale8, 4)) return AJ_ERR_INVALID_ARG;
    Guard guard(device);
    if (!guard.ok()) return AJ_ERR_CUDA;
    norm::Args a;
    a.x = x;
    a.r = residual;
    a.w = weight;
    a.r_out = residual_out;
    a.out = out;
    a.out8 = (uint8_t *)out8;
    a.scale8 = scale8;
    a.x_stride = x_stride;
    a.r_stride = residual_stride;
    a.r_out_stride = residual_out_stride;
    a.out_stride = out_stride;
    a.out8_stride = out8_stride;
    a.rows = (int)rows;
    a.d = d;
    a.eps = eps;
    auto ragged = [&](const void *p, long long stride, int bytes, unsigned n) { return p && (off(p, n) || (rows > 1 && (stride * bytes) % n != 0)); };
    const bool wide = d % 8 == 0 && !ragged(x, x_stride, e, 16) && !ragged(residual, residual_stride, e, 16) &&
                      !ragged(residual_out, residual_out_stride, e, 16) && !ragged(out, out_stride, e, 16) && !ragged(out8, out8_stride, 1, 8) && !off(weight, 16);
    return done(norm::launch(a, dtype == AJ_BF16, wide, (cudaStream_t)cuda_stream));
}

aj_status aj_add_norm_call(const aj_norm_args *a) {
    if (!a || !fits_int(a->device) || !fits_int(a->d) || !fits_int(a->dtype)) return AJ_ERR_INVALID_ARG;
    return aj_add_norm((int)a->device, a->x, a->x_stride, a->residual, a->residual_stride, a->weight, (float)a->eps, a->rows, (int)a->d, (aj_dtype)a->dtype,
                       a->residual_out, a->residual_out_stride, a->out, a->out_stride, a->out8, a->out8_stride, a->scale8, a->cuda_stream);
}

aj_status aj_score_create(aj_score *out, int device, int max_rows, int d, int V, int dtype, int max_top, unsigned flags) {
    if (!out) return AJ_ERR_INVALID_ARG;
    *out = nullptr;
    if (device < 0 || max_rows < 1 || d < 1 || V < 1 || max_top < 0 || max_top > AJ_SCORE_MAX_TOP) return AJ_ERR_INVALID_ARG;
    if (dtype != AJ_BF16 && dtype != AJ_F32 && dtype != AJ_E4M3) return AJ_ERR_INVALID_ARG;
    if (flags & ~AJ_SCORE_FLAG_FORCE_SIMT) return AJ_ERR_INVALID_ARG;
    if (d > 65536 || V > score::MAX_V) return AJ_ERR_UNSUPPORTED;
    int count = 0;
    if (cudaGetDeviceCount(&count) != cudaSuccess || device >= count) {
        cudaGetLastError();
        return AJ_ERR_CUDA;
    }
    int major = 0, sms = 0;
    if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, device) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess) {
        cudaGetLastError();
        return AJ_ERR_CUDA;
    }
    if (major != 10) return AJ_ERR_NOT_SM100;
    Guard guard(device);
    if (!guard.ok()) return AJ_ERR_CUDA;
    int max_pairs = 0;
    if (score::prepare_finish() != cudaSuccess || score::prepare_umma(sms, &max_pairs) != cudaSuccess) {
        cudaGetLastError();
        return AJ_ERR_CUDA;
    }
    aj_score h = new (std::nothrow) aj_score_s;
    if (!h) return AJ_ERR_CUDA;
    h->device = device;
    h->num_sms = sms;
    h->max_rows = max_rows;
    h->group = max_rows < score::group_rows(V) ? max_rows : score::group_rows(V);
    h->d = d;
    h->V = V;
    h->dtype = dtype;
    h->max_top = max_top;
    h->flags = flags;
    h->max_pairs = max_pairs;
    h->tile = score::one_sm_tile(V, sms);
    h->tensor = dtype != AJ_F32 && (long long)d * elem(dtype) % 16 == 0 && !(flags & AJ_SCORE_FLAG_FORCE_SIMT);
    if (h->tensor && (!driver_entry("cuTensorMapEncodeTiled", &h->encode) || !driver_entry("cuTensorMapReplaceAddress", &h->replace))) {
        cudaGetLastError();
        delete h;
        return AJ_ERR_CUDA;
    }
    // up to 128 rows in the one-SM kernel's tiles, or all of a group in tiles of 256: a row is whole tiles, so less than one more than V
    const size_t few = h->group < 128 ? h->group : 128, n_one = (V + h->tile - 1) / h->tile, n_wide = (V + 255) / 256;
    const size_t parts = few * n_one > h->group * n_wide ? few * n_one : h->group * n_wide;
    const size_t slots = (size_t)h->group * score::GATE_TOP * 4;
    if (cudaMalloc(&h->logits, (size_t)h->group * (V + 255) * 4) != cudaSuccess || cudaMalloc(&h->parts, parts * 16) != cudaSuccess ||
        cudaMalloc(&h->slots, slots) != cudaSuccess || zero_now(h->slots, slots) != cudaSuccess || cudaMalloc(&h->status, 256) != cudaSuccess ||
        zero_now(h->status, 256) != cudaSuccess) {
        cudaGetLastError();
        aj_score_destroy(h);
        return AJ_ERR_CUDA;
    }
    if (h->tensor && (!encode(h, &h->w_one, h->logits, V, d, h->tile) || !encode(h, &h->w_pair, h->logits, V, d, 128))) {
        aj_score_destroy(h);
        return AJ_ERR_CUDA;
    }
    *out = h;
    return AJ_OK;
}

aj_status aj_score_destroy(aj_score h) {
    if (!h) return AJ_ERR_INVALID_ARG;
    Guard guard(h->device);
    cudaFree(h->logits);
    cudaFree(h->parts);
    cudaFree(h->slots);
    cudaFree(h->status);
    delete h;
    return AJ_OK;
}

aj_status aj_score_tokens(aj_score h, const void *hidden, long long h_stride, const float *h_scale, const void *W, const float *w_scale,
                          const int32_t *tokens, int n_tok, int rows, int n_top, float inv_temperature, float *logprob, float *lse,
                          float *entropy, int32_t *top_id, float *top_logprob, void *cuda_stream) {
    if (!h || rows < 0 || n_tok < 0 || n_tok > AJ_SCORE_MAX_TOKENS || n_top < 0 || n_top > h->V) return AJ_ERR_INVALID_ARG;
    if (!(inv_temperature > 0.0f) || !(inv_temperature < 1e30f)) return AJ_ERR_INVALID_ARG;
    if (rows > h->max_rows || n_top > h->max_top) return AJ_ERR_WORKSPACE;
    h->last_launches = 0;
    if (rows == 0) return AJ_OK;
    const int e = elem(h->dtype);
    if (!hidden || !W || (rows > 1 && h_stride < h->d) || off(hidden, e) || off(W, e)) return AJ_ERR_INVALID_ARG;
    if ((h->dtype == AJ_E4M3) != (h_scale != nullptr) || !h_scale != !w_scale || off(h_scale, 4) || off(w_scale, 4)) return AJ_ERR_INVALID_ARG;
    if ((n_tok > 0 && (!tokens || !logprob)) || (n_top > 0 && !top_id)) return AJ_ERR_INVALID_ARG;
    if (off(tokens, 4) || off(logprob, 4) || off(lse, 4) || off(entropy, 4) || off(top_id, 4) || off(top_logprob, 4)) return AJ_ERR_INVALID_ARG;
    Guard guard(h->device);
    if (!guard.ok()) return AJ_ERR_CUDA;
    const cudaStream_t s = (cudaStream_t)cuda_stream;
    const bool tensor = h->tensor && !off(hidden, 16) && !off(W, 16) && (rows == 1 || h_stride * e % 16 == 0) && !off(w_scale, 16);
    const long long each = score::rows_each(rows, h->group);
    for (long long r0 = 0; r0 < rows; r0 += each) {
        score::Args a;
        a.h = (const char *)hidden + (size_t)r0 * h_stride * e;
        a.W = W;
        a.h_scale = h_scale ? h_scale + r0 : nullptr;
        a.w_scale = w_scale;
        a.tokens = n_tok ? tokens + (size_t)r0 * n_tok : nullptr;
        a.h_stride = h_stride;
        a.rows = (int)(rows - r0 < each ? rows - r0 : each);
        a.d = h->d;
        a.V = h->V;
        a.n_tok = n_tok;
        a.n_top = n_top;
        a.dtype = h->dtype;
        a.inv_t = inv_temperature;
        a.logprob = n_tok ? logprob + (size_t)r0 * n_tok : nullptr;
        a.lse = lse ? lse + r0 : nullptr;
        a.entropy = entropy ? entropy + r0 : nullptr;
        a.top_id = n_top ? top_id + (size_t)r0 * n_top : nullptr;
        a.top_logprob = n_top && top_logprob ? top_logprob + (size_t)r0 * n_top : nullptr;
        a.logits = h->logits;
        a.parts = h->parts;
        a.status = h->status;
        cudaError_t err;
        if (tensor) {
            const score::Plan p = score::plan_umma(a.rows, h->d, h->V, h->dtype, h->tile, h->num_sms, h->max_pairs);
            a.tile = p.tile;
            a.n_v = (h->V + p.tile - 1) / p.tile;
            a.ld = (long long)a.n_v * p.tile;
            if (h->rows_stride != h_stride || h->rows_n != a.rows || h->rows_box != p.box_rows) {
                h->rows_stride = -1;
                if (!encode(h, &h->rows, h->logits, a.rows, a.rows > 1 ? h_stride : h->d, p.box_rows)) return AJ_ERR_CUDA;
                h->rows_stride = h_stride, h->rows_n = a.rows, h->rows_box = p.box_rows;
            }
            CUtensorMap mh, mw;
            if (!at_address(h, &mh, h->rows, a.h) || !at_address(h, &mw, p.pair ? h->w_pair : h->w_one, W)) return AJ_ERR_CUDA;
            a.gate = n_top <= score::GATE_TOP && n_tok <= score::GATE_TOKENS;
            a.slots = h->slots;
            h->last_path = p.pair ? "umma_two_sm" : "umma_one_sm";
            err = score::launch_umma(mh, mw, a, p, s);
            h->last_launches += 2;
        } else {
            a.tile = 256;
            a.n_v = (h->V + 255) / 256;
            a.ld = (long long)a.n_v * a.tile;
            a.direct = a.n_v <= score::DIRECT_TILES;  // (a small f32 head: 10.6 us with a kernel for the tiles' sums, 9.8 without)
            h->last_path = "simt";
            err = score::launch_simt(a, s);
            h->last_launches += a.direct ? 2 : 3;
        }
        if (err == cudaSuccess) err = score::launch_finish(a, s);
        if (err != cudaSuccess) return done(err);
    }
    return AJ_OK;
}

aj_status aj_score_call(aj_score h, const aj_score_args *a) {
    if (!a || !fits_int(a->n_tok) || !fits_int(a->rows) || !fits_int(a->n_top)) return AJ_ERR_INVALID_ARG;
    return aj_score_tokens(h, a->hidden, a->h_stride, a->h_scale, a->W, a->w_scale, a->tokens, (int)a->n_tok, (int)a->rows, (int)a->n_top,
                           (float)a->inv_temperature, a->logprob, a->lse, a->entropy, a->top_id, a->top_logprob, a->cuda_stream);
}

aj_status aj_score_last_status(aj_score h) {
    if (!h) return AJ_ERR_INVALID_ARG;
    Guard guard(h->device);
    int s = 0;
    if (!guard.ok() || cudaDeviceSynchronize() != cudaSuccess || cudaMemcpy(&s, h->status, 4, cudaMemcpyDeviceToHost) != cudaSuccess) {
        cudaGetLastError();
        return AJ_ERR_CUDA;
    }
    if (s != 0 && zero_now(h->status, 4) != cudaSuccess) return AJ_ERR_CUDA;
    return s == DEV_TIMEOUT ? AJ_ERR_TIMEOUT : AJ_OK;
}

int aj_score_last_launch_count(aj_score h) { return h ? h->last_launches : 0; }
const char *aj_score_last_path(aj_score h) { return h ? h->last_path : "none"; }

}  // extern "C"
