// Host side of aj_score.h: argument checks, the handle's workspace, choice of kernel, launches.
// No call synchronises or allocates but aj_score_create, aj_score_destroy and aj_score_last_status.
#include "../../include/aj_score.h"

#include <new>

#include "aj_norm.cuh"
#include "aj_score.cuh"

using namespace aj;

struct aj_score_s {
    int device = 0, num_sms = 0;
    int max_rows = 0, group = 0, d = 0, V = 0, dtype = 0, max_top = 0;
    unsigned flags = 0;
    int tile = 0, n_v = 0;   // entries per tile of the workspace's layout, tiles
    long long ld = 0;        // entries of a row of the workspace
    float *logits = nullptr;
    float4 *parts = nullptr;
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

int elem(int dtype) { return dtype == AJ_BF16 ? 2 : dtype == AJ_F32 ? 4 : 1; }

}  // namespace

extern "C" {

aj_status aj_add_norm(int device, const void *x, long long x_stride, const void *residual, long long residual_stride, const float *weight,
                      float eps, long long rows, int d, aj_dtype dtype, void *residual_out, long long residual_out_stride, void *out,
                      long long out_stride, void *out8, long long out8_stride, float *scale8, void *cuda_stream) {
    if (device < 0 || rows < 0 || d < 1 || (dtype != AJ_BF16 && dtype != AJ_F32) || !(eps >= 0.0f) || !(eps < 1e30f)) return AJ_ERR_INVALID_ARG;
    if ((!out && !out8) || !out8 != !scale8) return AJ_ERR_INVALID_ARG;
    if (d > norm::MAX_D || rows > 0x7fffffffll) return AJ_ERR_UNSUPPORTED;
    if (rows == 0) return AJ_OK;
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
    if (score::prepare_finish() != cudaSuccess) {
        cudaGetLastError();
        return AJ_ERR_CUDA;
    }
    aj_score h = new (std::nothrow) aj_score_s;
    if (!h) return AJ_ERR_CUDA;
    h->device = device;
    h->num_sms = sms;
    h->max_rows = max_rows;
    h->group = max_rows < score::GROUP_ROWS ? max_rows : score::GROUP_ROWS;
    h->d = d;
    h->V = V;
    h->dtype = dtype;
    h->max_top = max_top;
    h->flags = flags;
    h->tile = 256;
    h->n_v = (V + h->tile - 1) / h->tile;
    h->ld = (long long)h->n_v * h->tile;
    if (cudaMalloc(&h->logits, (size_t)h->group * h->ld * 4) != cudaSuccess || cudaMalloc(&h->parts, (size_t)h->group * h->n_v * 16) != cudaSuccess ||
        cudaMalloc(&h->status, 256) != cudaSuccess || zero_now(h->status, 256) != cudaSuccess) {
        cudaGetLastError();
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
    // groups of rows, evenly
    const int n_groups = (rows + h->group - 1) / h->group, each = (rows + n_groups - 1) / n_groups;
    for (int r0 = 0; r0 < rows; r0 += each) {
        score::Args a;
        a.h = (const char *)hidden + (size_t)r0 * h_stride * e;
        a.W = W;
        a.h_scale = h_scale ? h_scale + r0 : nullptr;
        a.w_scale = w_scale;
        a.tokens = n_tok ? tokens + (size_t)r0 * n_tok : nullptr;
        a.h_stride = h_stride;
        a.rows = rows - r0 < each ? rows - r0 : each;
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
        a.ld = h->ld;
        a.tile = h->tile;
        a.n_v = h->n_v;
        a.status = h->status;
        h->last_path = "simt";
        cudaError_t err = score::launch_simt(a, s);
        if (err == cudaSuccess) err = score::launch_finish(a, false, s);
        if (err != cudaSuccess) return done(err);
        h->last_launches += 3;
    }
    return AJ_OK;
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
