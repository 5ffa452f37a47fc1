// aj_score_tokens on the CUDA cores: f32 storage, rows that no tensor map can describe, and the comparison path.
//
//   logits[m, v] = sum_k h[m, k] W[v, k]   one fixed order over k, f32
//
// Up to 8 rows: a warp per entry, its lanes along k, all rows at once; bound by the stream of W.  More rows: a CTA of 256
// threads computes a tile of 64 rows x 64 entries from k-slices of 32 staged in shared memory as f32, 4 x 4 outputs per thread; bound by
// the reads of shared memory that feed the multiply-adds.  A second kernel, a warp per row and tile, makes the tiles' sums.
#include "aj_score.cuh"

namespace aj {
namespace score {

namespace {

constexpr int BV = 64, BK = 32;

template <typename T> __device__ inline float widen(T x);
template <> __device__ inline float widen<float>(float x) { return x; }
template <> __device__ inline float widen<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <> __device__ inline float widen<__nv_fp8_e4m3>(__nv_fp8_e4m3 x) { return float(x); }

// Up to 8 rows: a warp takes entries in turn.
template <typename T> __global__ void __launch_bounds__(256) few_logits_kernel(Args a) {
    const T *h = (const T *)a.h, *W = (const T *)a.W;
    const int lane = threadIdx.x & 31;
    for (long long v = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); v < a.ld; v += (long long)gridDim.x * 8) {
        float acc[8] = {};
        if (v < a.V) {
#pragma unroll 4
            for (int k = lane; k < a.d; k += 32) {
                const float w = widen(W[(size_t)v * a.d + k]);
#pragma unroll
                for (int m = 0; m < 8; m++)
                    if (m < a.rows) acc[m] += w * widen(h[(size_t)m * a.h_stride + k]);
            }
        }
#pragma unroll
        for (int m = 0; m < 8; m++) {
            if (m >= a.rows) break;
#pragma unroll
            for (int o = 16; o; o >>= 1) acc[m] += __shfl_xor_sync(~0u, acc[m], o);
            if (lane == 0) {
                float x = acc[m];
                if (a.h_scale && v < a.V) x = x * a.h_scale[m] * a.w_scale[v];
                a.logits[(size_t)m * a.ld + v] = v < a.V ? x : -INFINITY;
            }
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(256) logits_kernel(Args a) {
    constexpr int TM = 64, RM = 4, RV = 4;  // outputs per thread
    constexpr int TX = BV / RV;             // threads along the entries
    static_assert(TX * (TM / RM) == 256, "256 threads cover the tile");
    __shared__ float sh[BK][TM + 4], sw[BK][BV + 4];
    const T *h = (const T *)a.h, *W = (const T *)a.W;
    const int v0 = blockIdx.x * BV, m0 = blockIdx.y * TM;
    const int tx = threadIdx.x % TX, ty = threadIdx.x / TX;
    float acc[RM][RV] = {};
    for (int k0 = 0; k0 < a.d; k0 += BK) {
        for (int i = threadIdx.x; i < TM * BK; i += 256) {
            const int m = i / BK, k = i % BK;
            sh[k][m] = m0 + m < a.rows && k0 + k < a.d ? widen(h[(size_t)(m0 + m) * a.h_stride + k0 + k]) : 0.0f;
        }
        for (int i = threadIdx.x; i < BV * BK; i += 256) {
            const int v = i / BK, k = i % BK;
            sw[k][v] = v0 + v < a.V && k0 + k < a.d ? widen(W[(size_t)(v0 + v) * a.d + k0 + k]) : 0.0f;
        }
        __syncthreads();
#pragma unroll 8
        for (int k = 0; k < BK; k++) {
            float x[RM], y[RV];
#pragma unroll
            for (int i = 0; i < RM; i++) x[i] = sh[k][ty * RM + i];
#pragma unroll
            for (int j = 0; j < RV; j++) y[j] = sw[k][tx * RV + j];
#pragma unroll
            for (int i = 0; i < RM; i++)
#pragma unroll
                for (int j = 0; j < RV; j++) acc[i][j] += x[i] * y[j];
        }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < RM; i++) {
        const int m = m0 + ty * RM + i;
        if (m >= a.rows) continue;
        const float s = a.h_scale ? a.h_scale[m] : 1.0f;
#pragma unroll
        for (int j = 0; j < RV; j++) {
            const int v = v0 + tx * RV + j;
            if (v >= a.ld) continue;
            float x = acc[i][j];
            if (a.w_scale && v < a.V) x = x * s * a.w_scale[v];
            a.logits[(size_t)m * a.ld + v] = v < a.V ? x : -INFINITY;
        }
    }
}

// Largest logit, S and T of each tile of a row: a warp per tile.
__global__ void __launch_bounds__(256) parts_kernel(Args a) {
    const int lane = threadIdx.x & 31, t = blockIdx.x * 8 + (threadIdx.x >> 5), m = blockIdx.y;
    if (t >= a.n_v) return;
    const float *x = a.logits + (size_t)m * a.ld + (size_t)t * a.tile;
    const float c = a.inv_t * LOG2E;
    float mx = -INFINITY;
    for (int i = lane; i < a.tile; i += 32) mx = max_nan(mx, x[i]);
#pragma unroll
    for (int o = 16; o; o >>= 1) mx = max_nan(mx, __shfl_xor_sync(~0u, mx, o));
    float S = 0.0f, T = 0.0f;
    for (int i = lane; i < a.tile; i += 32) {
        const float d = fmaxf((x[i] - mx) * c, -150.0f), e = ex2(d);
        S += e;
        T += d * e;
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        S += __shfl_xor_sync(~0u, S, o);
        T += __shfl_xor_sync(~0u, T, o);
    }
    if (lane == 0) a.parts[(size_t)m * a.n_v + t] = make_float4(mx, S, T, 0.0f);
}

template <typename T> void logits(const Args &a, cudaStream_t s) {
    const unsigned gx = (unsigned)((a.ld + BV - 1) / BV);
    if (a.rows <= 8)
        few_logits_kernel<T><<<(unsigned)((a.ld + 7) / 8 < 2048 ? (a.ld + 7) / 8 : 2048), 256, 0, s>>>(a);
    else
        logits_kernel<T><<<dim3(gx, (a.rows + 63) / 64), 256, 0, s>>>(a);
}

}  // namespace

cudaError_t launch_simt(const Args &a, cudaStream_t s) {
    if (a.dtype == F32)
        logits<float>(a, s);
    else if (a.dtype == BF16)
        logits<__nv_bfloat16>(a, s);
    else
        logits<__nv_fp8_e4m3>(a, s);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    parts_kernel<<<dim3((a.n_v + 7) / 8, a.rows), 256, 0, s>>>(a);
    return cudaGetLastError();
}

}  // namespace score
}  // namespace aj
