// aj_score_tokens on the CUDA cores: f32 storage, rows that no tensor map can describe, and the comparison path.
//
//   logits[m, v] = sum_k h[m, k] W[v, k]   one fixed order over k, f32
//
// Up to 8 rows: a warp per entry, its lanes along k (16 bytes at a time in f32), all rows at once; bound by the stream of W.
// More rows: a CTA of 256 threads computes a tile of 16, 32 or 64 rows x 128 entries, 2, 4 or 8 x 4 outputs per thread, from k-slices of 16 in shared
// memory as f32; the next slice is fetched into registers meanwhile.  Bound by the multiply-adds and the reads of shared memory that
// feed them.  A second kernel, a warp per row and tile, makes the tiles' sums; a head of few tiles leaves that to the last step.
//
// Measured, f32 (d = 4096): 5 rows, 128,256 entries 677 us, 3.1 TB/s; 264 rows, 32,000 entries 2313 us, 30 TFLOP/s; 17 rows in tiles of
// 32 1117 us (in tiles of 64 1832).
#include "aj_score.cuh"

namespace aj {
namespace score {

namespace {

template <typename T> __device__ inline float widen(T x);
template <> __device__ inline float widen<float>(float x) { return x; }
template <> __device__ inline float widen<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <> __device__ inline float widen<__nv_fp8_e4m3>(__nv_fp8_e4m3 x) { return float(x); }

// Up to 8 rows: a warp takes entries in turn.  VEC: f32, rows on 16 bytes and whole 16-byte pieces.
template <typename T, bool VEC> __global__ void __launch_bounds__(256) few_logits_kernel(Args a) {
    const T *h = (const T *)a.h, *W = (const T *)a.W;
    const int lane = threadIdx.x & 31;
    for (long long v = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); v < a.ld; v += (long long)gridDim.x * 8) {
        float acc[8] = {};
        if (v < a.V) {
            if constexpr (VEC) {
#pragma unroll 2
                for (int k = lane * 4; k < a.d; k += 128) {
                    const float4 w = __ldg(reinterpret_cast<const float4 *>(W + (size_t)v * a.d + k));
#pragma unroll
                    for (int m = 0; m < 8; m++) {
                        if (m >= a.rows) break;
                        const float4 x = __ldg(reinterpret_cast<const float4 *>(h + (size_t)m * a.h_stride + k));
                        acc[m] += w.x * x.x + w.y * x.y + w.z * x.z + w.w * x.w;
                    }
                }
            } else {
#pragma unroll 4
                for (int k = lane; k < a.d; k += 32) {
                    const float w = widen(W[(size_t)v * a.d + k]);
#pragma unroll
                    for (int m = 0; m < 8; m++)
                        if (m < a.rows) acc[m] += w * widen(h[(size_t)m * a.h_stride + k]);
                }
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

// RM: rows per thread, 2, 4 or 8
template <typename T, int RM> __global__ void __launch_bounds__(256) logits_kernel(Args a) {
    constexpr int TM = 8 * RM, TV = 128, BK = 16, RV = 4, PH = TM * BK / 256, PW = TV * BK / 256;
    __shared__ __align__(16) float sh[2][BK][TM + 4], sw[2][BK][TV + 4];
    const T *h = (const T *)a.h, *W = (const T *)a.W;
    const int v0 = blockIdx.x * TV, m0 = blockIdx.y * TM;
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;         // entries 4 tx .., rows RM ty ..
    const int lk = threadIdx.x & 15, lr = threadIdx.x >> 4;         // a thread fetches column lk of rows lr, lr + 16, ..
    float rh[PH], rw[PW];
    auto fetch = [&](int k0) {
        const bool on = k0 + lk < a.d;
#pragma unroll
        for (int i = 0; i < PH; i++) rh[i] = on && m0 + lr + 16 * i < a.rows ? widen(h[(size_t)(m0 + lr + 16 * i) * a.h_stride + k0 + lk]) : 0.0f;
#pragma unroll
        for (int i = 0; i < PW; i++) rw[i] = on && v0 + lr + 16 * i < a.V ? widen(W[(size_t)(v0 + lr + 16 * i) * a.d + k0 + lk]) : 0.0f;
    };
    auto put = [&](int b) {
#pragma unroll
        for (int i = 0; i < PH; i++) sh[b][lk][lr + 16 * i] = rh[i];
#pragma unroll
        for (int i = 0; i < PW; i++) sw[b][lk][lr + 16 * i] = rw[i];
    };
    float acc[RM][RV] = {};
    fetch(0);
    put(0);
    __syncthreads();
    for (int k0 = 0, b = 0; k0 < a.d; k0 += BK, b ^= 1) {
        if (k0 + BK < a.d) fetch(k0 + BK);
#pragma unroll
        for (int k = 0; k < BK; k++) {
            const float4 w = *reinterpret_cast<const float4 *>(&sw[b][k][tx * RV]);
            const float y[RV] = {w.x, w.y, w.z, w.w};
            float x[RM];
#pragma unroll
            for (int i = 0; i < RM; i += 2) {
                const float2 z = *reinterpret_cast<const float2 *>(&sh[b][k][ty * RM + i]);
                x[i] = z.x, x[i + 1] = z.y;
            }
#pragma unroll
            for (int i = 0; i < RM; i++)
#pragma unroll
                for (int j = 0; j < RV; j++) acc[i][j] += x[i] * y[j];
        }
        if (k0 + BK < a.d) put(b ^ 1);
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
    const int t = blockIdx.x * 8 + (threadIdx.x >> 5), m = blockIdx.y;
    if (t >= a.n_v) return;
    const float4 p = part_of_tile(a.logits + (size_t)m * a.ld + (size_t)t * a.tile, a.tile, a.inv_t * LOG2E);
    if ((threadIdx.x & 31) == 0) a.parts[(size_t)m * a.n_v + t] = p;
}

template <typename T> void logits(const Args &a, cudaStream_t s) {
    if (a.rows <= 8) {
        const unsigned grid = (unsigned)((a.ld + 7) / 8 < 2048 ? (a.ld + 7) / 8 : 2048);
        if constexpr (sizeof(T) == 4) {
            if (((reinterpret_cast<uintptr_t>(a.h) | reinterpret_cast<uintptr_t>(a.W)) & 15) == 0 && a.d % 4 == 0 && (a.rows == 1 || a.h_stride % 4 == 0)) {
                few_logits_kernel<T, true><<<grid, 256, 0, s>>>(a);
                return;
            }
        }
        few_logits_kernel<T, false><<<grid, 256, 0, s>>>(a);
    } else {
        // a tile of 64 rows costs the same however many of them there are
        const unsigned gx = (unsigned)((a.ld + 127) / 128);
        if (a.rows <= 16)
            logits_kernel<T, 2><<<gx, 256, 0, s>>>(a);
        else if (a.rows <= 32)
            logits_kernel<T, 4><<<gx, 256, 0, s>>>(a);
        else
            logits_kernel<T, 8><<<dim3(gx, (a.rows + 63) / 64), 256, 0, s>>>(a);
    }
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
    if (e != cudaSuccess || a.direct) return e;
    parts_kernel<<<dim3((a.n_v + 7) / 8, a.rows), 256, 0, s>>>(a);
    return cudaGetLastError();
}

}  // namespace score
}  // namespace aj
