// aj_add_norm: s = x + r, y = s * rsqrt(mean(s^2) + eps) * w, stored in the storage type and / or in 8 bits with a scale per row.
//
// A row lives in registers from its loads to its stores, so everything is read and written once: the sum of squares and,
// for 8 bits, the largest |y| are the only values that cross threads.  Short rows take a warp each, longer ones a CTA.
// Bound by HBM, or by latency when there are few rows.  Measured: one row of 4096 2.4 us (2.8 to 8 bits
// too); 2112 rows of 4096 in both forms 15.9 us, 4.9 TB/s, 1.8 waves of eight CTAs per SM; 16000 rows of 8192 to 8 bits 141 us, 6.5 TB/s.
#include "aj_norm.cuh"

#include <cuda_bf16.h>
#include <cuda_fp8.h>

namespace aj {
namespace norm {

namespace {

__device__ inline float max_nan(float a, float b) {  // NaN if one of them is
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// Eight neighbouring elements.  (Plain loads: a row may be written in place.  Loads that ask to be evicted first cost 8 % of a long
// stream, stores that do gain 5 to 10 %.)
template <typename T, bool WIDE> __device__ inline void load8(const T *p, int n, float (&y)[8]) {
    if constexpr (!WIDE) {
#pragma unroll
        for (int i = 0; i < 8; i++) y[i] = i < n ? float(p[i]) : 0.0f;
    } else if constexpr (sizeof(T) == 2) {
        const uint4 u = *reinterpret_cast<const uint4 *>(p);
        const uint32_t v[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; i++) y[2 * i] = __uint_as_float(v[i] << 16), y[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
    } else {
        const float4 a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
        y[0] = a.x, y[1] = a.y, y[2] = a.z, y[3] = a.w, y[4] = b.x, y[5] = b.y, y[6] = b.z, y[7] = b.w;
    }
}
template <typename T, bool WIDE> __device__ inline void store8(T *p, int n, const float (&y)[8]) {
    if constexpr (!WIDE) {
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (i < n) p[i] = T(y[i]);
    } else if constexpr (sizeof(T) == 2) {
        uint32_t v[4];
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(y[2 * i], y[2 * i + 1]);
            v[i] = *reinterpret_cast<const uint32_t *>(&b);
        }
        __stcs(reinterpret_cast<uint4 *>(p), make_uint4(v[0], v[1], v[2], v[3]));
    } else {
        __stcs(reinterpret_cast<float4 *>(p), make_float4(y[0], y[1], y[2], y[3]));
        __stcs(reinterpret_cast<float4 *>(p) + 1, make_float4(y[4], y[5], y[6], y[7]));
    }
}
template <bool WIDE> __device__ inline void store8_e4m3(uint8_t *p, int n, const float (&y)[8]) {
    uint32_t v[2];
#pragma unroll
    for (int i = 0; i < 2; i++)
        v[i] = (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(y[4 * i], y[4 * i + 1]), __NV_SATFINITE, __NV_E4M3) |
               (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(y[4 * i + 2], y[4 * i + 3]), __NV_SATFINITE, __NV_E4M3) << 16;
    if (WIDE) {
        __stcs(reinterpret_cast<uint2 *>(p), make_uint2(v[0], v[1]));
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (i < n) p[i] = (uint8_t)(v[i >> 2] >> (8 * (i & 3)));
    }
}

// TPR threads per row, up to C pieces of eight elements each: 8 * TPR * C >= d.
template <typename T, bool WIDE, int TPR, int C>
__global__ void __launch_bounds__(TPR < 128 ? 128 : TPR) add_norm_kernel(Args a) {
    constexpr int ROWS = TPR < 128 ? 128 / TPR : 1, WARPS = TPR / 32;
    const int lane = threadIdx.x & 31, at = threadIdx.x % TPR, warp = at >> 5;
    const long long row = (long long)blockIdx.x * ROWS + threadIdx.x / TPR;
    if (row >= a.rows) return;  // whole warps; rows of several warps have a CTA of their own
    __shared__ float red[2][WARPS];
    const T *x = (const T *)a.x + row * a.x_stride, *r = a.r ? (const T *)a.r + row * a.r_stride : nullptr;
    float s[C][8];
    float sum = 0.0f;
#pragma unroll
    for (int c = 0; c < C; c++) {
        const int i = (c * TPR + at) * 8, n = a.d - i;
#pragma unroll
        for (int j = 0; j < 8; j++) s[c][j] = 0.0f;
        if (n > 0) load8<T, WIDE>(x + i, n, s[c]);
    }
    if (r) {
#pragma unroll
        for (int c = 0; c < C; c++) {
            const int i = (c * TPR + at) * 8, n = a.d - i;
            float y[8] = {};
            if (n > 0) load8<T, WIDE>(r + i, n, y);
#pragma unroll
            for (int j = 0; j < 8; j++) s[c][j] += y[j];
        }
    }
#pragma unroll
    for (int c = 0; c < C; c++)
#pragma unroll
        for (int j = 0; j < 8; j++) sum += s[c][j] * s[c][j];
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
    if (WARPS > 1) {
        if (lane == 0) red[0][warp] = sum;
        __syncthreads();
        sum = 0.0f;
#pragma unroll
        for (int w = 0; w < WARPS; w++) sum += red[0][w];
    }
    const float mean = sum / (float)a.d + a.eps, inv = mean == 0.0f ? 0.0f : rsqrtf(mean);  // (zeros under eps = 0 stay zeros)
    float top = 0.0f;
#pragma unroll
    for (int c = 0; c < C; c++) {
        const int i = (c * TPR + at) * 8, n = a.d - i;
        if (n <= 0) continue;
        if (a.r_out) store8<T, WIDE>((T *)a.r_out + row * a.r_out_stride + i, n, s[c]);
        float w[8];
        load8<float, WIDE>(a.w + i, n, w);
#pragma unroll
        for (int j = 0; j < 8; j++) {
            s[c][j] = s[c][j] * inv * w[j];
            top = max_nan(top, fabsf(s[c][j]));
        }
        if (a.out) store8<T, WIDE>((T *)a.out + row * a.out_stride + i, n, s[c]);
    }
    if (!a.out8) return;
#pragma unroll
    for (int o = 16; o; o >>= 1) top = max_nan(top, __shfl_xor_sync(~0u, top, o));
    if (WARPS > 1) {
        if (lane == 0) red[1][warp] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WARPS; w++) top = max_nan(top, red[1][w]);
    }
    const float scale = top / 448.0f;
    if (at == 0) a.scale8[row] = scale;
    // f32 does not hold 448 / top below 448 / 2^128: there the row and its scale are lifted by 2^96 (no scale: zeros)
    const float lift = top < 0x1p-119f ? 0x1p96f : 1.0f, lifted = scale * lift;
    const float q = top >= 0x1p-119f ? 448.0f / top : lifted == 0.0f ? 0.0f : 1.0f / lifted;
#pragma unroll
    for (int c = 0; c < C; c++) {
        const int i = (c * TPR + at) * 8, n = a.d - i;
        if (n <= 0) continue;
#pragma unroll
        for (int j = 0; j < 8; j++) s[c][j] = s[c][j] * lift * q;
        store8_e4m3<WIDE>(a.out8 + row * a.out8_stride + i, n, s[c]);
    }
}

template <typename T, bool WIDE, int TPR, int C> cudaError_t go(const Args &a, cudaStream_t s) {
    constexpr int ROWS = TPR < 128 ? 128 / TPR : 1;
    add_norm_kernel<T, WIDE, TPR, C><<<(unsigned)((a.rows + (long long)ROWS - 1) / ROWS), TPR < 128 ? 128 : TPR, 0, s>>>(a);
    return cudaGetLastError();
}

template <typename T, bool WIDE> cudaError_t pick(const Args &a, cudaStream_t s) {
    if (a.d <= 256) return go<T, WIDE, 32, 1>(a, s);
    if (a.d <= 1024) return go<T, WIDE, 32, 4>(a, s);
    if (a.d <= 2048) return go<T, WIDE, 128, 2>(a, s);
    if constexpr (sizeof(T) == 2)  // (f32 never asks for these)
        if (a.d <= 8192 && fewer_threads(a.rows, a.d, true)) return a.d <= 4096 ? go<T, WIDE, 128, 4>(a, s) : go<T, WIDE, 256, 4>(a, s);
    if (a.d <= 4096) return go<T, WIDE, 256, 2>(a, s);
    if (a.d <= 8192) return go<T, WIDE, 512, 2>(a, s);
    if (a.d <= 16384) return go<T, WIDE, 512, 4>(a, s);
    return go<T, WIDE, 1024, 4>(a, s);
}

}  // namespace

cudaError_t launch(const Args &a, bool bf16, bool wide, cudaStream_t s) {
    if (bf16) return wide ? pick<__nv_bfloat16, true>(a, s) : pick<__nv_bfloat16, false>(a, s);
    return wide ? pick<float, true>(a, s) : pick<float, false>(a, s);
}

}  // namespace norm
}  // namespace aj
