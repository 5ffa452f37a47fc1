// Declarations shared by the scoring kernels.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include "aj_internal.cuh"

namespace aj {
namespace score {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

enum { BF16 = 0, F32 = 1, E4M3 = 2 };  // aj_dtype and AJ_E4M3

// Rows whose logits the workspace holds at once: up to ten row tiles of the two-SM kernel (1.3 GB at 128,256 entries), of a larger
// vocabulary as many as take 2 GB.
constexpr int GROUP_ROWS = 2560;
inline int group_rows(int V) {
    const long long n = (2ll << 30) / (4ll * V) / 256 * 256;
    return n < 256 ? 256 : n < GROUP_ROWS ? (int)n : GROUP_ROWS;
}
// Rows of each group of a call, evenly, in whole row tiles.  (In 64 bits: a call may have 2^31 - 1 rows.)
inline long long rows_each(long long rows, int group) {
    const long long n = (rows + group - 1) / group, even = (rows + n - 1) / n, tiles = (even + 255) / 256 * 256;
    return n == 1 ? even : tiles < group ? tiles : group;
}

// One group of rows on its way through a call.
struct Args {
    const void *h = nullptr, *W = nullptr;
    const float *h_scale = nullptr, *w_scale = nullptr;
    const int *tokens = nullptr;
    long long h_stride = 0;
    int rows = 0, d = 0, V = 0, n_tok = 0, n_top = 0, dtype = 0;
    float inv_t = 1.0f;
    float *logprob = nullptr, *lse = nullptr, *entropy = nullptr, *top_logprob = nullptr;
    int *top_id = nullptr;
    // workspace
    float *logits = nullptr;   // [rows][ld]
    float4 *parts = nullptr;   // [rows][n_v]: a tile's largest logit, S = sum 2^d and T = sum d 2^d, d = (logit - largest) * c
    long long ld = 0;
    int tile = 0, n_v = 0;     // entries per tile, tiles
    // Which tiles' logits are stored: all, or (gate) those that may hold an alternative or that hold a given token.  The largest
    // logits that a row's tiles had so far lie in n_top slots, as ordered integers, a tile's number modulo n_top being its slot:
    // n_top tiles reach the least of the slots, so what lies below it is no alternative.  Zero between calls.
    int gate = 0;
    unsigned *slots = nullptr;  // [rows][n_top]
    int direct = 0;  // the last step makes the tiles' sums itself (up to DIRECT_TILES of them)
    int *status = nullptr;
};

constexpr int DIRECT_TILES = 64;
constexpr int GATE_TOP = 16, GATE_TOKENS = 8;  // up to so many alternatives and given tokens per row

// How the tcgen05 kernel cuts a group of rows.
struct Plan {
    bool pair = false;         // two SMs per tile
    int tile = 0, n_v = 0, n_m = 0;  // entries per tile, tiles of entries, tiles of rows
    int box_rows = 0, num_kb = 0, stages = 0, grid = 0;
    int kps = 1;               // k-blocks per stage: 1 or 2
};
cudaError_t prepare_umma(int num_sms, int *max_pairs);
int one_sm_tile(int V, int num_sms);
Plan plan_umma(int rows, int d, int V, int dtype, int tile, int num_sms, int max_pairs);
// maps: h in boxes of box_rows, W in boxes of a CTA's share of a tile, both 128 bytes wide with 128-byte swizzle
cudaError_t launch_umma(const CUtensorMap &mh, const CUtensorMap &mw, const Args &a, const Plan &p, cudaStream_t s);
cudaError_t launch_simt(const Args &a, cudaStream_t s);
cudaError_t launch_finish(const Args &a, cudaStream_t s);  // as a programmatic dependent of the kernel before it
cudaError_t prepare_finish();
// The finishing kernel keeps two keys per tile, or per entry of AJ_SCORE_MAX_TOP tiles, in shared memory (128 KB at most).
constexpr int MAX_TILES = 8192, MAX_V = MAX_TILES * 256;

#ifdef __CUDACC__

__device__ inline float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ inline float max_nan(float a, float b) {  // NaN if one of them is
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ inline float max3_nan(float a, float b, float c) {
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// By a warp: a tile's largest logit, S and T (c = inv_temperature log2(e)), in every lane.
__device__ inline float4 part_of_tile(const float *x, int n, float c) {
    const int lane = threadIdx.x & 31;
    float mx = -INFINITY;
#pragma unroll 8
    for (int i = lane; i < n; i += 32) mx = max_nan(mx, x[i]);
#pragma unroll
    for (int o = 16; o; o >>= 1) mx = max_nan(mx, __shfl_xor_sync(~0u, mx, o));
    float S = 0.0f, T = 0.0f;
#pragma unroll 8
    for (int i = lane; i < n; i += 32) {
        const float d = fmaxf((x[i] - mx) * c, -150.0f), e = ex2(d);
        S += e;
        T += d * e;
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        S += __shfl_xor_sync(~0u, S, o);
        T += __shfl_xor_sync(~0u, T, o);
    }
    return make_float4(mx, S, T, 0.0f);
}

#endif

}  // namespace score
}  // namespace aj
