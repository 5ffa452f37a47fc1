// aj_score_tokens, second step: from the tiles' sums and logits of a row to its outputs.
//
//   M = max of the tiles' largest logits, w = 2^((largest - M) c), c = inv_temperature log2(e)
//   S = sum w S_t,  T = sum w (T_t + (largest - M) c S_t)
//   lse = inv_temperature M + ln S,  entropy = ln2 (log2 S - T / S): every term of T has one sign, so nothing cancels
//
// Alternatives: the n largest logits of a row (the lower entry first among equals) lie in the n tiles that come first by their
// largest logit (the lower tile first among equals): before an entry outside of them come those n tiles' largest.  So one warp
// picks the n tiles, all warps read those tiles' logits and keep the ones that are not below the n-th tile's largest, and one
// warp picks the n best of the few that are left.  Picking: each lane holds the best of its share as one 64-bit key (value,
// then the complement of the index), the warp takes the best of 32, and only the lane that had it looks again.
//
// Bound by latency: a CTA per row, some 8 KB of sums and n tiles per row.
#include "aj_score.cuh"

namespace aj {
namespace score {

namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32;

__device__ inline unsigned long long key_of(float x, int i) { return (unsigned long long)ordered_image(x) << 32 | (uint32_t)~i; }

// The largest of 32 keys, in every lane.
__device__ inline unsigned long long warp_best(unsigned long long k) {
    const uint32_t hi = warp_max_u32((uint32_t)(k >> 32));
    const uint32_t lo = warp_max_u32((uint32_t)(k >> 32) == hi ? (uint32_t)k : 0u);
    return (unsigned long long)hi << 32 | lo;
}

// By one warp: calls take(j, key) for the n largest of keys[0 .. count), in order.  Every key once, none is zero; keys that
// were taken are zero afterwards.
template <typename F> __device__ inline void pick(unsigned long long *keys, int count, int n, F take) {
    const int lane = threadIdx.x & 31;
    unsigned long long best = 0;
    int at = -1;
    auto look = [&]() {
        best = 0;
        for (int i = lane; i < count; i += 32)
            if (keys[i] > best) best = keys[i], at = i;
    };
    look();
    for (int j = 0; j < n; j++) {
        const unsigned long long k = warp_best(best);
        take(j, k);
        if (k != 0 && best == k) {
            keys[at] = 0;
            look();
        }
    }
}

__global__ void __launch_bounds__(THREADS) finish_kernel(Args a) {
    extern __shared__ unsigned long long smem[];
    unsigned long long *tiles = smem, *found = smem + a.n_v;      // [n_v], [n_top * tile]
    __shared__ float red[3][WARPS];
    __shared__ int chosen[64], n_found;
    __shared__ uint32_t floor_image;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, m = blockIdx.x;
    const float4 *parts = a.parts + (size_t)m * a.n_v;
    const float *logits = a.logits + (size_t)m * a.ld;
    const float c = a.inv_t * LOG2E;
    asm volatile("griddepcontrol.wait;" ::: "memory");

    float M = -INFINITY;
    for (int t = threadIdx.x; t < a.n_v; t += THREADS) {
        const float x = parts[t].x;
        if (a.n_top) tiles[t] = key_of(x, t);
        M = max_nan(M, x);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) M = max_nan(M, __shfl_xor_sync(~0u, M, o));
    if (lane == 0) red[0][warp] = M;
    if (threadIdx.x == 0) n_found = 0;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WARPS; w++) M = max_nan(M, red[0][w]);
    float S = 0.0f, T = 0.0f;
    for (int t = threadIdx.x; t < a.n_v; t += THREADS) {
        const float4 p = parts[t];
        const float d = fmaxf((p.x - M) * c, -150.0f), w = ex2(d);
        S += w * p.y;
        T += w * (p.z + d * p.y);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        S += __shfl_xor_sync(~0u, S, o);
        T += __shfl_xor_sync(~0u, T, o);
    }
    if (lane == 0) red[1][warp] = S, red[2][warp] = T;
    __syncthreads();
    S = T = 0.0f;
#pragma unroll
    for (int w = 0; w < WARPS; w++) S += red[1][w], T += red[2][w];
    const bool fine = M > -INFINITY && M < INFINITY;  // false for NaN
    const float nan = __int_as_float(0x7fffffff), log_s = logf(S);
    auto logprob = [&](float x) { return fine ? (x - M) * a.inv_t - log_s : nan; };
    if (threadIdx.x == 0) {
        if (a.lse) a.lse[m] = fine ? M * a.inv_t + log_s : nan;
        if (a.entropy) a.entropy[m] = fine ? log_s - T / S * LN2 : nan;
    }
    for (int i = threadIdx.x; i < a.n_tok; i += THREADS) {
        const int t = a.tokens[(size_t)m * a.n_tok + i];
        a.logprob[(size_t)m * a.n_tok + i] = (unsigned)t < (unsigned)a.V ? logprob(logits[t]) : nan;
    }
    if (a.n_top == 0) return;

    const int n_tiles = min(a.n_top, a.n_v);
    if (warp == 0)
        pick(tiles, a.n_v, n_tiles, [&](int j, unsigned long long k) {
            if (lane == 0) {
                chosen[j] = (int)~(uint32_t)k;
                // fewer tiles than alternatives: every entry counts
                if (j + 1 == n_tiles) floor_image = a.n_top <= a.n_v ? (uint32_t)(k >> 32) : 0u;
            }
        });
    __syncthreads();
    for (int j = warp; j < n_tiles; j += WARPS) {
        const int v0 = chosen[j] * a.tile;
        for (int i = lane; i < a.tile; i += 32) {
            const int v = v0 + i;
            if (v >= a.V) continue;
            const float x = logits[v];
            if (ordered_image(x) >= floor_image) found[atomicAdd(&n_found, 1)] = key_of(x, v);
        }
    }
    __syncthreads();
    if (warp == 0)
        pick(found, n_found, a.n_top, [&](int j, unsigned long long k) {
            if (lane == 0) {
                const int v = k ? (int)~(uint32_t)k : j;  // (a row with NaN may run out of candidates)
                a.top_id[(size_t)m * a.n_top + j] = v;
                if (a.top_logprob) a.top_logprob[(size_t)m * a.n_top + j] = logprob(logits[v]);
            }
        });
}

}  // namespace

cudaError_t prepare_finish() {
    cudaFuncAttributes fa;
    const cudaError_t e = cudaFuncGetAttributes(&fa, finish_kernel);
    if (e != cudaSuccess) return e;
    return cudaFuncSetAttribute(finish_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 232448 - (int)fa.sharedSizeBytes);
}

cudaError_t launch_finish(const Args &a, bool overlap, cudaStream_t s) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)a.rows);
    cfg.blockDim = dim3(THREADS);
    // a key per tile, and n_top tiles of candidates
    cfg.dynamicSmemBytes = a.n_top ? ((size_t)a.n_v + (size_t)a.n_top * a.tile) * 8 : 0;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = overlap;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, finish_kernel, a);
}

}  // namespace score
}  // namespace aj
