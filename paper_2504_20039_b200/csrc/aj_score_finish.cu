// aj_score_tokens, second step: from the tiles' sums and logits of a row to its outputs.
//
//   M = max of the tiles' largest logits, w = 2^((largest - M) c), c = inv_temperature log2(e)
//   S = sum w S_t,  T = sum w (T_t + (largest - M) c S_t)
//   lse = inv_temperature M + ln S,  entropy = ln2 (log2 S - T / S): every term of T has one sign, so nothing cancels
//
// Alternatives: the n largest logits of a row (the lower entry first among equals) lie in the n tiles that come first by their
// largest logit (the lower tile first among equals): before an entry outside of them come those n tiles' largest.  So one warp
// finds the border between these tiles and the others, all warps read the tiles' logits and keep the ones that are not below the least
// of the tiles' largest, and each of the few that are left counts how many come before it.  Their keys are 64 bits (value, then the
// complement of the index), so no two are equal and the order of collecting them does not matter.  (Picking the best n times,
// each time by the whole warp, took 0.8 us an alternative.)
//
// Bound by latency: a CTA per row, some 8 KB of sums and n tiles per row.
#include "aj_score.cuh"

namespace aj {
namespace score {

namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32;

__device__ inline unsigned long long key_of(float x, int i) { return (unsigned long long)ordered_image(x) << 32 | (uint32_t)~i; }

__device__ inline uint32_t warp_max(uint32_t x) { return warp_max_u32(x); }
__device__ inline uint32_t warp_min(uint32_t x) { return warp_min_u32(x); }
__device__ inline unsigned long long warp_max(unsigned long long x) {
    const uint32_t hi = warp_max_u32((uint32_t)(x >> 32));
    return (unsigned long long)hi << 32 | warp_max_u32((uint32_t)(x >> 32) == hi ? (uint32_t)x : 0u);
}
__device__ inline unsigned long long warp_min(unsigned long long x) { return ~warp_max(~x); }

// By one warp: the n-th largest of `count` numbers (1 <= n <= count), by halving the range that it can lie in: between the least and the
// largest of the lanes' largest, if that many are wanted.  Ends as soon as n lie above the middle, which is then as good a
// border: some 8 rounds where logits are as far apart as a model's.
template <typename K> __device__ inline K border(const K *x, int count, int n) {
    const int lane = threadIdx.x & 31;
    K most = 0;
#pragma unroll 4
    for (int i = lane; i < count; i += 32) most = x[i] > most ? x[i] : most;
    K lo = n <= 32 && count >= 32 ? warp_min(most) : 0, hi = warp_max(most);  // count(>= lo) >= n > count(> hi)
    while (lo < hi) {
        const K mid = lo + (hi - lo) / 2 + 1;
        int c = 0;
#pragma unroll 6
        for (int i = lane; i < count; i += 32) c += x[i] >= mid;
        c = __reduce_add_sync(~0u, c);
        if (c == n) return mid;
        if (c > n)
            lo = mid;
        else
            hi = mid - 1;
    }
    return lo;
}

// By one warp: the positions, in order, of the n numbers from a border on go to out; of those on the border the first.
template <typename K> __device__ inline void from_border(const K *x, int count, int n, K least, int *out) {
    const int lane = threadIdx.x & 31;
    int above = 0;
    for (int i = lane; i < count; i += 32) above += x[i] > least;
    int on = n - __reduce_add_sync(~0u, above);  // how many on the border belong to them
    for (int i0 = 0, at = 0; i0 < count; i0 += 32) {
        const K k = i0 + lane < count ? x[i0 + lane] : 0;
        const bool eq = i0 + lane < count && k == least;
        const unsigned before = (1u << lane) - 1, ties = __ballot_sync(~0u, eq);
        const bool in = (i0 + lane < count && k > least) || (eq && __popc(ties & before) < on);
        const unsigned who = __ballot_sync(~0u, in);
        if (in) out[at + __popc(who & before)] = i0 + lane;
        at += __popc(who);
        on = max(0, on - __popc(ties));
    }
}

__global__ void __launch_bounds__(THREADS) finish_kernel(Args a) {
    extern __shared__ unsigned long long found[];                 // [n_top * tile], then the tiles' largest
    uint32_t *tiles = reinterpret_cast<uint32_t *>(found + a.n_top * a.tile);
    __shared__ float red[3][WARPS];
    __shared__ int chosen[64], n_found;
    __shared__ uint32_t floor_image;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, m = blockIdx.x;
    const float4 *parts = a.parts + (size_t)m * a.n_v;
    const float *logits = a.logits + (size_t)m * a.ld;
    const float c = a.inv_t * LOG2E;
    // the given tokens are the caller's: their numbers can be read before the tiles are there
    const int tok = threadIdx.x < a.n_tok ? a.tokens[(size_t)m * a.n_tok + threadIdx.x] : -1;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (a.gate && threadIdx.x < a.n_top) a.slots[(size_t)m * a.n_top + threadIdx.x] = 0u;
    const float x_tok = (unsigned)tok < (unsigned)a.V ? logits[tok] : 0.0f;

    float M = -INFINITY;
#pragma unroll 4
    for (int t = threadIdx.x; t < a.n_v; t += THREADS) {
        const float x = parts[t].x;
        if (a.n_top) tiles[t] = ordered_image(x);
        M = max_nan(M, x);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) M = max_nan(M, __shfl_xor_sync(~0u, M, o));
    if (lane == 0) red[0][warp] = M;
    if (threadIdx.x == 0) n_found = 0;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WARPS; w++) M = max_nan(M, red[0][w]);
    const bool fine = M > -INFINITY && M < INFINITY;  // false for NaN
    const float nan = __int_as_float(0x7fffffff);
    const int n_tiles = min(a.n_top, a.n_v);
    if (warp == 0 && n_tiles) {
        const uint32_t least = border(tiles, a.n_v, n_tiles);
        from_border(tiles, a.n_v, n_tiles, least, chosen);
        // no alternative lies below the least of these tiles' largest (fewer tiles than alternatives: every entry counts)
        if (lane == 0) floor_image = a.n_top <= a.n_v ? least : 0u;
    }
    float S = 0.0f, T = 0.0f;
#pragma unroll 4
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
    for (int j = warp; j < n_tiles; j += WARPS) {
        const int v0 = chosen[j] * a.tile;
#pragma unroll 8
        for (int i = lane; i < a.tile; i += 32) {
            const int v = v0 + i;
            const float x = v < a.V ? logits[v] : -INFINITY;
            if (v < a.V && ordered_image(x) >= floor_image) found[atomicAdd(&n_found, 1)] = key_of(x, v);
        }
    }
    S = T = 0.0f;
#pragma unroll
    for (int w = 0; w < WARPS; w++) S += red[1][w], T += red[2][w];
    const float log_s = logf(S);
    auto logprob = [&](float x) { return fine ? (x - M) * a.inv_t - log_s : nan; };
    if (threadIdx.x == 0) {
        if (a.lse) a.lse[m] = fine ? M * a.inv_t + log_s : nan;
        if (a.entropy) a.entropy[m] = fine ? log_s - T / S * LN2 : nan;
    }
    if (threadIdx.x < a.n_tok) a.logprob[(size_t)m * a.n_tok + threadIdx.x] = (unsigned)tok < (unsigned)a.V ? logprob(x_tok) : nan;
    for (int i = threadIdx.x + THREADS; i < a.n_tok; i += THREADS) {
        const int t = a.tokens[(size_t)m * a.n_tok + i];
        a.logprob[(size_t)m * a.n_tok + i] = (unsigned)t < (unsigned)a.V ? logprob(logits[t]) : nan;
    }
    if (n_tiles == 0) return;
    __syncthreads();
    const int n = n_found;
    // the place of a candidate is the number of those before it
    auto place = [&](unsigned long long k, auto key, int count) {
        int before = 0;
#pragma unroll 4
        for (int i = 0; i < count; i++) before += key(i) > k;
        if (before < a.n_top) {
            a.top_id[(size_t)m * a.n_top + before] = (int)~(uint32_t)k;
            if (a.top_logprob) a.top_logprob[(size_t)m * a.n_top + before] = logprob(key_value(k));
        }
    };
    if (n < a.n_top) {  // only a row with NaN runs out of candidates
        for (int j = threadIdx.x; j < a.n_top; j += THREADS) {
            a.top_id[(size_t)m * a.n_top + j] = j;
            if (a.top_logprob) a.top_logprob[(size_t)m * a.n_top + j] = nan;
        }
    } else if (n <= THREADS) {
        if (threadIdx.x < n) place(found[threadIdx.x], [&](int i) { return found[i]; }, n);
    } else {  // many equal logits, or few tiles: first the n_top best of them
        if (warp == 0) {
            from_border(found, n, a.n_top, border(found, n, a.n_top), chosen);
            __syncwarp();
            for (int j = lane; j < a.n_top; j += 32) place(found[chosen[j]], [&](int i) { return found[chosen[i]]; }, a.n_top);
        }
    }
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
    // n_top tiles of candidates, and a number per tile
    cfg.dynamicSmemBytes = a.n_top ? (size_t)a.n_top * a.tile * 8 + (size_t)a.n_v * 4 : 0;
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
