// aj_score_tokens, second step: from the tiles' sums and logits of a row to its outputs.
//
//   M = max of the tiles' largest logits, w = 2^((largest - M) c), c = inv_temperature log2(e)
//   S = sum w S_t,  T = sum w (T_t + (largest - M) c S_t)
//   lse = inv_temperature M + ln S,  entropy = ln2 (log2 S - T / S): every term of T has one sign, so nothing cancels
//
// Alternatives: the n largest logits of a row (the lower entry first among equals) lie in the n tiles that come first by their
// largest logit (the lower tile first among equals): before an entry outside of them come those n tiles' largest.  So these
// tiles are found first, then all warps read their logits and keep the ones that are not below the least of the tiles' largest,
// and of the few that are left the n best are the answer.  (Picking the best n times took 0.8 us an
// alternative.)  Keys are 64 bits (value, then the complement of the index), so no two are equal and the order of collecting them does not matter.
//
// Bound by latency: a CTA per row, some 8 KB of sums and n tiles per row.  17 rows with 8 alternatives take 4 us after the tiles are
// there (loads 0.7, the tiles 1, their logits 1.1), without alternatives 2; 2112 rows 21, bound by instructions.  Rows of equal logits
// (zeros) take some 10 to 50 us more each wave of CTAs: more keys to halve.
#include "aj_score.cuh"

namespace aj {
namespace score {

namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32;

__device__ inline unsigned long long key_of(float x, int i) { return (unsigned long long)ordered_image(x) << 32 | (uint32_t)~i; }

// How many of keys[i0 .. i1) are like that; eight are read at a time.
template <typename P> __device__ __forceinline__ int count_if(const unsigned long long *keys, int i0, int i1, P like) {
    int n = 0, j = i0;
    for (; j + 8 <= i1; j += 8) {
        unsigned long long y[8];
#pragma unroll
        for (int u = 0; u < 8; u++) y[u] = keys[j + u];
#pragma unroll
        for (int u = 0; u < 8; u++) n += like(y[u]);
    }
    for (; j < i1; j++) n += like(keys[j]);
    return n;
}

// By all threads: take(key, place) for the n largest of `count` different keys (n <= count) of numbers below `limit`, with their places among
// them.  More than 64 are first cut to those from the n-th largest value on, found by
// halving the range that it can lie in, with each thread's values in registers; that ends as soon as n values lie above the middle.
// Where that leaves more than 64 (equal values: a row of zeros of a padded batch, of NaN), the lowest numbers among the equal ones
// are found in the same way.  Each key that is left then counts the ones before it.  `left` has room for all of them; keys are overwritten.
template <typename F>
__device__ __forceinline__ void top_of(unsigned long long *keys, int count, int n, int limit, unsigned long long *left, int *n_left, F take) {
    constexpr int KEEP = 4;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (count > 64) {
        __shared__ uint32_t tops[WARPS];
        __shared__ int sums[2][WARPS];
        uint32_t x[KEEP], most = 0;
#pragma unroll
        for (int j = 0; j < KEEP; j++) {
            const int i = threadIdx.x + j * THREADS;
            x[j] = i < count ? (uint32_t)(keys[i] >> 32) : 0u;
            most = max(most, x[j]);
        }
        for (int i = threadIdx.x + KEEP * THREADS; i < count; i += THREADS) most = max(most, (uint32_t)(keys[i] >> 32));
        most = warp_max_u32(most);
        if (lane == 0) tops[warp] = most;
        __syncthreads();
        uint32_t lo = ~0u, hi = 0;  // the warps' largest are WARPS of the values (0 where a warp has none)
#pragma unroll
        for (int w = 0; w < WARPS; w++) lo = min(lo, tops[w]), hi = max(hi, tops[w]);
        lo = n == 1 ? hi : n <= WARPS ? lo : 0u;
        for (int it = 0; lo < hi; it ^= 1) {  // count(>= lo) >= n > count(> hi)
            const uint32_t mid = lo + (hi - lo) / 2 + 1;
            int c = 0;
#pragma unroll
            for (int j = 0; j < KEEP; j++) c += x[j] >= mid;
            for (int i = threadIdx.x + KEEP * THREADS; i < count; i += THREADS) c += (uint32_t)(keys[i] >> 32) >= mid;
            c = __reduce_add_sync(~0u, c);
            if (lane == 0) sums[it][warp] = c;
            __syncthreads();
            c = 0;
#pragma unroll
            for (int w = 0; w < WARPS; w++) c += sums[it][w];
            if (c >= n)
                lo = mid;
            else
                hi = mid - 1;
            if (c == n) break;
        }
        for (int i = threadIdx.x; i < count; i += THREADS) {
            const unsigned long long k = keys[i];
            if ((uint32_t)(k >> 32) >= lo) left[atomicAdd(n_left, 1)] = k;
        }
        __syncthreads();
        count = *n_left;
        if (count > 64) {  // (ranking them all by counting took 1 ms a row with 20 alternatives)
            __shared__ int n_kept;
            if (threadIdx.x == 0) n_kept = 0;
            uint32_t from = ~(uint32_t)(limit - 1), to = ~0u;
            for (int it = 0; from < to; it ^= 1) {
                const uint32_t mid = from + (to - from) / 2 + 1;
                const unsigned long long least = (unsigned long long)lo << 32 | mid;
                int c = 0;
                for (int i = threadIdx.x; i < count; i += THREADS) c += left[i] >= least;
                c = __reduce_add_sync(~0u, c);
                if (lane == 0) sums[it][warp] = c;
                __syncthreads();
                c = 0;
#pragma unroll
                for (int w = 0; w < WARPS; w++) c += sums[it][w];
                if (c >= n)
                    from = mid;
                else
                    to = mid - 1;
                if (c == n) break;
            }
            for (int i = threadIdx.x; i < count; i += THREADS)
                if (left[i] >= ((unsigned long long)lo << 32 | from)) keys[atomicAdd(&n_kept, 1)] = left[i];
            __syncthreads();
            count = n_kept;
        } else {
            keys = left;
        }
    }
    for (int i = threadIdx.x; i < count; i += THREADS) {
        const unsigned long long k = keys[i];
        const int before = count_if(keys, 0, count, [&](unsigned long long y) { return y > k; });
        if (before < n) take(k, before);
    }
}

__global__ void __launch_bounds__(THREADS) finish_kernel(Args a) {
    constexpr int KEEP = 4;  // tiles whose sums a thread keeps; it reads those of more tiles twice
    extern __shared__ unsigned long long smem[];
    const int room = max(a.n_v, a.n_top * a.tile);
    unsigned long long *found = smem, *left = smem + room;
    __shared__ float red[3][WARPS];
    __shared__ int chosen[64], n_found, n_left[3];
    __shared__ uint32_t floor_image, reached;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, m = blockIdx.x;
    const float4 *parts = a.parts + (size_t)m * a.n_v;
    const float *logits = a.logits + (size_t)m * a.ld;
    const float c = a.inv_t * LOG2E;
    // the given tokens are the caller's: their numbers can be read before the tiles are there
    const int tok = threadIdx.x < a.n_tok ? a.tokens[(size_t)m * a.n_tok + threadIdx.x] : -1;
    if (threadIdx.x == 0) n_found = n_left[0] = n_left[1] = n_left[2] = 0;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    __shared__ float4 sums[DIRECT_TILES];
    if (a.direct) {
        for (int t = warp; t < a.n_v; t += WARPS) {
            const float4 q = part_of_tile(logits + (size_t)t * a.tile, a.tile, c);
            if (lane == 0) sums[t] = q;
        }
        __syncthreads();
        parts = sums;
    }
    float4 p[KEEP];
#pragma unroll
    for (int j = 0; j < KEEP; j++) p[j] = threadIdx.x + j * THREADS < a.n_v ? parts[threadIdx.x + j * THREADS] : make_float4(-INFINITY, 0.0f, 0.0f, 0.0f);
    const float x_tok = (unsigned)tok < (unsigned)a.V ? logits[tok] : 0.0f;
    const bool gated = a.gate && a.n_top;  // the slots say what at least n_top tiles reach
    if (gated && warp == 0) {
        unsigned *slot = a.slots + (size_t)m * a.n_top + lane;
        const uint32_t low = warp_min_u32(lane < a.n_top ? *slot : ~0u);
        if (lane < a.n_top) *slot = 0u;
        if (lane == 0) reached = low;
    }

    float M = -INFINITY;
#pragma unroll
    for (int j = 0; j < KEEP; j++) {
        const int t = threadIdx.x + j * THREADS;
        M = max_nan(M, p[j].x);
        if (a.n_top && !gated && t < a.n_v) found[t] = key_of(p[j].x, t);
    }
    for (int t = threadIdx.x + KEEP * THREADS; t < a.n_v; t += THREADS) {
        const float x = parts[t].x;
        M = max_nan(M, x);
        if (a.n_top && !gated) found[t] = key_of(x, t);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) M = max_nan(M, __shfl_xor_sync(~0u, M, o));
    if (lane == 0) red[0][warp] = M;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WARPS; w++) M = max_nan(M, red[0][w]);
    const bool fine = M > -INFINITY && M < INFINITY;  // false for NaN
    const float nan = __int_as_float(0x7fffffff);
    const int n_tiles = min(a.n_top, a.n_v);
    auto choose = [&](unsigned long long k, int place) {
        chosen[place] = (int)~(uint32_t)k;
        // no alternative lies below the least of these tiles' largest (fewer tiles than alternatives: every entry counts)
        if (place == n_tiles - 1) floor_image = a.n_top <= a.n_v ? (uint32_t)(k >> 32) : 0u;
    };
    if (gated) {  // a few more than n_top tiles, as a rule
#pragma unroll
        for (int j = 0; j < KEEP; j++) {
            const int t = threadIdx.x + j * THREADS;
            if (t < a.n_v && ordered_image(p[j].x) >= reached) found[atomicAdd(n_left, 1)] = key_of(p[j].x, t);
        }
        for (int t = threadIdx.x + KEEP * THREADS; t < a.n_v; t += THREADS) {
            const float x = parts[t].x;
            if (ordered_image(x) >= reached) found[atomicAdd(n_left, 1)] = key_of(x, t);
        }
        __syncthreads();
        top_of(found, n_left[0], n_tiles, a.n_v, left, n_left + 1, choose);
    } else if (n_tiles) {
        top_of(found, a.n_v, n_tiles, a.n_v, left, n_left + 1, choose);
    }
    float S = 0.0f, T = 0.0f;
    auto add = [&](const float4 &q) {
        const float d = fmaxf((q.x - M) * c, -150.0f), w = ex2(d);
        S += w * q.y;
        T += w * (q.z + d * q.y);
    };
#pragma unroll
    for (int j = 0; j < KEEP; j++) add(p[j]);
    for (int t = threadIdx.x + KEEP * THREADS; t < a.n_v; t += THREADS) add(parts[t]);
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        S += __shfl_xor_sync(~0u, S, o);
        T += __shfl_xor_sync(~0u, T, o);
    }
    if (lane == 0) red[1][warp] = S, red[2][warp] = T;
    __syncthreads();
    for (int j = warp; j < n_tiles; j += WARPS) {
        const int v0 = chosen[j] * a.tile;
        float x[8];  // a tile has up to 256 entries
#pragma unroll
        for (int i = 0; i < 8; i++) x[i] = i * 32 + lane < a.tile ? logits[v0 + i * 32 + lane] : 0.0f;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const int v = v0 + i * 32 + lane;
            if (i * 32 + lane < a.tile && v < a.V && ordered_image(x[i]) >= floor_image) found[atomicAdd(&n_found, 1)] = key_of(x[i], v);
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
    auto put = [&](int place, int v, float lp) {
        a.top_id[(size_t)m * a.n_top + place] = v;
        if (a.top_logprob) a.top_logprob[(size_t)m * a.n_top + place] = lp;
    };
    if (n_found < a.n_top) {  // only a row with NaN runs out of candidates
        for (int j = threadIdx.x; j < a.n_top; j += THREADS) put(j, j, nan);
        return;
    }
    top_of(found, n_found, a.n_top, a.V, left, n_left + 2, [&](unsigned long long k, int place) { put(place, (int)~(uint32_t)k, logprob(key_value(k))); });
}

}  // namespace

cudaError_t prepare_finish() {
    cudaFuncAttributes fa;
    const cudaError_t e = cudaFuncGetAttributes(&fa, finish_kernel);
    if (e != cudaSuccess) return e;
    return cudaFuncSetAttribute(finish_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 232448 - (int)fa.sharedSizeBytes);
}

cudaError_t launch_finish(const Args &a, cudaStream_t s) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)a.rows);
    cfg.blockDim = dim3(THREADS);
    // keys of the tiles or of n_top tiles' entries, and those of them that are left
    const size_t room = a.n_v > a.n_top * a.tile ? a.n_v : a.n_top * a.tile;
    cfg.dynamicSmemBytes = a.n_top ? room * 16 : 0;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, finish_kernel, a);
}

}  // namespace score
}  // namespace aj
