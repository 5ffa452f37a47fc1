// Eviction from the cache by accumulated attention weight.
//
// Per (sequence, key head) with more than `keep` slots: keep the `keep` largest keys, where a key is the weight's
// order-preserving integer image (the largest integer for the protected first and newest tokens, zero for NaN),
// lower slots first among equals; then move the r-th kept slot past `keep` into the r-th dropped slot below it.
// Sources lie at or past `keep` and destinations below it, so the moves touch disjoint slots and need no order.
//
// A cluster of CTAs serves one (sequence, head): each selects for itself (a radix select of three digits over
// keys in shared memory reads 8 bytes per slot, from L2 but for the first) and then makes its share of the moves,
// which are what costs: 4 * D elements read or written per moved slot.  With few (sequence, head) pairs a
// larger cluster spreads them over the SMs.  Nothing is written before every CTA of the cluster has selected, so the
// state arrays may be updated in place.
#include "aj_kv.cuh"

namespace aj {
namespace kv {

namespace {

constexpr int LIST_MAX = 4096;         // moves a CTA lists at a time
constexpr int KEYS_MAX = 40 * 1024;    // slots whose keys fit in shared memory; longer ones re-read the weights
constexpr int BINS = 2048;             // digits of 11, 11 and 10 bits: the first one is a float's sign, exponent and two
                                       // bits of its fraction, so that weights of one magnitude do not queue up at one counter

struct Shared {
    unsigned hist[BINS];
    unsigned scan[33], scan2[33];
    int newest, need;
    unsigned prefix;
};

__device__ inline unsigned warp_sum(unsigned x) {
#pragma unroll
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(~0u, x, o);
    return x;
}

// Exclusive prefix over the warps of one value per warp; scan[NWARP] gets the total.
template <int NWARP> __device__ inline void scan_warps(unsigned *scan, unsigned mine) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (lane == 0) scan[warp] = mine;
    __syncthreads();
    if (warp == 0) {
        unsigned x = lane < NWARP ? scan[lane] : 0u, y = x;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned z = __shfl_up_sync(~0u, y, o);
            if (lane >= o) y += z;
        }
        if (lane < NWARP) scan[lane] = y - x;
        if (lane == 31) scan[NWARP] = y;
    }
    __syncthreads();
}

template <int THREADS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) evict_kernel(EvictArgs a, unsigned *counters, int n_split, int keys_cap, int LIST) {
    constexpr int NWARP = THREADS / 32;
    extern __shared__ __align__(16) unsigned dyn[];
    __shared__ Shared sh;
    const View &v = a.v;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int part = blockIdx.x % n_split, item = blockIdx.x / n_split;
    const int h = item % v.Hkv, b = item / v.Hkv;
    const int L = min(max(__ldg(v.lens + b), 0), v.cap), keep = a.keep;
    const size_t at = (size_t)item * v.cap;
    const float *w_in = a.weight + at;
    const int *p_in = a.slot_pos + at;

    // The new length is written once every CTA of this sequence has read the old one (they may be one array).
    __syncthreads();
    if (threadIdx.x == 0) {
        const unsigned total = (unsigned)v.Hkv * n_split;
        __threadfence();
        if (atomicInc(counters + b, total - 1) == total - 1) a.lens_out[b] = min(L, keep);
    }
    if (L <= keep) {  // the same for the whole cluster
        for (int j = part * THREADS + threadIdx.x; j < L; j += n_split * THREADS) {
            if (a.weight_out != a.weight) a.weight_out[at + j] = w_in[j];
            if (a.slot_pos_out != a.slot_pos) a.slot_pos_out[at + j] = p_in[j];
        }
        return;
    }

    const int n_words = (L + 31) >> 5;
    unsigned *list = dyn;                  // [2][LIST] holes, movers
    unsigned *kept = dyn + 2 * LIST;       // [ceil(cap / 32)] one bit per slot
    unsigned *keys = kept + ((v.cap + 31) >> 5);
    const bool cached = L <= keys_cap;

    if (threadIdx.x == 0) {
        sh.newest = -0x7fffffff - 1;
        sh.prefix = 0;
        sh.need = keep;
    }
    __syncthreads();
    auto weight_key = [&](float w) -> unsigned { return w != w ? 0u : ordered_image(w); };
    int newest = -0x7fffffff - 1;
#pragma unroll 8
    for (int j = threadIdx.x; j < L; j += THREADS) {
        newest = max(newest, __ldcg(p_in + j));
        if (cached) keys[j] = weight_key(__ldcg(w_in + j));
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) newest = max(newest, __shfl_xor_sync(~0u, newest, o));
    if (lane == 0) atomicMax(&sh.newest, newest);
    __syncthreads();
    const long long recent_from = (long long)sh.newest - a.recent;
    auto fixed = [&](int j) {
        const int p = __ldcg(p_in + j);
        return p < a.sinks || p > recent_from;
    };
    auto key_at = [&](int j) -> unsigned { return cached ? keys[j] : fixed(j) ? 0xffffffffu : weight_key(__ldcg(w_in + j)); };

    for (int digit = 0; digit < 3; digit++) {
        const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, bins = digit == 2 ? 1024 : 2048;
        for (int i = threadIdx.x; i < BINS; i += THREADS) sh.hist[i] = 0;
        __syncthreads();
        const unsigned prefix = sh.prefix, high = digit == 0 ? 0u : digit == 1 ? ~0u << 21 : ~0u << 10;
#pragma unroll 8
        for (int j = threadIdx.x; j < L; j += THREADS) {
            unsigned k;
            if (digit == 0 && cached) {  // the protected slots become known only now
                k = fixed(j) ? 0xffffffffu : keys[j];
                keys[j] = k;
            } else {
                k = key_at(j);
            }
            if (((k ^ prefix) & high) == 0) atomicAdd(&sh.hist[(k >> shift) & (bins - 1)], 1u);
        }
        __syncthreads();
        // thread i holds the PER digits from bins - 1 - PER * i down
        constexpr int PER = BINS / THREADS;
        const int d0 = bins - 1 - PER * (int)threadIdx.x;
        unsigned c[PER], mine = 0;
#pragma unroll
        for (int i = 0; i < PER; i++) mine += c[i] = d0 >= 0 ? sh.hist[d0 - i] : 0u;
        unsigned up = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned z = __shfl_up_sync(~0u, up, o);
            if (lane >= o) up += z;
        }
        scan_warps<NWARP>(sh.scan, __shfl_sync(~0u, up, 31));
        unsigned before = sh.scan[warp] + up - mine;
        const unsigned want = (unsigned)sh.need;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < PER; i++) {
            if (before < want && want <= before + c[i]) {
                sh.prefix = prefix | ((unsigned)(d0 - i) << shift);
                sh.need = (int)(want - before);
            }
            before += c[i];
        }
        __syncthreads();
    }
    const unsigned thr = sh.prefix, need = (unsigned)sh.need;

    // one bit per slot: kept.  A warp takes a run of words; among keys equal to the threshold the lowest slots stay
    const int run = (n_words + NWARP - 1) / NWARP;
    const int w0 = warp * run, w1 = min(n_words, w0 + run);
    unsigned eq = 0;
    for (int w = w0; w < w1; w++) {
        const int j = w * 32 + lane;
        const unsigned k = j < L ? key_at(j) : 0u;
        const unsigned gt = __ballot_sync(~0u, j < L && k > thr), e = __ballot_sync(~0u, j < L && k == thr);
        if (lane == 0) kept[w] = gt;
        eq += __popc(e);
    }
    scan_warps<NWARP>(sh.scan, eq);
    unsigned rank = sh.scan[warp];
    for (int w = w0; w < w1 && rank < need; w++) {
        const int j = w * 32 + lane;
        const unsigned k = j < L ? key_at(j) : 0u;
        const unsigned e = __ballot_sync(~0u, j < L && k == thr);
        const bool mine = (e >> lane & 1) && rank + __popc(e & ((1u << lane) - 1)) < need;
        const unsigned add = __ballot_sync(~0u, mine);
        if (lane == 0) kept[w] |= add;
        rank += __popc(e);
    }
    __syncthreads();

    auto below = [&](int w) -> unsigned {  // bits of word w whose slot lies below keep
        const int n = keep - w * 32;
        return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1;
    };
    auto valid = [&](int w) -> unsigned {
        const int n = L - w * 32;
        return n >= 32 ? ~0u : (1u << n) - 1;
    };
    unsigned holes = 0, movers = 0;
    for (int w = w0 + lane; w < w1; w += 32) {
        holes += __popc(~kept[w] & below(w));
        movers += __popc(kept[w] & ~below(w) & valid(w));
    }
    scan_warps<NWARP>(sh.scan, warp_sum(holes));
    scan_warps<NWARP>(sh.scan2, warp_sum(movers));
    const int n_moves = (int)sh.scan2[NWARP];  // as many holes as movers
    const int share = (n_moves + n_split - 1) / n_split;
    const int m0 = part * share, m1 = min(n_moves, m0 + share);

    // every CTA of the cluster is done reading the weights and positions
    if (n_split > 1) {
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
    if (a.weight_out != a.weight || a.slot_pos_out != a.slot_pos) {
        for (int j = part * THREADS + threadIdx.x; j < keep; j += n_split * THREADS) {
            if (kept[j >> 5] >> (j & 31) & 1) {
                if (a.weight_out != a.weight) a.weight_out[at + j] = __ldcg(w_in + j);
                if (a.slot_pos_out != a.slot_pos) a.slot_pos_out[at + j] = __ldcg(p_in + j);
            }
        }
    }
    const int n16 = v.D * a.elem / 16;  // 16-byte pieces of a row
    for (int c0 = m0; c0 < m1; c0 += LIST) {
        const int c1 = min(m1, c0 + LIST);
        unsigned hr = sh.scan[warp], mr = sh.scan2[warp];
        for (int w = w0; w < w1; w += 32) {  // 32 words at a time, one per lane
            const int wl = w + lane;
            unsigned hb = 0, mb = 0;
            if (wl < w1) {
                hb = ~kept[wl] & below(wl);
                mb = kept[wl] & ~below(wl) & valid(wl);
            }
            unsigned hs = __popc(hb), ms = __popc(mb);
            const unsigned hc = hs, mc = ms;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const unsigned x = __shfl_up_sync(~0u, hs, o), y = __shfl_up_sync(~0u, ms, o);
                if (lane >= o) {
                    hs += x;
                    ms += y;
                }
            }
            int r = (int)(hr + hs - hc);
            for (; hb; hb &= hb - 1, r++)
                if (r >= c0 && r < c1) list[r - c0] = wl * 32 + __ffs(hb) - 1;
            r = (int)(mr + ms - mc);
            for (; mb; mb &= mb - 1, r++)
                if (r >= c0 && r < c1) list[LIST + r - c0] = wl * 32 + __ffs(mb) - 1;
            hr += __shfl_sync(~0u, hs, 31);
            mr += __shfl_sync(~0u, ms, 31);
        }
        __syncthreads();
        for (int i = threadIdx.x; i < c1 - c0; i += THREADS) {
            const int dst = list[i], src = list[LIST + i];
            a.weight_out[at + dst] = __ldcg(w_in + src);
            a.slot_pos_out[at + dst] = __ldcg(p_in + src);
            const int page = __ldg(v.table + (size_t)b * v.width + (dst >> v.page_shift));
            // a page that is not in the pool is never written
            list[i] = (unsigned)page < (unsigned)v.n_pages ? (unsigned)((page * v.Hkv + h) * v.page + (dst & (v.page - 1))) : ~0u;
            list[LIST + i] = (unsigned)page_row(v, b, h, src);
        }
        __syncthreads();
        const int pieces = (c1 - c0) * n16;
#pragma unroll 4
        for (int i = threadIdx.x; i < pieces; i += THREADS) {
            const int r = i / n16, c = i - r * n16;
            const size_t from = (size_t)list[LIST + r] * n16 + c;
            const uint4 x = __ldcg((const uint4 *)a.k_pages + from), y = __ldcg((const uint4 *)a.v_pages + from);
            if (list[r] != ~0u) {
                const size_t to = (size_t)list[r] * n16 + c;
                ((uint4 *)a.k_pages)[to] = x;
                ((uint4 *)a.v_pages)[to] = y;
            }
        }
        __syncthreads();
    }
}

}  // namespace

cudaError_t prepare_evict() {
    const cudaError_t e = allow_shared(evict_kernel<512>);
    return e == cudaSuccess ? allow_shared(evict_kernel<1024>) : e;
}

cudaError_t launch_evict(const EvictArgs &a, unsigned *counters, int num_sms, cudaStream_t s) {
    const int items = a.v.B * a.v.Hkv;
    int n_split = 1;
    while (n_split < 8 && items * n_split * 2 <= num_sms) n_split *= 2;
    const int words = (a.v.cap + 31) / 32, keys = a.v.cap < KEYS_MAX ? a.v.cap : KEYS_MAX;
    const int most = a.v.cap / 2 + 1, list = most < LIST_MAX ? most : LIST_MAX;  // at most half of the slots move
    // the keys share what the bit map of a very long cache leaves
    const size_t fixed = (size_t)(2 * list + words) * 4;
    const size_t room = 212 * 1024 - fixed;
    const int keys_cap = (size_t)keys * 4 <= room ? keys : (int)(room / 4);
    const size_t smem = fixed + (size_t)keys_cap * 4;
    // more CTAs than SMs: two CTAs of half the threads share an SM, so that one's barriers hide behind the other
    const bool half = items * n_split > num_sms && smem <= 96 * 1024;
    auto kernel = half ? evict_kernel<512> : evict_kernel<1024>;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(items * n_split);
    cfg.blockDim = dim3(half ? 512 : 1024);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = n_split;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, a, counters, n_split, keys_cap, list);
}

}  // namespace kv
}  // namespace aj
