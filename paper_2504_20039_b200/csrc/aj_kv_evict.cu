// Eviction from the cache by accumulated attention weight.
//
// Per (sequence, key head) with more than `keep` slots: keep the `keep` largest keys, where a key is the weight's
// order-preserving integer image (the largest integer for the protected first and newest tokens, zero for NaN),
// lower slots first among equals; then move the r-th kept slot past `keep` into the r-th dropped slot below it.
// Sources lie at or past `keep` and destinations below it, so the moves touch disjoint slots and need no order.
//
// A cluster of CTAs serves one (sequence, head), each a run of its slots: with few pairs a larger cluster spreads
// them over the SMs.  The threshold comes from a radix select of four digits: every CTA counts its own slots in shared
// memory and adds up the counts of the cluster through distributed shared memory.  Ranks of dropped and kept slots follow
// from prefix sums over warps and CTAs, and each rank's slots are written into the list of the CTA that makes the move, so
// that the moves (4 * D elements read or written per moved slot, the bulk of the bytes) are shared evenly.
// It is the chain of barriers that bounds it, not the bytes.  Measured in the kernel, 16,384 slots of 8 heads cut to 4096,
// cluster of 8, cold: 5 us until the newest position is known, 2 us a digit (mostly three of the four), 1 + 1 us for the bits
// and their ranks, 2 us for the lists, 6 us for the moves (26 MB), 22 us in all.
// Nothing is written before the whole cluster has read the state, so the state arrays may be updated in place.
#include "aj_kv.cuh"
#include "aj_ptx.cuh"

namespace aj {
namespace kv {

namespace {

constexpr int LIST_MAX = 4096;         // moves a CTA lists at a time
constexpr int KEYS_MAX = 32 * 1024;    // slots of a CTA whose keys fit in shared memory; more re-read the weights
// Digits of 9, 8, 8 and 7 bits: the first one is a float's sign and exponent, spread enough that a warp's counts do not queue
// up at one counter; and adding up 512 counters of 8 CTAs costs less than a digit more (2048 counters: 6,000 cycles).
constexpr int DIGITS = 4, BINS = 512;
constexpr int MAX_CLUSTER = 8;

struct Shared {
    unsigned hist[DIGITS][BINS];
    unsigned scan[33], scan2[33];
    int newest, need, ties;
    unsigned prefix, eq, holes, movers;
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

// A word of another CTA's shared memory.
__device__ inline unsigned ld_cluster(const void *p, int rank) {
    unsigned x;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(x) : "r"(map_to_cta(smem_u32(p), rank)) : "memory");
    return x;
}

// AHEAD: 16-byte pieces of K and of V that a thread has in flight while rows move; eight where the CTA has an SM to itself
// (8 pairs of 16,384 slots: 31 us with four, 29 with eight).
template <int THREADS, int AHEAD>
__global__ void __launch_bounds__(THREADS, AHEAD == 4 ? 1024 / THREADS : 1) evict_kernel(EvictArgs a, unsigned *counters, int n_split, int keys_cap, int list_len) {
    constexpr int NWARP = THREADS / 32;
    extern __shared__ __align__(16) unsigned dyn[];
    __shared__ Shared sh;
    const CacheView &v = a.v;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int part = blockIdx.x % n_split, item = blockIdx.x / n_split;
    const int h = item % v.Hkv, b = item / v.Hkv;
    const int L = min(max(*(const volatile int *)(v.lens + b), 0), v.cap), keep = a.keep;
    const size_t at = (size_t)item * v.cap;
    const float *w_in = a.weight + at;
    const int *p_in = a.slot_pos + at;

    for (int i = threadIdx.x; i < DIGITS * BINS; i += THREADS) (&sh.hist[0][0])[i] = 0;
    if (threadIdx.x == 0) {
        sh.newest = -0x7fffffff - 1;
        sh.prefix = 0;
        sh.need = keep;
    }
    __syncthreads();
    // The new length is written once every CTA of this sequence has read the old one (they may be one array).  The count goes
    // out as soon as this CTA has, and comes back while the rows move (counted at the end: 2 us more).
    const unsigned last = (unsigned)v.Hkv * n_split - 1;
    unsigned others = 0;
    auto count_in = [&]() {
        if (threadIdx.x == 0) asm volatile("atom.acq_rel.gpu.global.inc.u32 %0, [%1], %2;" : "=r"(others) : "l"(counters + b), "r"(last) : "memory");
    };
    auto leave = [&]() {
        if (threadIdx.x == 0 && others == last) a.lens_out[b] = min(L, keep);
    };
    if (L <= keep) {  // the same for the whole cluster
        count_in();
        for (int j = part * THREADS + threadIdx.x; j < L; j += n_split * THREADS) {
            if (a.weight_out != a.weight) a.weight_out[at + j] = w_in[j];
            if (a.slot_pos_out != a.slot_pos) a.slot_pos_out[at + j] = p_in[j];
        }
        leave();
        return;
    }
    auto cluster_sync = [&]() {
        if (n_split > 1) cluster_sync_all();
        else __syncthreads();
    };

    // this CTA's slots: words w_lo .. w_hi - 1 of 32, slots j_lo .. j_hi - 1
    const int n_words = (L + 31) >> 5, per = (n_words + n_split - 1) / n_split;
    const int w_lo = min(n_words, part * per), w_hi = min(n_words, w_lo + per), j_lo = w_lo * 32, j_hi = min(L, w_hi * 32);
    unsigned *list = dyn;                      // [2][list_len] holes, movers
    unsigned *kept = dyn + 2 * list_len;       // one bit per slot of this CTA
    unsigned *keys = kept + (((v.cap + 31) >> 5) + n_split - 1) / n_split;
    const bool cached = j_hi - j_lo <= keys_cap;

    auto weight_key = [&](float w) -> unsigned { return w != w ? 0u : ordered_image(w); };
    int newest = -0x7fffffff - 1;
#pragma unroll 4
    for (int j = j_lo + threadIdx.x; j < j_hi; j += THREADS) {
        newest = max(newest, __ldcg(p_in + j));
        if (cached) keys[j - j_lo] = weight_key(__ldcg(w_in + j));
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) newest = max(newest, __shfl_xor_sync(~0u, newest, o));
    if (lane == 0) atomicMax(&sh.newest, newest);
    cluster_sync();
    newest = n_split == 1 ? sh.newest : lane < n_split ? (int)ld_cluster(&sh.newest, lane) : -0x7fffffff - 1;
#pragma unroll
    for (int o = 4; o; o >>= 1) newest = max(newest, __shfl_xor_sync(~0u, newest, o));
    newest = __shfl_sync(~0u, newest, 0);
    const long long recent_from = (long long)newest - a.recent;
    auto fixed = [&](int j) {
        const int p = __ldcg(p_in + j);
        return p < a.sinks || p > recent_from;
    };
    auto key_at = [&](int j) -> unsigned { return cached ? keys[j - j_lo] : fixed(j) ? 0xffffffffu : weight_key(__ldcg(w_in + j)); };

    for (int digit = 0; digit < DIGITS; digit++) {
        const int shift = digit == 0 ? 23 : digit == 1 ? 15 : digit == 2 ? 7 : 0, bins = digit == 0 ? 512 : digit == 3 ? 128 : 256;
        unsigned *hist = sh.hist[digit];
        const unsigned prefix = sh.prefix, high = digit == 0 ? 0u : ~0u << (shift + (digit == 3 ? 7 : 8)), want = (unsigned)sh.need;
#pragma unroll 4
        for (int j = j_lo + threadIdx.x; j < j_hi; j += THREADS) {
            unsigned k;
            if (digit == 0 && cached) {  // the protected slots become known only now
                k = fixed(j) ? 0xffffffffu : keys[j - j_lo];
                keys[j - j_lo] = k;
            } else {
                k = key_at(j);
            }
            if (((k ^ prefix) & high) == 0) atomicAdd(&hist[(k >> shift) & (bins - 1)], 1u);
        }
        cluster_sync();
        // thread i holds the digit bins - 1 - i, summed over the cluster
        const int d = bins - 1 - (int)threadIdx.x;
        unsigned mine = 0;
        if (d >= 0) {
            if (n_split == 1) {
                mine = hist[d];
            } else {
                unsigned x[MAX_CLUSTER];
#pragma unroll
                for (int r = 0; r < MAX_CLUSTER; r++) x[r] = r < n_split ? ld_cluster(hist + d, r) : 0u;
#pragma unroll
                for (int r = 0; r < MAX_CLUSTER; r++) mine += x[r];
            }
        }
        unsigned up = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned z = __shfl_up_sync(~0u, up, o);
            if (lane >= o) up += z;
        }
        scan_warps<NWARP>(sh.scan, __shfl_sync(~0u, up, 31));
        const unsigned before = sh.scan[warp] + up - mine;
        if (before < want && want <= before + mine) {
            sh.prefix = prefix | ((unsigned)d << shift);
            sh.need = (int)(want - before);
            sh.ties = mine != want - before;
        }
        __syncthreads();
        if (!sh.ties) break;  // the digit's slots all stay: the lower digits decide nothing (mostly after the third)
    }
    const unsigned thr = sh.prefix, need = (unsigned)sh.need;
    const bool ties = sh.ties;  // more slots than places have the threshold itself as their key

    // what the CTAs before this one, and all of them, hold of a counter
    auto across = [&](const unsigned *p, unsigned &all) {
        const unsigned x = n_split == 1 ? (lane == 0 ? *p : 0u) : lane < n_split ? ld_cluster(p, lane) : 0u;
        all = warp_sum(x);
        return warp_sum(lane < part ? x : 0u);
    };
    // one bit per slot: kept.  A warp takes a run of words; among keys equal to the threshold the lowest slots stay
    const int run = (w_hi - w_lo + NWARP - 1) / NWARP;
    const int w0 = min(w_hi, w_lo + warp * run), w1 = min(w_hi, w0 + run);
    unsigned eq = 0;
    for (int w = w0; w < w1; w++) {
        const int j = w * 32 + lane;
        const unsigned k = j < L ? key_at(j) : 0u;
        const unsigned gt = __ballot_sync(~0u, j < L && k > thr), e = __ballot_sync(~0u, j < L && k == thr);
        if (lane == 0) kept[w - w_lo] = ties ? gt : gt | e;
        eq += __popc(e);
    }
    if (ties) {
        scan_warps<NWARP>(sh.scan, eq);
        if (threadIdx.x == 0) sh.eq = sh.scan[NWARP];
        cluster_sync();
        unsigned all;
        unsigned rank = across(&sh.eq, all) + sh.scan[warp];
        for (int w = w0; w < w1 && rank < need; w++) {
            const int j = w * 32 + lane;
            const unsigned k = j < L ? key_at(j) : 0u;
            const unsigned e = __ballot_sync(~0u, j < L && k == thr);
            const bool mine = (e >> lane & 1) && rank + __popc(e & ((1u << lane) - 1)) < need;
            const unsigned add = __ballot_sync(~0u, mine);
            if (lane == 0) kept[w - w_lo] |= add;
            rank += __popc(e);
        }
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
        holes += __popc(~kept[w - w_lo] & below(w));
        movers += __popc(kept[w - w_lo] & ~below(w) & valid(w));
    }
    scan_warps<NWARP>(sh.scan, warp_sum(holes));
    scan_warps<NWARP>(sh.scan2, warp_sum(movers));
    if (threadIdx.x == 0) {
        sh.holes = sh.scan[NWARP];
        sh.movers = sh.scan2[NWARP];
    }
    cluster_sync();
    unsigned n_moves;  // as many holes as movers
    const unsigned hole0 = across(&sh.holes, n_moves) + sh.scan[warp], mover0 = across(&sh.movers, n_moves) + sh.scan2[warp];
    count_in();
    const int share = min(list_len, (int)(n_moves + n_split - 1) / n_split);  // moves a CTA makes at a time

    const int n16 = v.D * a.elem / 16;  // 16-byte pieces of a row
    const float per_share = 1.0f / (float)share;  // ranks stay below 8 * 4096: the quotient of r + 1/2 never rounds up to the next
    for (int c0 = 0; c0 < (int)n_moves; c0 += share * n_split) {
        // ranks c0 + k * share .. go to CTA k of the cluster
        unsigned hr = hole0, mr = mover0;
        auto put = [&](unsigned bits, unsigned &r0, int slot, unsigned *to) {  // one slot per lane
            const int r = (int)(r0 + __popc(bits & ((1u << lane) - 1))) - c0;
            if ((bits >> lane & 1) && r >= 0 && r < share * n_split) {
                const int k = (int)(((float)r + 0.5f) * per_share);
                if (n_split == 1) to[r] = slot;
                else st_shared_cluster_u32(map_to_cta(smem_u32(to + (r - k * share)), k), (unsigned)slot);
            }
            r0 += __popc(bits);
        };
        for (int w = w0; w < w1; w++) {
            const unsigned bits = kept[w - w_lo];
            put(~bits & below(w), hr, w * 32 + lane, list);
            put(bits & ~below(w) & valid(w), mr, w * 32 + lane, list + list_len);
        }
        cluster_sync();  // the lists are complete; and the whole cluster is done reading the state below keep
        const int count = max(0, min(share, (int)n_moves - c0 - part * share));
        for (int i = threadIdx.x; i < count; i += THREADS) {
            const int dst = list[i], src = list[list_len + i];
            const int page = __ldg(v.table + (size_t)b * v.width + (dst >> v.page_shift));
            const unsigned from = (unsigned)page_row(v, b, h, src);
            const float w = __ldcg(w_in + src);
            const int p = __ldcg(p_in + src);
            // a page that is not in the pool is never written
            list[i] = (unsigned)page < (unsigned)v.n_pages ? (unsigned)((page * v.Hkv + h) * v.page + (dst & (v.page - 1))) : ~0u;
            list[list_len + i] = from;
            a.weight_out[at + dst] = w;
            a.slot_pos_out[at + dst] = p;
        }
        __syncthreads();
        const int pieces = count * n16;
        for (int i0 = threadIdx.x; i0 < pieces; i0 += AHEAD * THREADS) {
            uint4 x[AHEAD], y[AHEAD];
            size_t to[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; u++) {
                const int i = i0 + u * THREADS, r = i / n16, c = i - r * n16;
                to[u] = ~(size_t)0;
                if (i < pieces && list[r] != ~0u) {
                    const size_t from = (size_t)list[list_len + r] * n16 + c;
                    to[u] = (size_t)list[r] * n16 + c;
                    x[u] = __ldcg((const uint4 *)a.k_pages + from);
                    y[u] = __ldcg((const uint4 *)a.v_pages + from);
                }
            }
#pragma unroll
            for (int u = 0; u < AHEAD; u++)
                if (to[u] != ~(size_t)0) {
                    ((uint4 *)a.k_pages)[to[u]] = x[u];
                    ((uint4 *)a.v_pages)[to[u]] = y[u];
                }
        }
        if (c0 + share * n_split < (int)n_moves) cluster_sync();  // the lists are free again
    }
    // slots that stay where they are
    if (a.weight_out != a.weight || a.slot_pos_out != a.slot_pos) {
        const int end = min(j_hi, keep);
        for (int j0 = j_lo + threadIdx.x; j0 < end; j0 += 4 * THREADS) {
            float w[4];
            int p[4];
            bool on[4];
#pragma unroll
            for (int u = 0; u < 4; u++) {
                const int j = j0 + u * THREADS;
                on[u] = j < end && (kept[(j >> 5) - w_lo] >> (j & 31) & 1);
                if (on[u]) w[u] = __ldcg(w_in + j), p[u] = __ldcg(p_in + j);
            }
#pragma unroll
            for (int u = 0; u < 4; u++) {
                const size_t to = at + j0 + u * THREADS;
                if (on[u] && a.weight_out != a.weight) a.weight_out[to] = w[u];
                if (on[u] && a.slot_pos_out != a.slot_pos) a.slot_pos_out[to] = p[u];
            }
        }
    }
    if (n_moves == 0) cluster_sync();  // no CTA leaves while another may still read its counters
    leave();
}

}  // namespace

// clusters[i]: how many clusters of 2^i CTAs of 1024 threads the device holds at once (a cluster stays within one GPC).
cudaError_t prepare_evict(int (&clusters)[4]) {
    cudaError_t e = allow_shared(evict_kernel<512, 4>);
    if (e == cudaSuccess) e = allow_shared(evict_kernel<512, 8>);
    if (e == cudaSuccess) e = allow_shared(evict_kernel<1024, 4>);
    for (int i = 0; i < 4 && e == cudaSuccess; i++) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(1 << i);
        cfg.blockDim = dim3(1024);
        cfg.dynamicSmemBytes = 96 * 1024;
        cudaLaunchAttribute attr;
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = 1 << i;
        attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
        e = cudaOccupancyMaxActiveClusters(&clusters[i], evict_kernel<1024, 4>, &cfg);
    }
    return e;
}

cudaError_t launch_evict(const EvictArgs &a, unsigned *counters, const int (&clusters)[4], int num_sms, cudaStream_t s) {
    const int items = a.v.B * a.v.Hkv;
    // as many CTAs per pair as run at once (8 pairs of 16,384 slots: 76 us alone, 29 in clusters of 8), but no fewer than 1024
    // slots for a CTA: the barriers of a cluster cost more than the slots that it takes off a CTA's hands (16 pairs of 300
    // slots: 34 us in clusters of 8, 12 alone)
    int log_split = 0;
    while (log_split < 3 && items <= clusters[log_split + 1] && (1024 << log_split) < a.v.cap) log_split++;
    const int n_split = 1 << log_split;
    const int cap = (((a.v.cap + 31) / 32) + n_split - 1) / n_split * 32;  // slots of a CTA
    const int keys_want = cap < KEYS_MAX ? cap : KEYS_MAX;
    const int most = (a.v.cap / 2 + n_split) / n_split, list = most < LIST_MAX ? most : LIST_MAX;  // at most half of the slots move
    // the keys share what the bit map of a very long cache leaves
    const size_t fixed = (size_t)(2 * list + cap / 32) * 4;
    const size_t room = 196 * 1024 - fixed;
    const int keys_cap = (size_t)keys_want * 4 <= room ? keys_want : (int)(room / 4);
    const size_t smem = fixed + (size_t)keys_cap * 4;
    // Half the threads where there is little to do for each, so that barriers are cheaper, and where there are more CTAs than
    // SMs: two then share an SM, and one's barriers hide behind the other (256 pairs of 2,100 slots: 23 us, with all threads
    // 33; 16 pairs: 16 and 18).
    const bool half = smem <= 80 * 1024 && (items * n_split > num_sms || cap <= 2048);
    auto kernel = !half ? evict_kernel<1024, 4> : items * n_split > num_sms ? evict_kernel<512, 4> : evict_kernel<512, 8>;
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
    cfg.numAttrs = n_split > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, a, counters, n_split, keys_cap, list);
}

}  // namespace kv
}  // namespace aj
