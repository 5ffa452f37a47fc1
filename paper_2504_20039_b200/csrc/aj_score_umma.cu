// aj_score_tokens, first step, on tcgen05: logits[m, v] = sum_k h[m, k] W[v, k], and of each tile of entries the largest
// logit, S = sum 2^d and T = sum d 2^d with d = (logit - largest) * inv_temperature * log2(e).
//
// Rows of hidden states lie along the UMMA M axis (TMEM lanes), entries along N (TMEM columns): a thread of the epilogue owns one
// row, and a tile's maximum and sums need no other thread.
//   up to 128 rows   one SM per tile of 128 rows x up to 256 entries.  Bound by the stream of W; the tile's width (one_sm_tile)
//                    weighs the balance over the SMs against what a tile costs.  Only the rows that exist are staged (rounded up to 8): the MMA reads 128
//                    rows from there on, and what the others hold reaches no lane that is looked at.
//   more             two SMs (cta_group::2) per tile of 256 rows x 256 entries: each stages its own 128 rows and half of the
//                    entries.  Bound by the tensor pipe (an MMA of N = 256 takes 128 cycles and holds its issuing thread as long).
//
//   warp 0      TMA: 128-byte wide boxes of h and W (128-byte swizzle) into a ring of stages, one 128-byte k-block each
//   warp 1      issues tcgen05.mma into one of two accumulators of 256 columns
//   warps 2-5   epilogue: maximum, exponentials and the logits' store, while the other accumulator fills
//
// bf16 and e4m3 differ in the instruction and in the scales that the epilogue puts on the sums (times h_scale, times w_scale).
// Every logit is one sum over k in a fixed order.  Every wait is bounded (aj_ptx.cuh).
//
// Measured (d = 4096, 128,256 entries, the whole call from a graph): 17 rows 165 to 170 us for 1.05 GB, 6.2 to 6.4 TB/s; in 8 bits 89 to 92 us,
// 5.7 to 5.9 TB/s; 2112 rows 1410 us alone, 1.57 PFLOP/s, and 1490 to 1550 back to back, where the power limit lowers the clock (on zeros 1182); 2048
// rows in 8 bits 783 us. 129 to 256 rows are bound by W too (200 rows 213 us, in 8 bits 122); 264 rows take nine tenths of what 512 take (350 to
// 370 and 404 us; in 8 bits 206 and 229), for whole row tiles are multiplied.
#include "aj_score.cuh"
#include "aj_ptx.cuh"

namespace aj {
namespace score {

namespace {

constexpr int THREADS = 192;
constexpr int SMEM = 232448, RING = 224 * 1024, MAX_STAGES = 32;
constexpr int BARS = 2 * MAX_STAGES + 4;

template <bool PAIR> __device__ inline void umma_e4m3(uint32_t d, unsigned long long a, unsigned long long b, uint32_t idesc, uint32_t acc) {
    if constexpr (PAIR)
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc)
            : "memory");
}
// e4m3 x e4m3 -> f32, both operands K-major
__device__ constexpr uint32_t instr_desc_e4m3(int m, int n) { return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24); }

__device__ inline void store8(float *p, const float *x) {
    asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]),
                 "f"(x[7])
                 : "memory");
}

template <bool PAIR, bool EIGHT>
__global__ void __launch_bounds__(THREADS, 1)
score_umma_kernel(const __grid_constant__ CUtensorMap tmap_h, const __grid_constant__ CUtensorMap tmap_w, Args a, Plan p) {
    extern __shared__ __align__(1024) uint8_t smem[];  // swizzled tiles need 1024-byte alignment
    const uint32_t base = smem_u32(smem), bars = base + RING;
    auto full = [&](int s) { return bars + 8u * s; };
    auto empty = [&](int s) { return bars + 8u * (MAX_STAGES + s); };
    auto acc_full = [&](int b) { return bars + 8u * (2 * MAX_STAGES + b); };
    auto acc_empty = [&](int b) { return bars + 8u * (2 * MAX_STAGES + 2 + b); };
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(smem + RING + 8 * BARS);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);

    const int warp = __shfl_sync(~0u, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const uint32_t rank = PAIR ? cluster_ctarank() : 0;  // 0: leader
    const int unit = PAIR ? blockIdx.x >> 1 : blockIdx.x, units = PAIR ? gridDim.x >> 1 : gridDim.x;
    constexpr int ROWS = PAIR ? 256 : 128;
    const int n_tiles = p.n_m * p.n_v, tile = p.tile, tile_cta = PAIR ? tile >> 1 : tile;
    const int stages = p.stages, kps = p.kps;
    const uint32_t a_bytes = (uint32_t)p.box_rows * 128u, sub_bytes = a_bytes + (uint32_t)tile_cta * 128u, stage_bytes = kps * sub_bytes;

    if (threadIdx.x == 0) {
        for (int s = 0; s < stages; s++) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), 1);
        }
        for (int b = 0; b < 2; b++) {
            mbar_init(acc_full(b), 1);
            mbar_init(acc_empty(b), PAIR ? 8 : 4);  // the warps that drain it, in both CTAs
        }
        *abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == 1) {
        if (PAIR)
            tmem_alloc_pair(smem_u32(const_cast<uint32_t *>(tmem_slot)), 512);
        else
            tmem_alloc(smem_u32(const_cast<uint32_t *>(tmem_slot)), 512);
    }
    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_sync_all();  // the peer's barriers exist before anything is sent to them
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    // Programmatic dependent launch: nothing of the caller's or the workspace is touched before this wait returns.
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    auto give_up = [&]() {
        *abort_flag = 1;
        atomicCAS(a.status, DEV_OK, DEV_TIMEOUT);
    };

    if (warp == 0) {
        if (lane == 0) {
            // ---------------------------------------------------------------- TMA
            const unsigned long long pol_h = policy_evict_last(), pol_w = p.n_m == 1 ? policy_evict_first() : policy_evict_normal();
            constexpr int BK = EIGHT ? 128 : 64;
            int s = 0;
            uint32_t ph = 0;
            bool ok = true;
            for (int t = unit; ok && t < n_tiles; t += units) {
                const int v_tile = t / p.n_m, m_tile = t - v_tile * p.n_m;
                const int row = m_tile * ROWS + (int)rank * 128, v = v_tile * tile + (int)rank * tile_cta;
                for (int kb = 0; kb < p.num_kb; kb += kps) {
                    if (!mbar_wait(empty(s), ph ^ 1u, abort_flag)) {
                        give_up();
                        ok = false;
                        break;
                    }
                    const uint32_t bar = PAIR ? map_to_cta(full(s), 0) : full(s);
                    if (rank == 0) mbar_expect_tx(full(s), (PAIR ? 2u : 1u) * stage_bytes);
                    for (int j = 0; j < kps; j++) {
                        const uint32_t dst = base + s * stage_bytes + j * sub_bytes;
                        const int kc = (kb + j) * BK;
                        if (PAIR) {
                            tma_load_2d_pair(dst + a_bytes, &tmap_w, kc, v, bar, pol_w);
                            tma_load_2d_pair(dst, &tmap_h, kc, row, bar, pol_h);
                        } else {
                            tma_load_2d(dst + a_bytes, &tmap_w, kc, v, bar, pol_w);
                            tma_load_2d(dst, &tmap_h, kc, row, bar, pol_h);
                        }
                    }
                    if (++s == stages) {
                        s = 0;
                        ph ^= 1u;
                    }
                }
            }
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            // ---------------------------------------------------------------- MMA
            const uint32_t idesc = EIGHT ? instr_desc_e4m3(ROWS, tile) : instr_desc(ROWS, tile);
            int s = 0, it = 0;
            uint32_t ph = 0;
            bool ok = true, ready = false;
            for (int t = unit; ok && t < n_tiles; t += units, ++it) {
                const int b = it & 1;
                if (!mbar_wait(acc_empty(b), ((uint32_t)(it >> 1) & 1u) ^ 1u, abort_flag)) {
                    give_up();
                    break;
                }
                tc_fence_after();
                const uint32_t d = tmem + (uint32_t)(b * 256);
                for (int kb = 0; kb < p.num_kb; kb += kps) {
                    if (!ready && !mbar_wait(full(s), ph, abort_flag)) {
                        give_up();
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const int s_next = s + 1 == stages ? 0 : s + 1;
                    const uint32_t ph_next = s + 1 == stages ? ph ^ 1u : ph;
                    for (int j = 0; j < kps; j++) {
                        const uint32_t at = base + s * stage_bytes + j * sub_bytes;
                        const unsigned long long ad = smem_desc_sw128(at), bd = smem_desc_sw128(at + a_bytes);
#pragma unroll
                        for (int k = 0; k < 4; k++) {
                            const uint32_t acc = (uint32_t)((kb | j | k) != 0);
                            if constexpr (EIGHT)
                                umma_e4m3<PAIR>(d, ad + 2ull * k, bd + 2ull * k, idesc, acc);
                            else if constexpr (PAIR)
                                umma_bf16_pair(d, ad + 2ull * k, bd + 2ull * k, idesc, acc);
                            else
                                umma_bf16(d, ad + 2ull * k, bd + 2ull * k, idesc, acc);
                            // the next stage is looked at while this one's MMAs run, not after them
                            if (k == 2 && j + 1 == kps) ready = mbar_test(full(s_next), ph_next);
                        }
                    }
                    if (PAIR)
                        umma_commit_pair(empty(s));
                    else
                        umma_commit(empty(s));
                    s = s_next;
                    ph = ph_next;
                }
                if (ok) {
                    if (PAIR)
                        umma_commit_pair(acc_full(b));
                    else
                        umma_commit(acc_full(b));
                }
            }
        }
    } else {
        // -------------------------------------------------------------------- epilogue: thread = row
        const int q = warp & 3;  // the quadrant of lanes that this warp reads
        const float c = a.inv_t * LOG2E;
        int it = 0;
        for (int t = unit; t < n_tiles; t += units, ++it) {
            const int v_tile = t / p.n_m, m_tile = t - v_tile * p.n_m;
            const int row0 = m_tile * ROWS + (int)rank * 128 + q * 32, row = row0 + lane, b = it & 1;
            const bool valid = row < a.rows;
            const int v0 = v_tile * tile;
            const float sh = EIGHT && valid ? __ldg(a.h_scale + row) : 1.0f;
            // asked before the accumulator is ready; an old slot is only lower, and then a tile is stored that need not be
            uint32_t least = 0;
            bool asked = false;
            if (a.gate) {
                least = ~0u;
                if (valid) {
                    for (int i = 0; i < a.n_top; i++) least = min(least, __ldcg(a.slots + (size_t)row * a.n_top + i));
                    for (int i = 0; i < a.n_tok; i++) asked |= (unsigned)(__ldg(a.tokens + (size_t)row * a.n_tok + i) - v0) < (unsigned)tile;
                }
            }
            // the whole warp takes one decision, so the aligned TMEM loads below stay converged
            if (!__all_sync(~0u, mbar_wait(acc_full(b), (uint32_t)(it >> 1) & 1u, abort_flag))) {
                give_up();
                break;
            }
            tc_fence_after();
            if (row0 < a.rows) {
                const uint32_t acc = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(b * 256);
                // 32 logits of the row; entries past V are -infinity
                auto load = [&](int j, float (&x)[32]) {
                    tmem_ld32(acc + j, x);
                    const int v = v0 + j;
                    if (v + 32 <= a.V) {
                        if (EIGHT) {
#pragma unroll
                            for (int i = 0; i < 32; i += 4) {
                                const float4 w = __ldg(reinterpret_cast<const float4 *>(a.w_scale + v + i));
                                x[i] = x[i] * sh * w.x, x[i + 1] = x[i + 1] * sh * w.y, x[i + 2] = x[i + 2] * sh * w.z, x[i + 3] = x[i + 3] * sh * w.w;
                            }
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; i++) {
                            if (v + i >= a.V)
                                x[i] = -INFINITY;
                            else if (EIGHT)
                                x[i] = x[i] * sh * __ldg(a.w_scale + v + i);
                        }
                    }
                };
                // One pass: S and T relative to the largest logit so far, which a chunk may raise.
                float mx = -INFINITY, S = 0.0f, T = 0.0f;
#pragma unroll 1
                for (int j = 0; j < tile; j += 32) {
                    float x[32];
                    load(j, x);
                    float m4[4] = {mx, mx, mx, mx};
#pragma unroll
                    for (int i = 0; i < 32; i += 8)
#pragma unroll
                        for (int k = 0; k < 4; k++) m4[k] = max3_nan(m4[k], x[i + k], x[i + 4 + k]);
                    const float top = max3_nan(max3_nan(m4[0], m4[1], m4[2]), m4[3], m4[3]);
                    // (all of them -infinity: nothing to raise, the differences are NaN and count as -150)
                    const float up = fmaxf((mx - top) * c, -150.0f), w = ex2(up);
                    T = w * (T + up * S);
                    S *= w;
                    mx = top;
                    float s4[4] = {}, t4[4] = {};
#pragma unroll
                    for (int i = 0; i < 32; i++) {
                        const float d = fmaxf((x[i] - top) * c, -150.0f), e = ex2(d);  // 2^-150 is zero, and so is d 2^d
                        s4[i & 3] += e;
                        t4[i & 3] += d * e;
                    }
                    S += (s4[0] + s4[1]) + (s4[2] + s4[3]);
                    T += (t4[0] + t4[1]) + (t4[2] + t4[3]);
                }
                const bool store = valid && (!a.gate || asked || (a.n_top && ordered_image(mx) >= least));
                if (a.gate && a.n_top && store) atomicMax(a.slots + (size_t)row * a.n_top + v_tile % a.n_top, ordered_image(mx));
                if (__any_sync(~0u, store)) {
                    float *to = a.logits + (size_t)row * a.ld + v0;
#pragma unroll 1
                    for (int j = 0; j < tile; j += 32) {
                        float x[32];
                        load(j, x);
                        if (store) {
#pragma unroll
                            for (int i = 0; i < 32; i += 8) store8(to + j + i, x + i);
                        }
                        __syncwarp();
                    }
                }
                if (valid) a.parts[(size_t)row * p.n_v + v_tile] = make_float4(mx, S, T, 0.0f);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (PAIR)
                    mbar_arrive_cluster(map_to_cta(acc_empty(b), 0));
                else
                    mbar_arrive(acc_empty(b));
            }
        }
    }

    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 1 && *abort_flag) {
        // copies or MMAs may still be in flight after an abort: give them time to land
        const unsigned long long t0 = globaltimer_ns();
        while (globaltimer_ns() - t0 < 200000ull) __nanosleep(1000);
    }
    if (PAIR) cluster_sync_all();  // neither CTA leaves, or frees tensor memory, while the other may still signal it
    if (warp == 1) {
        tc_fence_after();
        if (PAIR)
            tmem_dealloc_pair(tmem, 512);
        else
            tmem_dealloc(tmem, 512);
    }
}

template <bool PAIR, bool EIGHT> cudaError_t launch(const CUtensorMap &mh, const CUtensorMap &mw, const Args &a, const Plan &p, cudaStream_t s) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)p.grid);
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = SMEM;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 2;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = PAIR ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, score_umma_kernel<PAIR, EIGHT>, mh, mw, a, p);
}

template <bool PAIR, bool EIGHT> cudaError_t allow() {
    return cudaFuncSetAttribute(score_umma_kernel<PAIR, EIGHT>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM);
}

}  // namespace

cudaError_t prepare_umma(int num_sms, int *max_pairs) {
    cudaError_t e = allow<false, false>();
    if (e == cudaSuccess) e = allow<false, true>();
    if (e == cudaSuccess) e = allow<true, false>();
    if (e == cudaSuccess) e = allow<true, true>();
    if (e != cudaSuccess) return e;
    // pairs that can run at once (a pair needs both SMs of a pair free)
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(num_sms & ~1));
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = SMEM;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int clusters = 0;
    e = cudaOccupancyMaxActiveClusters(&clusters, score_umma_kernel<true, true>, &cfg);
    if (e != cudaSuccess) return e;
    if (clusters < 1) return cudaErrorInvalidConfiguration;
    *max_pairs = clusters < num_sms / 2 ? clusters : num_sms / 2;
    return cudaSuccess;
}

// Entries per tile of the one-SM kernel: the multiple of 32 with the least (tiles in turn on an SM) x (entries + 64), the narrowest of
// equals.  A tile streams its entries, and has its rows staged again, an epilogue, and latencies that a narrow one cannot hide: at
// d = 4096 in bf16 tiles of 32, 64 and 96 entries take 17 to 18 us each on 148 SMs, 128 take 24, 224 take 40.  Measured over heads of 3,000 to
// 1,000,000 entries, d from 256 to 8192, 1 to 128 rows, both types, every width: the choice is within 6 % of the best one, 0.5 % on
// average, and so for any constant from 40 to 96.  50,257 entries, 17 rows: 192 (chosen) 72 us, 96 78, 32 188; 200,064: 256 (chosen) 251,
// 192 253, 32 778; 128,256: 224 (chosen) 164, 96 184; 12,000: 96 (chosen) 27.3, 224 31.4, 64 43.
int one_sm_tile(int V, int num_sms) {
    int best = 256;
    long long least = 0;
    for (int t = 32; t <= 256; t += 32) {
        const int n = (V + t - 1) / t;
        if (n > MAX_TILES) continue;
        const long long cost = (long long)((n + num_sms - 1) / num_sms) * (t + 64);
        if (least == 0 || cost < least) {
            least = cost;
            best = t;
        }
    }
    return best;
}

Plan plan_umma(int rows, int d, int V, int dtype, int tile, int num_sms, int max_pairs) {
    Plan p;
    p.pair = rows > 128;
    p.tile = p.pair ? 256 : tile;
    p.n_v = (V + p.tile - 1) / p.tile;
    p.n_m = p.pair ? (rows + 255) / 256 : 1;
    p.box_rows = p.pair ? 128 : (rows + 7) & ~7;
    p.num_kb = (int)(((long long)d * (dtype == E4M3 ? 1 : 2) + 127) / 128);
    // two k-blocks per stage, so that the issuing thread tests and commits half as often (2048 rows 1515 -> 1350 us, 17 rows 169 -> 166),
    // where three such stages fit
    const int sub = (p.box_rows + (p.pair ? 128 : p.tile)) * 128;
    p.kps = p.num_kb % 2 == 0 && RING / (2 * sub) >= 3 ? 2 : 1;
    const int stage = sub * p.kps;
    // the MMA reads 128 rows (16 KB) from a k-block's rows on, of which box_rows are staged: past the k-block where it is smaller, so
    // the last k-block of the last stage begins no later than 16 KB before the end of the block's shared memory
    const int latest = (SMEM - 16384 - (p.kps - 1) * sub) / stage + 1;
    p.stages = RING / stage < latest ? RING / stage : latest;
    if (p.stages > MAX_STAGES) p.stages = MAX_STAGES;
    const int n = p.n_m * p.n_v;
    p.grid = p.pair ? 2 * (n < max_pairs ? n : max_pairs) : (n < num_sms ? n : num_sms);
    return p;
}

cudaError_t launch_umma(const CUtensorMap &mh, const CUtensorMap &mw, const Args &a, const Plan &p, cudaStream_t s) {
    if (a.dtype == E4M3) return p.pair ? launch<true, true>(mh, mw, a, p, s) : launch<false, true>(mh, mw, a, p, s);
    return p.pair ? launch<true, false>(mh, mw, a, p, s) : launch<false, false>(mh, mw, a, p, s);
}

}  // namespace score
}  // namespace aj
