// aj_kv_weigh for many query rows per key head (verified windows, prompts), bf16 and head sizes 64 and 128, on tcgen05.
//
//   S^T = K Q^T   128 slots x up to 256 rows, f32 in tensor memory;   weight_out[j] += sum over columns of exp2(S - lse)
//
// Slots lie on the 128 lanes and query rows on the columns, so that one thread owns one slot and adds up its columns: no
// exchange between lanes, no join between CTAs.  Roles: warps 0-3 and 4-7 add up the columns of every other block of
// 128 slots (accumulators of 256 columns, two of them), warp 8 issues the products, warp 9 brings the blocks of K in
// by TMA.  The queries of a (sequence, key head) lie in shared memory as the second operand, 256 rows at a time;
// more rows (a prompt) walk over the CTA's blocks again, which then come from L2.
//
// Bound: K from HBM up to about 170 rows (32 KB per block against 128 x rows exponentials at 16 per clock and SM), the
// exponentials above.  The line of blocks is cut as in the small kernel.  Measured: 8 sequences of 1000 .. 8192 slots, windows
// of 33 rows x 4 heads of which 1 to 33 count, 88 MB: 25 to 43 us back to back, 34 in the mean of ten draws of the counts; where it
// takes 30, 5 go by before the first products, 3 for each further (sequence, head) of a CTA, and the blocks between them pass
// at 4.4 TB/s.  A prompt of 4096, 3465 rows of it counted: 407 us, with 192 M exponentials, 43 us of their unit.
// Every wait is bounded (aj_ptx.cuh).
#include "aj_kv.cuh"
#include "aj_kv_tc.cuh"
#include "aj_ptx.cuh"

namespace aj {
namespace kv {

namespace {

constexpr int BLK = 128, ROWS = 256, THREADS = 320;

template <bool X> struct Const {
    static constexpr bool value = X;
};

template <int D> struct Cfg {
    static constexpr int TILE = BLK * D * 2, QB = ROWS * D * 2;
    static constexpr int STAGES = D == 128 ? 4 : 8;
    static constexpr int BARS = 2 * STAGES + 6;
    static constexpr int NEG_AT = QB + STAGES * TILE + BARS * 8 + 16;  // per row: -lse * log2(e); then its slot
    static constexpr int PRE_AT = NEG_AT + 2 * ROWS * 4;
    static constexpr int smem(int B) { return PRE_AT + (B + 1) * 8; }
    static_assert(PRE_AT + (4096 + 1) * 8 <= 232448, "the largest batch of a handle fits");
};

struct Seg {                      // the CTA's blocks of one (sequence, key head)
    int b, h, blk, n, units, w;   // first block, blocks, blocks of the sequence, cost of a block
    long long at;                 // place on the line of block `blk`
    Seq s;
    int counted;                  // rows that count
};

template <int D>
__global__ void __launch_bounds__(THREADS, 1) weigh_umma_kernel(const __grid_constant__ CUtensorMap tmap_k, WeighArgs a) {
    using C = Cfg<D>;
    constexpr int NS = C::STAGES, HALVES = D / 64;
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t base = smem_u32(smem), ring = base + C::QB, bars = ring + NS * C::TILE;
    auto full = [&](int s) { return bars + 8u * s; };
    auto empty = [&](int s) { return bars + 8u * (NS + s); };
    auto acc_full = [&](int x) { return bars + 8u * (2 * NS + x); };
    auto acc_empty = [&](int x) { return bars + 8u * (2 * NS + 2 + x); };
    const uint32_t q_ready = bars + 8u * (2 * NS + 4), drained = bars + 8u * (2 * NS + 5);
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(smem + C::QB + NS * C::TILE + C::BARS * 8);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
    float *neg = reinterpret_cast<float *>(smem + C::NEG_AT);
    int *row_slot = reinterpret_cast<int *>(neg + ROWS);
    long long *pre = reinterpret_cast<long long *>(smem + C::PRE_AT);  // [B + 1]
    const CacheView &v = a.v;
    const int warp = __shfl_sync(~0u, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int s = 0; s < NS; s++) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), 1);
        }
        for (int x = 0; x < 2; x++) {
            mbar_init(acc_full(x), 1);
            mbar_init(acc_empty(x), 128);
        }
        mbar_init(q_ready, 256);
        mbar_init(drained, 1);
        *abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == 8) tmem_alloc(smem_u32(const_cast<uint32_t *>(tmem_slot)), 512);

    auto enter = [&](Seg &c, int b) {
        c.b = b;
        c.s = seq_of(v, b);
        c.counted = min(c.s.nq, a.n_rows ? max(__ldg(a.n_rows + b), 0) : c.s.nq) * v.G;
        c.units = (c.s.L + BLK - 1) / BLK;
        c.w = 4 + (c.counted + 7) / 8;
    };
    for (int b = threadIdx.x; b < v.B; b += THREADS) {
        Seg c;
        enter(c, b);
        pre[b + 1] = (long long)c.units * v.Hkv * c.w;
    }
    if (threadIdx.x == 0) pre[0] = 0;
    __syncthreads();
    if (warp == 0) {
        long long carry = 0;
        for (int b0 = 1; b0 <= v.B; b0 += 32) {
            long long x = b0 + lane <= v.B ? pre[b0 + lane] : 0;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long y = __shfl_up_sync(~0u, x, o);
                if (lane >= o) x += y;
            }
            if (b0 + lane <= v.B) pre[b0 + lane] = carry + x;
            carry += __shfl_sync(~0u, x, 31);
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    const long long total = pre[v.B], per = (total + gridDim.x - 1) / gridDim.x;
    const long long from = per * blockIdx.x, to = min(total, from + per);
    auto give_up = [&]() {
        *abort_flag = 1;
        atomicCAS(a.status, DEV_OK, DEV_TIMEOUT);
    };

    // the segments of this CTA, in the same order for every role
    auto fit = [&](Seg &c) {  // blocks of this (sequence, head) that begin before `to`
        c.n = c.at < to ? (int)min((long long)(c.units - c.blk), (to - c.at + c.w - 1) / c.w) : 0;
    };
    auto settle = [&](Seg &c) {
        if (c.h < v.Hkv) return;
        int b = c.b + 1;
        while (b < v.B && pre[b] == pre[b + 1]) b++;
        c.at = total;
        if (b >= v.B) return;
        c.at = pre[b];
        c.h = c.blk = 0;
        enter(c, b);
    };
    auto first_seg = [&]() {
        Seg c;
        int lo = 0, hi = v.B;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (pre[mid] <= from) lo = mid; else hi = mid;
        }
        enter(c, lo);
        const int k = (int)((from - pre[lo] + c.w - 1) / c.w);
        c.h = k / c.units;
        c.blk = k - c.h * c.units;
        c.at = pre[lo] + (long long)k * c.w;
        settle(c);
        fit(c);
        return c;
    };
    auto next_seg = [&](Seg &c) {
        c.at += (long long)c.n * c.w;
        c.blk += c.n;
        if (c.blk == c.units) {
            c.blk = 0;
            c.h++;
            settle(c);
        }
        fit(c);
    };
    // does a row of the chunk r0 .. r0 + rows - 1 see a slot of the block?
    auto live = [&](const Seg &c, int blk, int r0, int rows) {
        const int p0 = c.s.L - c.s.nq, j0 = blk * BLK;
        if (rows <= 0 || j0 > p0 + (r0 + rows - 1) / v.G) return false;
        return v.window == 0 || j0 < v.sinks || (long long)j0 + BLK - 1 > (long long)p0 + r0 / v.G - v.window;
    };

    // (a chunk without such a block has no queries: its barrier would run ahead of the issuing warp)
    auto any_live = [&](const Seg &c, int r0, int rows) {
        for (int u = 0; u < c.n; u++)
            if (live(c, c.blk + u, r0, rows)) return true;
        return false;
    };

    if (from < to) {
        if (warp == 9) {
            // ---------------------------------------------------------------- TMA
            const unsigned long long pol = policy_evict_normal();
            const int per_tile = BLK >> v.page_shift;
            uint32_t g = 0;
            bool ok = true;
            for (Seg c = first_seg(); ok && c.n > 0; next_seg(c))
                for (int r0 = 0; ok && r0 < c.counted; r0 += ROWS)
                    for (int u = 0; ok && u < c.n; u++) {
                        if (!live(c, c.blk + u, r0, min(ROWS, c.counted - r0))) continue;
                        const int s = g % NS, slot = (c.blk + u) * BLK + (lane << v.page_shift);
                        const bool on = lane < per_tile && slot < c.s.L;
                        const int row = on ? (page_of(v, c.b, slot) * v.Hkv + c.h) << v.page_shift : 0;
                        const unsigned which = __ballot_sync(~0u, on);
                        ok = __all_sync(~0u, mbar_wait(empty(s), ((g / NS) & 1u) ^ 1u, abort_flag));
                        if (!ok) {
                            give_up();
                            break;
                        }
                        const bool leader = elect_one();
                        if (leader) mbar_expect_tx(full(s), __popc(which) * (uint32_t)(HALVES * v.page * 128));
                        for (int p = 0; p < per_tile; p++) {
                            const int r = __shfl_sync(~0u, row, p);
                            if ((which >> p & 1) && leader) {
#pragma unroll
                                for (int hf = 0; hf < HALVES; hf++)
                                    tma_load_2d(ring + s * C::TILE + hf * 16384 + (uint32_t)(p << v.page_shift) * 128u, &tmap_k, hf * 64, r, full(s), pol);
                            }
                        }
                        __syncwarp();
                        g++;
                    }
            int never = 0;  // every copy has landed and every stage is released before the CTA may leave
            for (uint32_t i = g > NS ? g - NS : 0; i < g; i++) {
                mbar_wait(full(i % NS), (i / NS) & 1u, &never);
                if (ok && !__all_sync(~0u, mbar_wait(empty(i % NS), (i / NS) & 1u, abort_flag))) {
                    give_up();
                    ok = false;
                }
            }
        } else if (warp == 8) {
            // ---------------------------------------------------------------- MMA
            uint32_t g = 0, n_q = 0;
            bool ok = true;
            auto wait = [&](uint32_t bar, uint32_t parity) {
                if (ok && !__all_sync(~0u, mbar_wait(bar, parity & 1u, abort_flag))) {
                    give_up();
                    ok = false;
                }
                tc_fence_after();
                return ok;
            };
            const unsigned long long qd = smem_desc_sw128(base);
            for (Seg c = first_seg(); ok && c.n > 0; next_seg(c))
                for (int r0 = 0; ok && r0 < c.counted; r0 += ROWS) {
                    const int rows = min(ROWS, c.counted - r0);
                    if (!any_live(c, r0, rows)) continue;
                    if (!wait(q_ready, n_q++)) break;
                    const uint32_t idesc = instr_desc(128, (rows + 15) & ~15);
                    for (int u = 0; ok && u < c.n; u++) {
                        if (!live(c, c.blk + u, r0, rows)) continue;
                        const uint32_t s = g % NS, x = g & 1;
                        if (!wait(full(s), g / NS)) break;
                        if (!wait(acc_empty(x), (g >> 1) ^ 1u)) break;
                        const unsigned long long kd = smem_desc_sw128(ring + s * C::TILE);
                        if (elect_one()) {
#pragma unroll
                            for (int k = 0; k < D / 16; k++)
                                umma_bf16(tmem + x * ROWS, kd + (k / 4) * (16384 >> 4) + 2 * (k % 4), qd + (k / 4) * ((ROWS * 128) >> 4) + 2 * (k % 4), idesc, k != 0);
                            umma_commit(empty(s));
                            umma_commit(acc_full(x));
                        }
                        __syncwarp();
                        g++;
                    }
                }
            int never = 0;
            if (elect_one()) umma_commit(drained);
            __syncwarp();
            mbar_wait(drained, 0, &never);
        } else {
            // ---------------------------------------------------------------- queries, and the columns' sums
            const int x = warp >> 2, row = threadIdx.x & 127;
            const uint32_t t_acc = tmem + x * ROWS + ((uint32_t)((warp & 3) * 32) << 16);
            const uint64_t scale2 = f2(a.scale_log2, a.scale_log2);
            uint32_t g = 0;
            bool dead = false;
            for (Seg c = first_seg(); c.n > 0; next_seg(c)) {
                const int p0 = c.s.L - c.s.nq, n_chunks = max(1, (c.counted + ROWS - 1) / ROWS);
                for (int ch = 0; ch < n_chunks; ch++) {
                    const int r0 = ch * ROWS, rows = min(ROWS, c.counted - r0);
                    bar_sync(1, 256);  // both warpgroups are done with the queries, and with the sums of the last chunk
                    if (any_live(c, r0, rows)) {
                        constexpr int CPR = D / 8;
                        const int n16 = (rows + 15) & ~15;
                        const __nv_bfloat16 *qp = (const __nv_bfloat16 *)a.q + (size_t)c.s.row0 * a.q_stride + (size_t)c.h * v.G * D;
#pragma unroll 4
                        for (int i = threadIdx.x; i < n16 * CPR; i += 256) {
                            const int r = i / CPR, cc = i % CPR, t = (r0 + r) / v.G;
                            const uint32_t dst = base + (cc >> 3) * (ROWS * 128) + r * 128 + (((cc & 7) ^ (r & 7)) << 4);
                            const bool on = r < rows;
                            const void *src = on ? (const void *)(qp + (size_t)t * a.q_stride + (size_t)(r0 + r - t * v.G) * D + cc * 8) : a.q;
                            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(on ? 16 : 0) : "memory");
                        }
                        {  // a row that does not count, or saw nothing: exp2(-inf) = 0
                            const int r = r0 + (int)threadIdx.x, t = r / v.G;
                            float l = -INFINITY;
                            if ((int)threadIdx.x < rows) l = __ldg(a.lse + ((size_t)c.s.row0 + t) * v.Hq + c.h * v.G + r - t * v.G);
                            neg[threadIdx.x] = l == -INFINITY ? -INFINITY : -l * LOG2E;
                            row_slot[threadIdx.x] = p0 + t;
                        }
                        asm volatile("cp.async.wait_all;" ::: "memory");
                        fence_async_shared();
                        mbar_arrive(q_ready);
                        bar_sync(1, 256);
                    }
                    for (int u = 0; u < c.n; u++) {
                        const int j0 = (c.blk + u) * BLK, j = j0 + row;
                        const bool on = live(c, c.blk + u, r0, rows);
                        // every block is written in the first chunk; the warpgroup whose turn it is takes the blocks without a row
                        if (on ? (int)(g & 1) != x : ch > 0 || (u & 1) != x) {
                            g += on;
                            continue;
                        }
                        const size_t at = ((size_t)c.b * v.Hkv + c.h) * v.cap + j;
                        const float *w_from = ch == 0 ? a.weight : a.weight_out;
                        const float before = j < c.s.L ? w_from[at] : 0.0f;
                        uint64_t sum[2] = {0, 0};
                        if (on) {
                            if (!dead && !__all_sync(~0u, mbar_wait(acc_full(x), (g >> 1) & 1u, abort_flag))) {
                                give_up();
                                dead = true;  // go through the motions, so that the barriers stay matched
                            }
                            tc_fence_after();
                            // does every row of the chunk see every slot of the block?
                            const bool masked = p0 + r0 / v.G < j0 + BLK - 1 || (v.window && j0 <= p0 + (r0 + rows - 1) / v.G - v.window);
                            auto use = [&](uint32_t (&sc)[64], int c0, auto is_masked) {
#pragma unroll
                                for (int q = 0; q < 64; q += 16) {
                                    if (c0 + q >= rows) break;
                                    if (c0 + q + 16 > rows) {  // columns that no product wrote
#pragma unroll
                                        for (int i = q; i < q + 16; i++)
                                            if (c0 + i >= rows) sc[i] = 0u;
                                    }
                                    // one bit per row that sees this slot; the others' exponentials count as zero, whatever
                                    // their lse is (a NaN there is no business of a slot that the row does not see)
                                    uint32_t seen = 0;
                                    if (is_masked.value) {
#pragma unroll
                                        for (int i = 0; i < 16; i++)
                                            if (sees(v, row_slot[(c0 + q + i) & (ROWS - 1)], j)) seen |= 1u << i;
                                    }
                                    auto pair = [&](uint64_t y, int i) {
                                        float a = ex2(lo(y)), b = ex2(hi(y));
                                        if (is_masked.value) {
                                            a = seen >> (i - q) & 1 ? a : 0.0f;
                                            b = seen >> (i - q + 1) & 1 ? b : 0.0f;
                                        }
                                        return f2(a, b);
                                    };
#pragma unroll
                                    for (int i = q; i < q + 16; i += 4) {
                                        const ulonglong2 n4 = *reinterpret_cast<const ulonglong2 *>(neg + c0 + i);
                                        const uint64_t y0 = fma2(f2(__uint_as_float(sc[i]), __uint_as_float(sc[i + 1])), scale2, n4.x), y1 = fma2(f2(__uint_as_float(sc[i + 2]), __uint_as_float(sc[i + 3])), scale2, n4.y);
                                        sum[0] = add2(sum[0], pair(y0, i));
                                        sum[1] = add2(sum[1], pair(y1, i + 2));
                                    }
                                }
                            };
                            for (int c0 = 0; c0 < rows; c0 += 64) {
                                uint32_t sc[64];
                                tmem_ld64(t_acc + c0, sc);
                                if (masked) use(sc, c0, Const<true>());
                                else use(sc, c0, Const<false>());
                            }
                            tc_fence_before();
                            mbar_arrive(acc_empty(x));
                            g++;
                        }
                        if (j < c.s.L) a.weight_out[at] = before + ((lo(sum[0]) + lo(sum[1])) + (hi(sum[0]) + hi(sum[1])));
                    }
                }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 8) tmem_dealloc(*tmem_slot, 512);
}

template <int D> cudaError_t weigh(const WeighArgs &a, const CUtensorMap &mk, int num_sms, cudaStream_t s) {
    const int smem = Cfg<D>::smem(a.v.B);
    weigh_umma_kernel<D><<<num_sms, THREADS, smem, s>>>(mk, a);
    return cudaGetLastError();
}

}  // namespace

cudaError_t prepare_weigh_umma() {
    const cudaError_t e = allow_shared(weigh_umma_kernel<64>);
    return e == cudaSuccess ? allow_shared(weigh_umma_kernel<128>) : e;
}

cudaError_t launch_weigh_umma(const WeighArgs &a, const CUtensorMap &mk, int num_sms, cudaStream_t s) {
    return a.v.D == 64 ? weigh<64>(a, mk, num_sms, s) : weigh<128>(a, mk, num_sms, s);
}

}  // namespace kv
}  // namespace aj
