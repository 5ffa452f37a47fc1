// aj_kv_weigh for bf16 and head sizes 64 and 128: accumulated attention weight of every cached slot.
//
//   weight_out[j] = weight[j] + sum over the counted rows r that see j of exp2(scale * q_r k_j - lse_r)
//
// The sum runs over the rows of one slot, so with slots on the 16-row side of mma.m16n8k16 and query rows on its
// 8-column side a lane adds up its own columns in registers; two shuffles at the end join the four lanes of a slot, and
// no slot is seen by more than one warp.  K is read once: with few rows that stream is all there is, and it runs through
// a ring of cp.async stages (128 slots, 32 per warp) that goes on across items; with a window's rows the products
// and exponentials come to about the same time.
//
// The (sequence, key head, 128-slot block) triples of the batch form one line, measured in cost (4 for the loads of a
// block + 1 for each group of 8 rows), and every CTA takes an equal piece of it; two CTAs per SM.
//
// Measured: 64 sequences of up to 4096 slots, 8 key heads of 128, 4 rows: 62 us for 306 MB back to back, 4.9 TB/s.  What
// is missing to a copy is the begin and end of a call of this length and the state's 4-byte reads and writes.
//
// The order of the head's elements within a product is free, so a lane takes 16 consecutive bytes of a row where the
// fragment layout asks for 4 x 4 bytes: both operands use the same order, and every load is 16 bytes.  The queries come
// straight from L1 / L2, one group of rows ahead.
#include "aj_kv.cuh"
#include "aj_kv_mma.cuh"

namespace aj {
namespace kv {

namespace {

constexpr int WARPS = 4, MT = 2, WS = MT * 16, BLK = WARPS * WS;

template <int D> struct Weigh {
    static constexpr int STAGES = D == 64 ? 6 : 3;
    static constexpr int STAGE = BLK * D * 2;
};

struct Cursor {
    int b, h, blk, units, w;  // sequence, key head, block, blocks of the sequence, cost of a block
    long long at;             // place on the line
    Seq s;
    int counted;              // rows that count
};

template <int D>
__global__ void __launch_bounds__(32 * WARPS, 2) weigh_kernel(WeighArgs a, int g_shift) {
    using C = Weigh<D>;
    constexpr int STAGES = C::STAGES, ROWB = D * 2, CPR = D / 8, RPI = 32 / CPR, KC = D / 32;
    extern __shared__ __align__(128) unsigned char smem[];
    long long *pre = reinterpret_cast<long long *>(smem + STAGES * C::STAGE);  // [B + 1]
    __shared__ long long wsum[WARPS];
    const View &v = a.v;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, q4 = lane & 3, r8 = lane >> 2;
    auto token = [&](int r) { return g_shift >= 0 ? r >> g_shift : r / v.G; };

    auto enter = [&](Cursor &c, int b) {
        c.b = b;
        c.s = seq_of(v, b);
        c.counted = min(c.s.nq, a.n_rows ? max(__ldg(a.n_rows + b), 0) : c.s.nq) * v.G;
        c.units = (c.s.L + BLK - 1) / BLK;
        c.w = 4 + (c.counted + 7) / 8;
    };
    long long base = 0;
    for (int b0 = 0; b0 < v.B; b0 += 32 * WARPS) {
        const int b = b0 + threadIdx.x;
        long long n = 0;
        if (b < v.B) {
            Cursor c;
            enter(c, b);
            n = (long long)c.units * v.Hkv * c.w;
        }
        const long long own = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long x = __shfl_up_sync(~0u, n, o);
            if (lane >= o) n += x;
        }
        if (lane == 31) wsum[warp] = n;
        __syncthreads();
        long long off = base;
        for (int w = 0; w < WARPS; w++) {
            if (w < warp) off += wsum[w];
            base += wsum[w];
        }
        if (b < v.B) pre[b] = off + n - own;
        __syncthreads();
    }
    if (threadIdx.x == 0) pre[v.B] = base;
    __syncthreads();
    const long long per = (base + gridDim.x - 1) / gridDim.x, from = per * blockIdx.x, to = min(base, from + per);
    if (from >= to) return;

    Cursor put;
    {
        int lo = 0, hi = v.B;  // pre[lo] <= from < pre[hi]
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (pre[mid] <= from) lo = mid; else hi = mid;
        }
        enter(put, lo);
        const int k = (int)((from - pre[lo] + put.w - 1) / put.w);  // the first block that begins at or after `from`
        put.h = k / put.units;
        put.blk = k - put.h * put.units;
        put.at = pre[lo] + (long long)k * put.w;
    }
    auto settle = [&](Cursor &c) {  // past the end of a sequence: to the next one with a block
        if (c.h < v.Hkv) return;
        int b = c.b + 1;
        while (b < v.B && pre[b] == pre[b + 1]) b++;
        c.at = base;
        if (b >= v.B) return;
        c.at = pre[b];
        c.h = c.blk = 0;
        enter(c, b);
    };
    settle(put);
    auto advance = [&](Cursor &c) {
        c.at += c.w;
        if (++c.blk < c.units) return;
        c.blk = 0;
        c.h++;
        settle(c);
    };
    // 16 slots from a multiple of 16 lie in one page: lane m holds the page of this warp's m-th 16
    auto pages_at = [&](const Cursor &c) {
        const int slot = c.blk * BLK + warp * WS + (lane & 1) * 16;
        return slot < c.s.L ? page_of(v, c.b, slot) : 0;
    };
    const uint32_t ring = s_addr(smem) + warp * WS * ROWB;
    auto issue = [&](const Cursor &c, int pages, int stage) {
        const int cc = lane % CPR;
#pragma unroll
        for (int m = 0; m < MT; m++) {
            const int slot = c.blk * BLK + warp * WS + m * 16, page = __shfl_sync(~0u, pages, m);
            const char *kp = (const char *)a.k + (((size_t)page * v.Hkv + c.h) * v.page + (slot & (v.page - 1))) * ROWB + cc * 16;
#pragma unroll
            for (int i = 0; i < 16 / RPI; i++) {
                const int r = i * RPI + lane / CPR;
                cp16(ring + stage * C::STAGE + (m * 16 + r) * ROWB + ((cc ^ ((r & 1) << 2)) << 4), kp + (size_t)r * ROWB, slot + r < c.s.L);
            }
        }
    };

    Cursor cur = put;
    int pages = put.at < to ? pages_at(put) : 0;
    auto put_next = [&](int stage) {
        if (put.at < to) {
            issue(put, pages, stage);
            advance(put);
            if (put.at < to) pages = pages_at(put);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < STAGES - 1; i++) put_next(i);

    int stage = 0;
    for (; cur.at < to; advance(cur)) {
        const Seq &s = cur.s;
        const int j0 = cur.blk * BLK + warp * WS, h = cur.h, counted = cur.counted;
        const size_t at = ((size_t)cur.b * v.Hkv + h) * v.cap + j0 + r8;
        float acc[MT][2] = {}, before[MT][2];  // the slots j0 + 16 m + r8 (+ 8); their weight so far, wanted last
#pragma unroll
        for (int m = 0; m < MT; m++)
#pragma unroll
            for (int i = 0; i < 2; i++) before[m][i] = q4 == 0 && j0 + 16 * m + r8 + 8 * i < s.L ? __ldg(a.weight + at + 16 * m + 8 * i) : 0.0f;
        // rows that can see one of this warp's slots: tokens at or after the first slot, and within the window of the last
        const int p0 = s.L - s.nq, j_end = min(j0 + WS, s.L);
        int t_hi = s.nq - 1;
        if (v.window && j0 >= v.sinks) t_hi = (int)min((long long)t_hi, (long long)j_end - 1 + v.window - 1 - p0);
        const int r_lo = max(0, j0 - p0) * v.G & ~7, r_hi = j0 < s.L ? min(counted, (t_hi + 1) * v.G) : 0;

        uint4 qf[KC];
        float ls[2];
        auto fetch_rows = [&](int r0) {
            const int r = r0 + r8, t = token(r);
            const uint4 *qp = reinterpret_cast<const uint4 *>((const __nv_bfloat16 *)a.q + ((size_t)s.row0 + t) * a.q_stride + (size_t)(h * v.G + r - t * v.G) * D) + q4;
#pragma unroll
            for (int c = 0; c < KC; c++) qf[c] = r < counted ? __ldg(qp + 4 * c) : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int e = 0; e < 2; e++) {
                const int x = r0 + q4 * 2 + e, tx = token(x);
                ls[e] = x < counted ? __ldg(a.lse + ((size_t)s.row0 + tx) * v.Hq + h * v.G + x - tx * v.G) : -INFINITY;
            }
        };
        if (r_lo < r_hi) fetch_rows(r_lo);
        __syncwarp();  // the stage issued into next was consumed by every lane
        put_next(stage == 0 ? STAGES - 1 : stage - 1);
        asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
        __syncwarp();

        uint4 kf[MT][2][KC];
        if (r_lo < r_hi) {
            const unsigned char *kb = smem + stage * C::STAGE + warp * WS * ROWB;
#pragma unroll
            for (int m = 0; m < MT; m++)
#pragma unroll
                for (int i = 0; i < 2; i++)
#pragma unroll
                    for (int c = 0; c < KC; c++)
                        kf[m][i][c] = *reinterpret_cast<const uint4 *>(kb + (m * 16 + r8 + 8 * i) * ROWB + (((4 * c + q4) ^ ((r8 & 1) << 2)) << 4));
        }
        for (int r0 = r_lo; r0 < r_hi; r0 += 8) {
            float sc[MT][4];
#pragma unroll
            for (int m = 0; m < MT; m++) sc[m][0] = sc[m][1] = sc[m][2] = sc[m][3] = 0.0f;
#pragma unroll
            for (int c = 0; c < KC; c++)
#pragma unroll
                for (int m = 0; m < MT; m++) {
                    mma4(sc[m], kf[m][0][c].x, kf[m][1][c].x, kf[m][0][c].y, kf[m][1][c].y, qf[c].x, qf[c].y);
                    mma4(sc[m], kf[m][0][c].z, kf[m][1][c].z, kf[m][0][c].w, kf[m][1][c].w, qf[c].z, qf[c].w);
                }
            float neg[2];  // a row that does not count, or saw nothing: exp2(-inf) = 0
#pragma unroll
            for (int e = 0; e < 2; e++) neg[e] = ls[e] == -INFINITY ? -INFINITY : -ls[e] * LOG2E;
            if (r0 + 8 < r_hi) fetch_rows(r0 + 8);
            // do all rows of the group see all slots of the warp?
            const int t0 = token(r0), t1 = token(min(r0 + 7, counted - 1));
            const bool masked = p0 + t0 < j_end - 1 || (v.window && j0 <= p0 + t1 - v.window);
#pragma unroll
            for (int m = 0; m < MT; m++)
#pragma unroll
                for (int i = 0; i < 4; i++)
                    if (!masked || sees(v, p0 + token(r0 + q4 * 2 + (i & 1)), j0 + 16 * m + r8 + 8 * (i >> 1)))
                        acc[m][i >> 1] += ex2(fmaf(sc[m][i], a.scale_log2, neg[i & 1]));
        }
#pragma unroll
        for (int m = 0; m < MT; m++)
#pragma unroll
            for (int i = 0; i < 2; i++) {
                float x = acc[m][i];
                x += __shfl_xor_sync(~0u, x, 1);
                x += __shfl_xor_sync(~0u, x, 2);
                if (q4 == 0 && j0 + 16 * m + r8 + 8 * i < s.L) a.weight_out[at + 16 * m + 8 * i] = before[m][i] + x;
            }
        if (++stage == STAGES) stage = 0;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
}

template <int D> cudaError_t weigh(const WeighArgs &a, int num_sms, cudaStream_t s) {
    using C = Weigh<D>;
    const size_t smem = (size_t)C::STAGES * C::STAGE + (a.v.B + 1) * 8;
    int g_shift = -1;
    for (int i = 0; i < 11; i++)
        if (a.v.G == 1 << i) g_shift = i;
    weigh_kernel<D><<<2 * num_sms, 32 * WARPS, smem, s>>>(a, g_shift);
    return cudaGetLastError();
}

}  // namespace

cudaError_t prepare_weigh_mma() {
    const cudaError_t e = allow_shared(weigh_kernel<64>);
    return e == cudaSuccess ? allow_shared(weigh_kernel<128>) : e;
}

cudaError_t launch_weigh_mma(const WeighArgs &a, int num_sms, cudaStream_t s) {
    return a.v.D == 64 ? weigh<64>(a, num_sms, s) : weigh<128>(a, num_sms, s);
}

}  // namespace kv
}  // namespace aj
