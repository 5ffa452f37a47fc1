// aj_kv_weigh for bf16 and head sizes 64 and 128: accumulated attention weight of every cached slot.
//
//   weight_out[j] = weight[j] + sum over the counted rows r that see j of exp2(scale * q_r k_j - lse_r)
//
// The sum runs over the rows of one slot, so with slots on the 16-row side of mma.m16n8k16 and query rows on its
// 8-column side a lane adds up its own columns in registers; two shuffles at the end join the four lanes of a slot, and
// no slot is seen by more than one warp.  A warp holds 32 slots' keys in registers for the whole call (8 warps: 256
// slots per CTA) and walks over the rows, whose fragments come from L1.  K is read once; with few rows that is all.
// The order of the head's elements within a product is free, so a lane takes 16 consecutive bytes of a row where the
// fragment layout asks for 4 x 4 bytes: both operands use the same order, and every load is 16 bytes.
#include "aj_kv.cuh"

namespace aj {
namespace kv {

namespace {

constexpr int WARPS = 8, MT = 2, SLOTS = WARPS * MT * 16;

__device__ inline void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <int D>
__global__ void __launch_bounds__(32 * WARPS, 2) weigh_mma_kernel(WeighArgs a) {
    constexpr int KC = D / 32;  // 16-byte pieces of a row that a lane holds
    const View &v = a.v;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, q4 = lane & 3, r8 = lane >> 2;
    const int h = blockIdx.y % v.Hkv, b = blockIdx.y / v.Hkv;
    const Seq s = seq_of(v, b);
    const int j0 = (blockIdx.x * WARPS + warp) * MT * 16;
    if (j0 >= s.L) return;
    const int counted = min(s.nq, a.n_rows ? max(__ldg(a.n_rows + b), 0) : s.nq) * v.G;

    // this lane's slots: j0 + 16 m + r8 (+ 8)
    uint4 kf[MT][2][KC];
#pragma unroll
    for (int m = 0; m < MT; m++) {
        const int slot = j0 + 16 * m;
        const size_t row0 = slot < s.L ? page_row(v, b, h, slot) : 0;  // 16 slots from a multiple of 16 lie in one page
#pragma unroll
        for (int i = 0; i < 2; i++) {
            const bool on = slot + r8 + 8 * i < s.L;
            const uint4 *p = reinterpret_cast<const uint4 *>((const __nv_bfloat16 *)a.k + (row0 + r8 + 8 * i) * D) + q4;
#pragma unroll
            for (int c = 0; c < KC; c++) kf[m][i][c] = on ? __ldg(p + 4 * c) : make_uint4(0, 0, 0, 0);
        }
    }
    // rows that can see one of this warp's slots: tokens at or after the first slot, and within the window of the last
    const int p0 = s.L - s.nq, j_end = min(j0 + MT * 16, s.L);
    const int t_lo = max(0, j0 - p0);
    int t_hi = s.nq - 1;
    if (v.window && j0 >= v.sinks) t_hi = (int)min((long long)t_hi, (long long)j_end - 1 + v.window - 1 - p0);
    const int r_lo = t_lo * v.G & ~7, r_hi = min(counted, (t_hi + 1) * v.G);

    float acc[MT][2] = {};
    for (int r0 = r_lo; r0 < r_hi; r0 += 8) {
        uint4 qf[KC];
        const int rq = r0 + r8, tq = rq / v.G;
        const uint4 *qp = reinterpret_cast<const uint4 *>((const __nv_bfloat16 *)a.q + ((size_t)s.row0 + tq) * a.q_stride + (size_t)(h * v.G + rq - tq * v.G) * D) + q4;
#pragma unroll
        for (int c = 0; c < KC; c++) qf[c] = rq < counted ? __ldg(qp + 4 * c) : make_uint4(0, 0, 0, 0);
        float ls[2];
        int pos[2];
#pragma unroll
        for (int e = 0; e < 2; e++) {
            const int r = r0 + q4 * 2 + e, t = r / v.G;
            pos[e] = p0 + t;
            ls[e] = INFINITY;  // a row that does not count, or saw nothing: exp2(-inf) = 0
            if (r < counted) {
                const float x = __ldg(a.lse + ((size_t)s.row0 + t) * v.Hq + h * v.G + r - t * v.G);
                if (x != -INFINITY) ls[e] = x * LOG2E;
            }
        }
        float sc[MT][4];
#pragma unroll
        for (int m = 0; m < MT; m++) {
            sc[m][0] = sc[m][1] = sc[m][2] = sc[m][3] = 0.0f;
#pragma unroll
            for (int c = 0; c < KC; c++) {
                mma(sc[m], kf[m][0][c].x, kf[m][1][c].x, kf[m][0][c].y, kf[m][1][c].y, qf[c].x, qf[c].y);
                mma(sc[m], kf[m][0][c].z, kf[m][1][c].z, kf[m][0][c].w, kf[m][1][c].w, qf[c].z, qf[c].w);
            }
        }
        // all rows of the group see all slots of the warp?
        const int t0 = r0 / v.G, t1 = min(r0 + 7, counted - 1) / v.G;
        const bool masked = p0 + t0 < j_end - 1 || (v.window && j0 <= p0 + t1 - v.window);
#pragma unroll
        for (int m = 0; m < MT; m++)
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int e = i & 1;
                if (!masked || sees(v, pos[e], j0 + 16 * m + r8 + 8 * (i >> 1))) acc[m][i >> 1] += ex2(fmaf(sc[m][i], a.scale_log2, -ls[e]));
            }
    }
#pragma unroll
    for (int m = 0; m < MT; m++)
#pragma unroll
        for (int i = 0; i < 2; i++) {
            float x = acc[m][i];
            x += __shfl_xor_sync(~0u, x, 1);
            x += __shfl_xor_sync(~0u, x, 2);
            const int j = j0 + 16 * m + r8 + 8 * i;
            if (q4 == 0 && j < s.L) {
                const size_t at = ((size_t)b * v.Hkv + h) * v.cap + j;
                a.weight_out[at] = a.weight[at] + x;
            }
        }
}

}  // namespace

cudaError_t launch_weigh_mma(const WeighArgs &a, cudaStream_t s) {
    const dim3 grid((unsigned)((a.v.cap + SLOTS - 1) / SLOTS), a.v.B * a.v.Hkv);
    if (a.v.D == 64)
        weigh_mma_kernel<64><<<grid, 32 * WARPS, 0, s>>>(a);
    else
        weigh_mma_kernel<128><<<grid, 32 * WARPS, 0, s>>>(a);
    return cudaGetLastError();
}

}  // namespace kv
}  // namespace aj
