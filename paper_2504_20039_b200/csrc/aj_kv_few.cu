// aj_kv_attend for few query rows per key head (a decode step: new tokens x query heads per key head <= 16), bf16.
//
// Every key and value is read once and meets few rows, so the kernel is bound by the stream of pages from HBM.  Scores
// are computed transposed, S^T = K Q^T and O^T = V^T P^T, with keys (then head elements) on the 16-row side of
// mma.m16n8k16 and the query rows on its 8-column side: 8 rows fill the instruction, where rows on the 16-row
// side would leave it half to seven eighths empty.  (At one to sixteen rows the work is 1/16 of what tcgen05 is built
// for, and a 128-row tile of it would wait for its softmax on one to sixteen lanes.)
//
// The (sequence, key head, 64-slot block) triples of the whole batch form one line that is cut into equal pieces, one
// per CTA, two CTAs per SM: sequences of any mix of lengths are balanced without the host knowing them, and a CTA's
// ring of loads (cp.async, three stages of 64 slots, K and V) runs on across the items.  Each warp loads and
// consumes its own 16 slots of a block, so no barrier of the CTA is on the way; the four warps' running (maximum, sum,
// output) are joined at the end of an item.  An item that spans CTAs leaves partial results in the workspace and the
// CTA that arrives last joins them, in the order of the CTAs.
//
// Measured: 64 sequences of up to 8191 slots, 8 key heads of 128, 4 rows: 159 us for 932 MB back to back, 5.9 TB/s, nine
// tenths of a plain copy; with a window of 4096, 32 sequences, 8 rows: 90 us, 5.8 TB/s.
//
// The running maximum is only a common reference: it is raised when a score exceeds it by more than RAISE (one
// vote per block instead of six shuffles), and weights far above 1 are as exact in bf16 and f32 as weights up to 1.
#include "aj_kv.cuh"
#include "aj_kv_mma.cuh"

namespace aj {
namespace kv {

namespace {

constexpr int BLK = 64, WARPS = 4, STAGES = 3;

// The blocks of slots that the new tokens of a sequence see: n_sink blocks from 0, then those from first_blk on.
struct Span {
    int n_sink, first_blk, units, first;
};
__device__ inline Span span_of(const View &v, const Seq &s) {
    Span r;
    r.first = v.window ? max(0, s.L - s.nq - v.window + 1) : s.first;
    r.first = min(r.first, s.L);
    r.first_blk = r.first / BLK;
    r.n_sink = min((min(v.sinks, r.first) + BLK - 1) / BLK, r.first_blk);
    r.units = s.nq > 0 ? max(1, r.n_sink + (s.L + BLK - 1) / BLK - r.first_blk) : 0;
    return r;
}

template <int D, int NT> struct Few {
    static constexpr int STAGE = 2 * BLK * D * 2;
    static constexpr int JOIN_FLOATS = WARPS * 8 * (D / 2 + 4);  // half a row at a time: two CTAs must fit an SM
    static constexpr int MAX_PARTS = 296;
    static constexpr int SCRATCH = (JOIN_FLOATS > MAX_PARTS * 8 ? JOIN_FLOATS : MAX_PARTS * 8) * 4;
    static constexpr int PART = 8 * NT * (D + 2);  // floats of one partial result
};

// Position in the line of blocks.
struct Cursor {
    int b, h, blk;  // sequence, key head, block within the item
    Seq s;
    Span sp;
};

template <int D, int NT, bool SHARED>
__global__ void __launch_bounds__(32 * WARPS, 2) attend_few_kernel(AttendArgs a) {
    using C = Few<D, NT>;
    constexpr int ROWB = D * 2, CPR = D / 8, RPI = 32 / CPR, KS = D / 16;
    extern __shared__ __align__(128) unsigned char smem[];
    float *scratch = reinterpret_cast<float *>(smem + STAGES * C::STAGE);
    int *pre = reinterpret_cast<int *>(smem + STAGES * C::STAGE + C::SCRATCH);  // [B + 1]
    __shared__ float sm_m[WARPS][8 * NT], sm_l[WARPS][8 * NT];
    __shared__ int wsum[WARPS], last_flag;
    const View &v = a.v;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    // the line of blocks: prefix sums over the sequences
    int base = 0;
    for (int b0 = 0; b0 < v.B; b0 += 32 * WARPS) {
        const int b = b0 + threadIdx.x;
        int n = b < v.B ? span_of(v, seq_of<SHARED>(v, b)).units * v.Hkv : 0;
        const int own = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(~0u, n, o);
            if (lane >= o) n += x;
        }
        if (lane == 31) wsum[warp] = n;
        __syncthreads();
        int off = base;
        for (int w = 0; w < WARPS; w++) {
            if (w < warp) off += wsum[w];
            base += wsum[w];
        }
        if (b < v.B) pre[b] = off + n - own;
        __syncthreads();
    }
    if (threadIdx.x == 0) pre[v.B] = base;
    __syncthreads();
    const int total = base, per = (total + gridDim.x - 1) / gridDim.x;
    const int u0 = min(total, (int)blockIdx.x * per), u1 = min(total, u0 + per);
    // A shared call: the kernel before it (over the shared slots) and this one run side by side; the join waits for this one only,
    // so this one waits for the other before it ends.
    if (SHARED) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (u0 >= u1) {
        if (SHARED) asm volatile("griddepcontrol.wait;" ::: "memory");
        return;
    }

    auto seek = [&](int u) {
        Cursor c;
        int lo = 0, hi = v.B;  // pre[lo] <= u < pre[hi]
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (pre[mid] <= u) lo = mid; else hi = mid;
        }
        c.b = lo;
        c.s = seq_of<SHARED>(v, lo);
        c.sp = span_of(v, c.s);
        const int r = u - pre[lo];
        c.h = r / c.sp.units;
        c.blk = r - c.h * c.sp.units;
        return c;
    };
    auto advance = [&](Cursor &c) {
        if (++c.blk < c.sp.units) return;
        c.blk = 0;
        if (++c.h < v.Hkv) return;
        c.h = 0;
        do {
            if (++c.b >= v.B) return;
        } while (pre[c.b] == pre[c.b + 1]);
        c.s = seq_of<SHARED>(v, c.b);
        c.sp = span_of(v, c.s);
    };
    auto slot_of = [&](const Cursor &c) {  // first slot of this warp's 16 in the cursor's block
        return (c.blk < c.sp.n_sink ? c.blk : c.blk - c.sp.n_sink + c.sp.first_blk) * BLK + warp * 16;
    };
    auto page_at = [&](const Cursor &c) {  // 16 slots from a multiple of 16 lie in one page
        const int slot = slot_of(c);
        return slot < c.s.L ? page_of(v, c.b, slot) : 0;
    };
    const uint32_t ring = s_addr(smem) + warp * 16 * ROWB;
    auto issue = [&](const Cursor &c, int page, int stage) {
        const int slot = slot_of(c);
        const size_t row0 = ((size_t)page * v.Hkv + c.h) * v.page + (slot & (v.page - 1));
        const int cc = lane % CPR;
        const uint32_t dst = ring + stage * C::STAGE;
        const char *kp = (const char *)a.k + row0 * ROWB + cc * 16, *vp = (const char *)a.vv + row0 * ROWB + cc * 16;
#pragma unroll
        for (int i = 0; i < 16 / RPI; i++) {
            const int r = i * RPI + lane / CPR;
            // slots that none of the new tokens sees are read as zeros, whatever they hold
            const bool on = slot + r < c.s.L && (slot + r >= c.sp.first || slot + r < v.sinks);
            const uint32_t d = dst + r * ROWB + ((cc ^ (r & 7)) << 4);
            cp16(d, kp + (size_t)r * ROWB, on);
            cp16(d + BLK * ROWB, vp + (size_t)r * ROWB, on);
        }
    };

    Cursor put = seek(u0), cur = put;
    int next_u = u0, next_page = page_at(put);
#pragma unroll
    for (int i = 0; i < STAGES - 1; i++) {
        if (next_u < u1) {
            issue(put, next_page, i);
            if (++next_u < u1) {
                advance(put);
                next_page = page_at(put);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    }

    uint32_t qf[NT][KS][2];
    float o[KS][NT][4], m[NT][2], l[NT][2];
    int stage = 0;
    bool begins = true;  // the cursor has just entered an item

    for (int u = u0; u < u1; u++) {
        const int n_rows = cur.s.nq * v.G;
        const int p_lo = cur.s.L - cur.s.nq;
        if (begins) {
            begins = false;
#pragma unroll
            for (int n = 0; n < NT; n++) {
                const int r = n * 8 + (lane >> 2);
                const uint32_t *qp = nullptr;
                if (r < n_rows)
                    qp = reinterpret_cast<const uint32_t *>((const __nv_bfloat16 *)a.q + ((size_t)cur.s.row0 + r / v.G) * a.q_stride +
                                                            (size_t)(cur.h * v.G + r % v.G) * D) + (lane & 3);
#pragma unroll
                for (int k = 0; k < KS; k++) {
                    qf[n][k][0] = qp ? __ldg(qp + k * 8) : 0u;
                    qf[n][k][1] = qp ? __ldg(qp + k * 8 + 4) : 0u;
                    o[k][n][0] = o[k][n][1] = o[k][n][2] = o[k][n][3] = 0.0f;
                }
                m[n][0] = m[n][1] = -INFINITY;
                l[n][0] = l[n][1] = 0.0f;
            }
        }
        __syncwarp();  // the stage issued into next was consumed by every lane
        if (next_u < u1) {
            issue(put, next_page, stage == 0 ? STAGES - 1 : stage - 1);
            if (++next_u < u1) {
                advance(put);
                next_page = page_at(put);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
        __syncwarp();
        const uint32_t kb = ring + stage * C::STAGE, vb = kb + BLK * ROWB;
        const int mi = lane >> 3, mr = lane & 7;

        float s[NT][2][4];
#pragma unroll
        for (int n = 0; n < NT; n++)
#pragma unroll
            for (int i = 0; i < 4; i++) s[n][0][i] = s[n][1][i] = 0.0f;
#pragma unroll
        for (int k = 0; k < KS; k++) {
            uint32_t af[4];
            const int key = (mi & 1) * 8 + mr, c = k * 2 + (mi >> 1);
            ldsm4(af, kb + key * ROWB + ((c ^ (key & 7)) << 4));
#pragma unroll
            for (int n = 0; n < NT; n++) mma(s[n][k & 1], af, qf[n][k][0], qf[n][k][1]);
        }
        const int slot = slot_of(cur), blk0 = slot - warp * 16;
        const bool masked = blk0 + BLK > p_lo + 1 || (v.window && blk0 <= cur.s.L - 1 - v.window);
        bool raise = false;
#pragma unroll
        for (int n = 0; n < NT; n++)
#pragma unroll
            for (int i = 0; i < 4; i++) {
                float x = (s[n][0][i] + s[n][1][i]) * a.scale_log2;
                if (masked) {
                    const int j = slot + (lane >> 2) + (i >> 1) * 8;
                    const int r = min(n * 8 + (lane & 3) * 2 + (i & 1), n_rows - 1);
                    if (!sees(v, p_lo + r / v.G, j)) x = -INFINITY;
                }
                s[n][0][i] = x;
                raise |= x > m[n][i & 1] + RAISE;
            }
        if (__any_sync(~0u, raise)) {
#pragma unroll
            for (int n = 0; n < NT; n++)
#pragma unroll
                for (int e = 0; e < 2; e++) {
                    float x = fmaxf(s[n][0][e], s[n][0][e + 2]);
                    x = fmaxf(x, __shfl_xor_sync(~0u, x, 4));
                    x = fmaxf(x, __shfl_xor_sync(~0u, x, 8));
                    x = fmaxf(x, __shfl_xor_sync(~0u, x, 16));
                    x = fmaxf(x, m[n][e]);
                    const float c = x == -INFINITY ? 1.0f : ex2(m[n][e] - x);
                    m[n][e] = x;
                    l[n][e] *= c;
#pragma unroll
                    for (int k = 0; k < KS; k++) {
                        o[k][n][e] *= c;
                        o[k][n][e + 2] *= c;
                    }
                }
        }
        uint32_t pf[NT][2];
#pragma unroll
        for (int n = 0; n < NT; n++) {
            float p[4];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const float ref = m[n][i & 1] == -INFINITY ? 0.0f : m[n][i & 1];
                p[i] = ex2(s[n][0][i] - ref);
            }
            l[n][0] += p[0] + p[2];
            l[n][1] += p[1] + p[3];
            pf[n][0] = transpose8(pack(p[0], p[1]));
            pf[n][1] = transpose8(pack(p[2], p[3]));
        }
#pragma unroll
        for (int k = 0; k < KS; k++) {
            uint32_t af[4];
            const int key = (mi >> 1) * 8 + mr, c = k * 2 + (mi & 1);
            ldsm4t(af, vb + key * ROWB + ((c ^ (key & 7)) << 4));
#pragma unroll
            for (int n = 0; n < NT; n++) mma(o[k][n], af, pf[n][0], pf[n][1]);
        }
        if (++stage == STAGES) stage = 0;

        const bool ends = cur.blk + 1 == cur.sp.units;
        if (ends || u + 1 == u1) {
            // ---- join the warps; then store, or leave a partial result and join those if this CTA is the last
            const int item = cur.b * v.Hkv + cur.h;
            const int i0 = pre[cur.b] + cur.h * cur.sp.units, i1 = i0 + cur.sp.units;  // the item's piece of the line
            const int c0 = i0 / per, c1 = (i1 - 1) / per;                            // and the CTAs it spans
            const bool whole = c0 == c1;
            float *mine = a.parts + ((size_t)blockIdx.x * 2 + (u0 <= i0 ? 1 : 0)) * C::PART;
#pragma unroll
            for (int n = 0; n < NT; n++)
#pragma unroll
                for (int e = 0; e < 2; e++) {
                    float x = l[n][e];
                    x += __shfl_xor_sync(~0u, x, 4);
                    x += __shfl_xor_sync(~0u, x, 8);
                    x += __shfl_xor_sync(~0u, x, 16);
                    if (lane < 4) {
                        sm_m[warp][n * 8 + lane * 2 + e] = m[n][e];
                        sm_l[warp][n * 8 + lane * 2 + e] = x;
                    }
                }
            auto store = [&](int r, int d, float4 x, float mm, float ll) {  // four elements of an output row
                if (SHARED && cur.s.first) {  // a part of the row, to be joined with the shared slots
                    const int rr = cur.s.row0 - rows_of(v).base, rowg = rr * v.G + r;
                    *reinterpret_cast<float4 *>(pre_o(a, v.n_chunks, cur.h, rowg) + d) = x;
                    if (d == 0) a.own_ml[(size_t)(rr + r / v.G) * v.Hq + cur.h * v.G + r % v.G] = make_float2(mm, ll);
                    return;
                }
                const float inv = ll == 0.0f ? 0.0f : 1.0f / ll;  // a sum that is NaN stays one
                const size_t row = (size_t)cur.s.row0 + r / v.G;
                const int head = cur.h * v.G + r % v.G;
                uint2 y;
                y.x = pack(x.x * inv, x.y * inv);
                y.y = pack(x.z * inv, x.w * inv);
                *reinterpret_cast<uint2 *>((__nv_bfloat16 *)a.out + row * a.out_stride + (size_t)head * D + d) = y;
                if (d == 0 && a.lse) a.lse[row * v.Hq + head] = ll == 0.0f ? -INFINITY : (mm + log2f(ll)) * LN2;
            };
#pragma unroll
            for (int nh = 0; nh < 2 * NT; nh++) {
                constexpr int H = D / 2;
                const int n = nh >> 1, hf = nh & 1;
#pragma unroll
                for (int k = 0; k < KS / 2; k++)
#pragma unroll
                    for (int i = 0; i < 4; i++)
                        scratch[(warp * 8 + (lane & 3) * 2 + (i & 1)) * (H + 4) + k * 16 + (lane >> 2) + (i >> 1) * 8] = o[hf * (KS / 2) + k][n][i];
                __syncthreads();
                const int rows = min(8, n_rows - n * 8);
                for (int i = threadIdx.x; i < rows * (H / 4); i += 32 * WARPS) {
                    const int r = i / (H / 4), dh = (i - r * (H / 4)) * 4, d = hf * H + dh, rr = n * 8 + r;
                    float mm = -INFINITY, ll = 0.0f;
                    float4 x = make_float4(0, 0, 0, 0);
#pragma unroll
                    for (int w = 0; w < WARPS; w++) mm = fmaxf(mm, sm_m[w][rr]);
                    const float ref = mm == -INFINITY ? 0.0f : mm;
#pragma unroll
                    for (int w = 0; w < WARPS; w++) {
                        const float c = ex2(sm_m[w][rr] - ref);
                        const float4 y = *reinterpret_cast<const float4 *>(scratch + (w * 8 + r) * (H + 4) + dh);
                        ll += c * sm_l[w][rr];
                        x.x += c * y.x;
                        x.y += c * y.y;
                        x.z += c * y.z;
                        x.w += c * y.w;
                    }
                    if (whole) {
                        store(rr, d, x, mm, ll);
                    } else {
                        *reinterpret_cast<float4 *>(mine + rr * D + d) = x;
                        if (d == 0) {
                            mine[8 * NT * D + rr] = mm;
                            mine[8 * NT * (D + 1) + rr] = ll;
                        }
                    }
                }
                __syncthreads();
            }
            if (!whole) {
                __threadfence();
                __syncthreads();
                if (threadIdx.x == 0) last_flag = atomicAdd(a.counters + item, 1u) == (unsigned)(c1 - c0);
                __syncthreads();
                if (last_flag) {
                    __threadfence();
                    const int n_parts = c1 - c0 + 1;
                    // the first CTA of an item holds it in its second place, the others in their first
                    auto part = [&](int i) { return a.parts + ((size_t)(c0 + i) * 2 + (i == 0 ? 1 : 0)) * C::PART; };
#pragma unroll
                    for (int n = 0; n < NT; n++) {
                        const int rows = min(8, n_rows - n * 8);
                        for (int i = threadIdx.x; i < n_parts * 8; i += 32 * WARPS) scratch[i] = __ldcg(part(i >> 3) + 8 * NT * D + n * 8 + (i & 7));
                        __syncthreads();
                        for (int i = threadIdx.x; i < rows * (D / 4); i += 32 * WARPS) {
                            const int r = i / (D / 4), d = (i - r * (D / 4)) * 4, rr = n * 8 + r;
                            float mm = -INFINITY, ll = 0.0f;
                            float4 x = make_float4(0, 0, 0, 0);
                            for (int w = 0; w < n_parts; w++) mm = fmaxf(mm, scratch[w * 8 + r]);
                            const float ref = mm == -INFINITY ? 0.0f : mm;
#pragma unroll 8
                            for (int w = 0; w < n_parts; w++) {
                                const float4 y = __ldcg(reinterpret_cast<const float4 *>(part(w) + rr * D + d));
                                const float c = ex2(scratch[w * 8 + r] - ref);
                                ll += c * __ldcg(part(w) + 8 * NT * (D + 1) + rr);
                                x.x += c * y.x;
                                x.y += c * y.y;
                                x.z += c * y.z;
                                x.w += c * y.w;
                            }
                            store(rr, d, x, mm, ll);
                        }
                        __syncthreads();
                    }
                    if (threadIdx.x == 0) a.counters[item] = 0u;
                }
            }
            begins = true;
        }
        advance(cur);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (SHARED) asm volatile("griddepcontrol.wait;" ::: "memory");
}

template <int D, int NT, bool SHARED> cudaError_t few(const AttendArgs &a, int num_sms, cudaStream_t s) {
    using C = Few<D, NT>;
    const size_t smem = (size_t)STAGES * C::STAGE + C::SCRATCH + (a.v.B + 1) * 4;
    auto kernel = attend_few_kernel<D, NT, SHARED>;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2 * num_sms < C::MAX_PARTS ? 2 * num_sms : C::MAX_PARTS);
    cfg.blockDim = dim3(32 * WARPS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = SHARED ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, a);
}

}  // namespace

template <bool SHARED> static cudaError_t prepare() {
    cudaError_t e = allow_shared(attend_few_kernel<64, 1, SHARED>);
    if (e == cudaSuccess) e = allow_shared(attend_few_kernel<64, 2, SHARED>);
    if (e == cudaSuccess) e = allow_shared(attend_few_kernel<128, 1, SHARED>);
    return e == cudaSuccess ? allow_shared(attend_few_kernel<128, 2, SHARED>) : e;
}

cudaError_t prepare_attend_few() {
    const cudaError_t e = prepare<false>();
    return e == cudaSuccess ? prepare<true>() : e;
}

size_t few_parts_floats(int D, int num_sms) { return (size_t)(2 * num_sms < 296 ? 2 * num_sms : 296) * 2 * 16 * (D + 2); }

template <bool SHARED> static cudaError_t launch(const AttendArgs &a, int num_sms, cudaStream_t s) {
    const bool one = a.v.n_q * a.v.G <= 8;
    if (a.v.D == 64) return one ? few<64, 1, SHARED>(a, num_sms, s) : few<64, 2, SHARED>(a, num_sms, s);
    return one ? few<128, 1, SHARED>(a, num_sms, s) : few<128, 2, SHARED>(a, num_sms, s);
}

cudaError_t launch_attend_few(const AttendArgs &a, int num_sms, cudaStream_t s) {
    return a.v.shared ? launch<true>(a, num_sms, s) : launch<false>(a, num_sms, s);
}

}  // namespace kv
}  // namespace aj
