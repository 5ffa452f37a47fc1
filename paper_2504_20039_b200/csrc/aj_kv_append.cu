// Norms of queries and keys per head, position rotation, and the write of new tokens into the cache's pages.
//
//   y = x * rsqrt(mean(x^2) + eps) * w,   (a, b) -> (a cos - b sin, b cos + a sin) per rotated pair,
// in 32 bits with one rounding on the store.  The pass reads and writes (Hq + 2 Hkv) * D elements per token and
// nothing else of that size, so it is bound by memory.  Measured: 8 ragged prompts of up to 4096 tokens, 64 + 8 + 8 heads of
// 128, 766 MB: 139 us, 5.5 TB/s, 0.84 of a plain copy; a single token takes what its launch takes.
#include "aj_kv.cuh"

namespace aj {
namespace kv {

namespace {

// ---- any head size and rotation: one warp per head vector, the vector in shared memory

template <typename T>
__global__ void __launch_bounds__(128) append_any_kernel(AppendArgs a) {
    __shared__ float buf[4][256];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, D = a.v.D;
    const int heads = a.v.Hq + 2 * a.v.Hkv;
    const long long at = (long long)blockIdx.x * 4 + warp;  // (token of the batch, head)
    const int b = blockIdx.y;
    const int t = (int)(at / heads), hh = (int)(at % heads);
    const Seq s = seq_of(a.v, b);
    if (t >= s.nq) return;
    const size_t row = (size_t)s.row0 + t;
    const int slot = s.L - s.nq + t;
    const bool is_q = hh < a.v.Hq, is_v = hh >= a.v.Hq + a.v.Hkv;
    const int h = is_q ? hh : is_v ? hh - a.v.Hq - a.v.Hkv : hh - a.v.Hq;
    const T *src = (is_q ? (const T *)a.q + row * a.q_stride : is_v ? (const T *)a.vv + row * a.v_stride : (const T *)a.k + row * a.k_stride) + (size_t)h * D;
    T *dst = nullptr;
    if (is_q) {
        dst = (T *)a.q_out + row * a.q_out_stride + (size_t)h * D;
    } else if (slot >= 0) {
        const int p = __ldg(a.v.table + (size_t)b * a.v.width + (slot >> a.v.page_shift));
        if ((unsigned)p < (unsigned)a.v.n_pages)
            dst = (T *)(is_v ? a.v_pages : a.k_pages) + (((size_t)p * a.v.Hkv + h) * a.v.page + (slot & (a.v.page - 1))) * D;
    }
    const int pos = a.positions ? __ldg(a.positions + row) : slot;
    if (hh >= a.v.Hq && !is_v && slot >= 0 && lane == 0) {
        const size_t i = ((size_t)b * a.v.Hkv + h) * a.v.cap + slot;
        if (a.slot_pos) a.slot_pos[i] = pos;
        if (a.weight) a.weight[i] = 0.0f;
    }
    float sq = 0.0f;
    for (int d = lane; d < D; d += 32) {
        const float x = to_f32(src[d]);
        buf[warp][d] = x;
        sq += x * x;
    }
    const float *w = is_q ? a.q_norm : is_v ? nullptr : a.k_norm;
    float r = 1.0f;
    if (w) {
        for (int o = 16; o; o >>= 1) sq += __shfl_xor_sync(~0u, sq, o);
        r = rsqrtf(sq / (float)D + a.eps);
    }
    __syncwarp();
    if (!dst) return;
    const int half = a.rot >> 1;
    const float *cs = a.cos_sin + (size_t)min(max(pos, 0), max(a.n_pos - 1, 0)) * a.rot;
    for (int d = lane; d < D; d += 32) {
        auto y = [&](int i) { return w ? buf[warp][i] * r * __ldg(w + i) : buf[warp][i]; };
        float x = y(d);
        if (!is_v && d < a.rot) {
            const int i = a.interleaved ? d >> 1 : (d < half ? d : d - half);
            const bool second = a.interleaved ? d & 1 : d >= half;
            const float o = y(a.interleaved ? d ^ 1 : second ? d - half : d + half);
            const float c = __ldg(cs + i), sn = __ldg(cs + half + i);
            x = second ? x * c + o * sn : x * c - o * sn;
        }
        dst[d] = from_f32<T>(x);
    }
}

// ---- head sizes 64 and 128 in 16-byte pieces: E elements per lane, D / E lanes per head vector
//
// A warp takes one token and UNROLL x (vectors per warp) neighbouring heads: all loads are issued first, and the
// token's cosines and sines stay in registers for all of them.  The other element of a rotated pair lies in the same
// lane (PAIRS) or `mate` lanes away (mate = rot / 2 / E, a power of two), one shuffle per element.

constexpr int UNROLL = 8, FAST_WARPS = 4;  // 2 and 4 heads at a time: 185 and 162 us for the prompts that take 138 us with 8

template <typename T, int D, bool PAIRS>
__global__ void __launch_bounds__(32 * FAST_WARPS) append_vec_kernel(AppendArgs a, int chunks) {
    constexpr int E = 16 / (int)sizeof(T), LV = D / E, VW = 32 / LV;
    const View &v = a.v;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane / LV, i0 = (lane % LV) * E;
    const long long at = (long long)blockIdx.x * FAST_WARPS + warp;
    const int b = blockIdx.y, t = (int)(at / chunks), first = (int)(at - (long long)t * chunks) * (UNROLL * VW) + sub;
    const Seq s = seq_of(v, b);
    if (t >= s.nq) return;
    const size_t row = (size_t)s.row0 + t;
    const int slot = s.L - s.nq + t, heads = v.Hq + 2 * v.Hkv;
    union Piece {
        uint4 u;
        T t[E];
    } x[UNROLL];
    // rows shifted so that head hh of q, k and v together lies at hh * D
    const T *q_row = (const T *)a.q + row * a.q_stride + i0, *k_row = (const T *)a.k + row * a.k_stride + i0 - (size_t)v.Hq * D;
    const T *v_row = (const T *)a.vv + row * a.v_stride + i0 - (size_t)(v.Hq + v.Hkv) * D;
#pragma unroll
    for (int u = 0; u < UNROLL; u++) {
        const int hh = first + u * VW;
        const T *src = (hh < v.Hq ? q_row : hh < v.Hq + v.Hkv ? k_row : v_row) + hh * D;
        x[u].u = hh < heads ? __ldcs(reinterpret_cast<const uint4 *>(src)) : make_uint4(0, 0, 0, 0);
    }
    int page = -1;
    if (slot >= 0) {
        page = __ldg(v.table + (size_t)b * v.width + (slot >> v.page_shift));
        if ((unsigned)page >= (unsigned)v.n_pages) page = -1;
    }
    T *q_dst = (T *)a.q_out + row * a.q_out_stride + i0;
    const size_t in_pages = ((size_t)max(page, 0) * v.Hkv * v.page + (slot & (v.page - 1))) * D + i0;  // head 0's row of the slot
    const int head_step = v.page * D;
    T *k_dst = (T *)a.k_pages + in_pages - (size_t)v.Hq * head_step, *v_dst = (T *)a.v_pages + in_pages - (size_t)(v.Hq + v.Hkv) * head_step;
    const int pos = a.positions ? __ldg(a.positions + row) : slot;
    const int half = a.rot >> 1, mate = half / E;
    const bool turns = i0 < a.rot, second = !PAIRS && i0 >= half;
    float co[PAIRS ? E / 2 : E], si[PAIRS ? E / 2 : E];
    if (turns) {
        const float *cs = a.cos_sin + (size_t)min(max(pos, 0), a.n_pos - 1) * a.rot + (PAIRS ? i0 >> 1 : second ? i0 - half : i0);
#pragma unroll
        for (int e = 0; e < (PAIRS ? E / 2 : E); e += 2) {
            const float2 c2 = __ldg(reinterpret_cast<const float2 *>(cs + e)), s2 = __ldg(reinterpret_cast<const float2 *>(cs + half + e));
            co[e] = c2.x;
            co[e + 1] = c2.y;
            si[e] = s2.x;
            si[e + 1] = s2.y;
        }
    }
#pragma unroll
    for (int u = 0; u < UNROLL; u++) {
        const int hh = first + u * VW;
        const bool is_q = hh < v.Hq, is_v = hh >= v.Hq + v.Hkv;
        float y[E];
#pragma unroll
        for (int e = 0; e < E; e++) y[e] = to_f32(x[u].t[e]);
        const float *w = is_q ? a.q_norm : a.k_norm;
        if (a.q_norm || a.k_norm) {  // uniform; the lanes of one vector agree on w
            float sq = 0.0f;
#pragma unroll
            for (int e = 0; e < E; e++) sq += y[e] * y[e];
#pragma unroll
            for (int o = LV / 2; o; o >>= 1) sq += __shfl_xor_sync(~0u, sq, o);
            if (w && !is_v) {
                const float r = rsqrtf(sq * (1.0f / D) + a.eps);
#pragma unroll
                for (int e = 0; e < E; e += 4) {
                    const float4 g = __ldg(reinterpret_cast<const float4 *>(w + i0 + e));
                    y[e] *= r * g.x;
                    y[e + 1] *= r * g.y;
                    y[e + 2] *= r * g.z;
                    y[e + 3] *= r * g.w;
                }
            }
        }
        if (PAIRS) {
            if (turns && !is_v) {
#pragma unroll
                for (int e = 0; e < E; e += 2) {
                    const float p = y[e], q = y[e + 1];
                    y[e] = p * co[e / 2] - q * si[e / 2];
                    y[e + 1] = q * co[e / 2] + p * si[e / 2];
                }
            }
        } else if (a.rot) {
#pragma unroll
            for (int e = 0; e < E; e++) {
                const float o = __shfl_xor_sync(~0u, y[e], mate);
                if (turns && !is_v) y[e] = second ? y[e] * co[e] + o * si[e] : y[e] * co[e] - o * si[e];
            }
        }
        if (!is_v) {
#pragma unroll
            for (int e = 0; e < E; e++) x[u].t[e] = from_f32<T>(y[e]);
        }
        if (hh >= heads) continue;
        if (is_q) {
            *reinterpret_cast<uint4 *>(q_dst + hh * D) = x[u].u;
        } else if (page >= 0) {
            *reinterpret_cast<uint4 *>((is_v ? v_dst : k_dst) + (size_t)hh * head_step) = x[u].u;
        }
        if (!is_q && !is_v && i0 == 0 && slot >= 0) {
            const size_t i = ((size_t)b * v.Hkv + hh - v.Hq) * v.cap + slot;
            if (a.slot_pos) a.slot_pos[i] = pos;
            if (a.weight) a.weight[i] = 0.0f;
        }
    }
}

template <typename T, int D> cudaError_t append_vec(const AppendArgs &a, cudaStream_t s) {
    constexpr int E = 16 / (int)sizeof(T), VW = 32 / (D / E);
    const int heads = a.v.Hq + 2 * a.v.Hkv, chunks = (heads + UNROLL * VW - 1) / (UNROLL * VW);
    const dim3 grid((unsigned)(((long long)a.v.n_q * chunks + FAST_WARPS - 1) / FAST_WARPS), a.v.B);
    if (a.interleaved)
        append_vec_kernel<T, D, true><<<grid, 32 * FAST_WARPS, 0, s>>>(a, chunks);
    else
        append_vec_kernel<T, D, false><<<grid, 32 * FAST_WARPS, 0, s>>>(a, chunks);
    return cudaGetLastError();
}

// Can the vector kernel rotate by `rot` elements?  Whole pieces on both sides, and partners at a power of two.
bool vec_rotation(int rot, int interleaved, int E) {
    if (rot == 0) return true;
    if (interleaved) return rot % E == 0;
    const int mate = rot / 2 / E;
    return rot / 2 % E == 0 && mate > 0 && (mate & (mate - 1)) == 0;
}

}  // namespace

cudaError_t launch_append(const AppendArgs &a, bool bf16, cudaStream_t s) {
    const int heads = a.v.Hq + 2 * a.v.Hkv, D = a.v.D;
    if ((D == 64 || D == 128) && vec_rotation(a.rot, a.interleaved, bf16 ? 8 : 4)) {
        if (bf16) return D == 64 ? append_vec<__nv_bfloat16, 64>(a, s) : append_vec<__nv_bfloat16, 128>(a, s);
        return D == 64 ? append_vec<float, 64>(a, s) : append_vec<float, 128>(a, s);
    }
    const dim3 grid((unsigned)(((long long)a.v.n_q * heads + 3) / 4), a.v.B);
    if (bf16)
        append_any_kernel<__nv_bfloat16><<<grid, 128, 0, s>>>(a);
    else
        append_any_kernel<float><<<grid, 128, 0, s>>>(a);
    return cudaGetLastError();
}

}  // namespace kv
}  // namespace aj
