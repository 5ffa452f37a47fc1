// Norms of queries and keys per head, position rotation, and the write of new tokens into the cache's pages.
//
//   y = x * rsqrt(mean(x^2) + eps) * w,   (a, b) -> (a cos - b sin, b cos + a sin) per rotated pair,
// in 32 bits with one rounding on the store.  The pass reads and writes (Hq + 2 Hkv) * D elements per token and
// nothing else of that size, so it is bound by memory.
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

}  // namespace

cudaError_t launch_append(const AppendArgs &a, bool bf16, cudaStream_t s) {
    const int heads = a.v.Hq + 2 * a.v.Hkv;
    const dim3 grid((unsigned)(((long long)a.v.n_q * heads + 3) / 4), a.v.B);
    if (bf16)
        append_any_kernel<__nv_bfloat16><<<grid, 128, 0, s>>>(a);
    else
        append_any_kernel<float><<<grid, 128, 0, s>>>(a);
    return cudaGetLastError();
}

}  // namespace kv
}  // namespace aj
