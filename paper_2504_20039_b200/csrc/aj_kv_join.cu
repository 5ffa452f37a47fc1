// aj_kv_attend_shared, last step: a row's results over the chunks of the shared slots and over its sequence's own slots, joined.
//
//   m = max m_c,  out = sum e^(m_c - m) O_c / sum e^(m_c - m) l_c,  lse = m + log of that sum
//
// A warp per (row, query head).  Lane c holds the maximum and sum of part c, so the weights cost one exponential and a few
// shuffles; then each lane adds up its D / 32 elements, all parts in flight at once.  Bound by latency for few rows, by the parts' bytes
// in L2 for many.  Measured: 2048 rows x heads of 4 parts 6 us, 33792 of 2 parts 15 to 20.  A row without a part of its own (a sequence that is not behind the shared slots) has its result
// already and is left alone; the mark that says so is put back for the next call.
#include "aj_kv.cuh"

namespace aj {
namespace kv {

namespace {

constexpr int WARPS = 8;

template <int D> __global__ void __launch_bounds__(32 * WARPS) join_kernel(AttendArgs a) {
    constexpr int E = D / 32;
    const View &v = a.v;
    const int lane = threadIdx.x & 31, n = v.n_chunks;
    const long long id = (long long)blockIdx.x * WARPS + (threadIdx.x >> 5);
    const int row = (int)(id / v.Hq), head = (int)(id - (long long)row * v.Hq), h = head / v.G, rowg = row * v.G + head - h * v.G;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const Rows rows = rows_of(v);
    if (row >= rows.n) return;
    float2 *own = a.own_ml + (size_t)row * v.Hq + head;
    float2 ml = make_float2(-INFINITY, 0.0f);
    if (lane < n) ml = *pre_ml(a, lane, h, rowg);
    if (lane == n) ml = *own;
    if (__shfl_sync(~0u, ml.y, n) == -1.0f) return;
    if (lane == n) own->y = -1.0f;
    float m = ml.x;
#pragma unroll
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, o));
    const float ref = m == -INFINITY ? 0.0f : m, w = lane <= n ? ex2(ml.x - ref) : 0.0f;  // a part that is NaN makes the sum NaN
    float l = lane <= n ? w * ml.y : 0.0f;
#pragma unroll
    for (int o = 16; o; o >>= 1) l += __shfl_xor_sync(~0u, l, o);
    float y[E] = {};
#pragma unroll 4
    for (int c = 0; c <= n; c++) {
        const float *p = pre_o(a, c, h, rowg) + lane * E;
        const float wc = __shfl_sync(~0u, w, c);
        if constexpr (E == 4) {
            const float4 f = *reinterpret_cast<const float4 *>(p);
            y[0] += wc * f.x, y[1] += wc * f.y, y[2] += wc * f.z, y[3] += wc * f.w;
        } else {
            const float2 f = *reinterpret_cast<const float2 *>(p);
            y[0] += wc * f.x, y[1] += wc * f.y;
        }
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    const size_t at = (size_t)rows.base + row;
    __nv_bfloat16 *o = (__nv_bfloat16 *)a.out + at * a.out_stride + (size_t)head * D + lane * E;
    if constexpr (E == 4) {
        const __nv_bfloat162 p = __floats2bfloat162_rn(y[0] * inv, y[1] * inv), q = __floats2bfloat162_rn(y[2] * inv, y[3] * inv);
        *reinterpret_cast<uint2 *>(o) = make_uint2(*reinterpret_cast<const uint32_t *>(&p), *reinterpret_cast<const uint32_t *>(&q));
    } else {
        *reinterpret_cast<__nv_bfloat162 *>(o) = __floats2bfloat162_rn(y[0] * inv, y[1] * inv);
    }
    if (lane == 0 && a.lse) a.lse[at * v.Hq + head] = l == 0.0f ? -INFINITY : (m + log2f(l)) * LN2;
}

__global__ void mark_kernel(float2 *own_ml, size_t n) {
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i < n) own_ml[i] = make_float2(0.0f, -1.0f);
}

}  // namespace

// Every row without a part of its own, on return and for every stream: a sum whose bytes are those of -1.
cudaError_t mark_now(float2 *own_ml, size_t n) {
    cudaStream_t s;
    cudaError_t e = cudaStreamCreateWithFlags(&s, cudaStreamNonBlocking);
    if (e != cudaSuccess) return e;
    mark_kernel<<<(unsigned)((n + 255) / 256), 256, 0, s>>>(own_ml, n);
    e = cudaGetLastError();
    const cudaError_t e2 = cudaStreamSynchronize(s);
    cudaStreamDestroy(s);
    return e != cudaSuccess ? e : e2;
}

cudaError_t launch_join(const AttendArgs &a, cudaStream_t s) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(((long long)a.v.pre_rows * a.v.Hq + WARPS - 1) / WARPS));
    cfg.blockDim = dim3(32 * WARPS);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return a.v.D == 64 ? cudaLaunchKernelEx(&cfg, join_kernel<64>, a) : cudaLaunchKernelEx(&cfg, join_kernel<128>, a);
}

}  // namespace kv
}  // namespace aj
