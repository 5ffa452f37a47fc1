// CUDA-core kernels of aj_kv_attend and aj_kv_weigh: f32 storage, and bf16 with a head size that the tensor-core
// kernels do not take.
//
//   s_j = scale * q k_j,  m = max s,  l = sum exp(s - m),  o = sum exp(s - m) v / l       one pass, running m and l
//
// A warp's lanes split the head; the warp takes 32 / R keys at a time for R query rows of one key head, so that
// one transposing butterfly leaves exactly one (key, row) score in each lane: 31 shuffles per 32 scores where
// reducing each by itself would take 160.  Warps of a CTA take keys in turn, and CTAs take pieces of the
// key range; a piece's unnormalised result goes to the workspace and the piece that arrives last joins them in the
// order of the pieces, so the bits do not depend on the order of arrival.
//
// Measured: one token against 1037 f32 slots of 8 key heads (4.3 MB): 10 us, of which the launch is most.
// Where bf16 can go to the tensor cores it does: 64 sequences of up to 8191 slots, 4 rows, 780 us here and 170 there; windows
// of 132 rows 10.1 ms and 0.15; weights of 4 rows 382 and 74 us, of 132 rows 390 and 34.
#include "aj_kv.cuh"

namespace aj {
namespace kv {

namespace {

constexpr int WARPS = 8;

// Values 0..31 of every lane, summed over the lanes; lane l gets the sum of value l.
__device__ inline float transposed_sum(float (&v)[32]) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) {
        const bool up = lane & o;
#pragma unroll
        for (int i = 0; i < o; i++) {
            const float send = up ? v[i] : v[i + o], stay = up ? v[i + o] : v[i];
            v[i] = stay + __shfl_xor_sync(~0u, send, o);
        }
    }
    return v[0];
}

// This lane's NE elements of a row: NE consecutive ones where the row is exactly 32 * NE long (VEC), else every 32nd.
template <typename T, int NE, bool VEC> __device__ inline void load_part(const T *row, int D, float (&x)[NE]) {
    const int lane = threadIdx.x & 31;
    if (VEC) {
        constexpr int BYTES = NE * (int)sizeof(T);
        union {
            T t[NE];
            uint32_t u[BYTES / 4];
        } r;
        const T *p = row + lane * NE;
        if constexpr (BYTES >= 16) {
#pragma unroll
            for (int i = 0; i < BYTES / 16; i++) *reinterpret_cast<uint4 *>(r.u + 4 * i) = __ldg(reinterpret_cast<const uint4 *>(p) + i);
        } else if constexpr (BYTES == 8) {
            *reinterpret_cast<uint2 *>(r.u) = __ldg(reinterpret_cast<const uint2 *>(p));
        } else {
            r.u[0] = __ldg(reinterpret_cast<const uint32_t *>(p));
        }
#pragma unroll
        for (int i = 0; i < NE; i++) x[i] = to_f32(r.t[i]);
    } else {
#pragma unroll
        for (int i = 0; i < NE; i++) x[i] = lane + 32 * i < D ? to_f32(__ldg(row + lane + 32 * i)) : 0.0f;
    }
}
template <int NE, bool VEC> __device__ inline int elem_at(int i) {
    const int lane = threadIdx.x & 31;
    return VEC ? lane * NE + i : lane + 32 * i;
}

template <typename T, int NE, bool VEC, int R>
__global__ void __launch_bounds__(32 * WARPS) attend_simt_kernel(AttendArgs a, int n_rb, int splits) {
    constexpr int KS = 32 / R;  // keys a warp takes at a time
    extern __shared__ float sm[];
    const CacheView &v = a.v;
    const int D = v.D, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int item = blockIdx.x, split = blockIdx.y;
    const int rb = item % n_rb, h = (item / n_rb) % v.Hkv, b = item / (n_rb * v.Hkv);
    const Seq s = seq_of(v, b);
    const int n_rows = min(R, s.nq * v.G - rb * R);
    if (n_rows <= 0) return;
    const int t_lo = (rb * R) / v.G, t_hi = (rb * R + n_rows - 1) / v.G;
    const int p_lo = s.L - s.nq + t_lo, p_hi = s.L - s.nq + t_hi;
    // visible slots of these rows: the sinks before the window's reach, then first .. p_hi
    const int first = v.window ? max(0, p_lo - v.window + 1) : 0;
    const int n_sink = min(v.sinks, first);
    const int total = n_sink + max(0, p_hi + 1 - first);
    const int chunk = max((total + splits - 1) / splits, WARPS * KS);
    const int used = max(1, (total + chunk - 1) / chunk);
    if (split >= used) return;
    const int u0 = split * chunk, u1 = min(total, u0 + chunk);

    float q[R][NE], o[R][NE];
#pragma unroll
    for (int r = 0; r < R; r++) {
#pragma unroll
        for (int i = 0; i < NE; i++) q[r][i] = o[r][i] = 0.0f;
        if (r < n_rows) {
            const int idx = rb * R + r;
            load_part<T, NE, VEC>((const T *)a.q + ((size_t)s.row0 + idx / v.G) * a.q_stride + (size_t)(h * v.G + idx % v.G) * D, D, q[r]);
        }
    }
    const int my_r = lane % R, my_k = lane / R;  // the (key, row) whose score this lane holds
    const int my_p = s.L - s.nq + (rb * R + my_r) / v.G;
    float m = -INFINITY, l = 0.0f;
    const T *kp = (const T *)a.k, *vp = (const T *)a.vv;

    for (int u = u0 + warp * KS; u < u1; u += WARPS * KS) {
        const int j = u + my_k < n_sink ? u + my_k : u + my_k - n_sink + first;
        const bool in = u + my_k < u1;
        size_t row = in ? page_row(v, b, h, j) : 0;
        float kk[KS][NE], vv[KS][NE];
#pragma unroll
        for (int i = 0; i < KS; i++) {
            const size_t ri = __shfl_sync(~0u, (unsigned long long)row, i * R);
            const bool ok = u + i < u1;
            if (ok) {
                load_part<T, NE, VEC>(kp + ri * D, D, kk[i]);
                load_part<T, NE, VEC>(vp + ri * D, D, vv[i]);
            } else {
#pragma unroll
                for (int e = 0; e < NE; e++) kk[i][e] = vv[i][e] = 0.0f;
            }
        }
        float part[32];
#pragma unroll
        for (int i = 0; i < KS; i++)
#pragma unroll
            for (int r = 0; r < R; r++) {
                float x = 0.0f;
#pragma unroll
                for (int e = 0; e < NE; e++) x = fmaf(q[r][e], kk[i][e], x);
                part[i * R + r] = x;
            }
        const float dot = transposed_sum(part);
        const float sc = in && my_r < n_rows && sees(v, my_p, j) ? dot * a.scale_log2 : -INFINITY;
        float mx = sc;
#pragma unroll
        for (int off = R; off < 32; off <<= 1) mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, off));
        const float m_new = fmaxf(m, mx);
        const float base = m_new == -INFINITY ? 0.0f : m_new;
        const float corr = exp2f(m - base), p = exp2f(sc - base);
        l = l * corr + p;
        m = m_new;
        if (__any_sync(~0u, corr != 1.0f)) {
#pragma unroll
            for (int r = 0; r < R; r++) {
                const float c = __shfl_sync(~0u, corr, r);
#pragma unroll
                for (int e = 0; e < NE; e++) o[r][e] *= c;
            }
        }
#pragma unroll
        for (int i = 0; i < KS; i++)
#pragma unroll
            for (int r = 0; r < R; r++) {
                const float c = __shfl_sync(~0u, p, i * R + r);
                // a weight of zero leaves the value out altogether: a masked slot may hold NaN
#pragma unroll
                for (int e = 0; e < NE; e++) o[r][e] = c != 0.0f ? fmaf(c, vv[i][e], o[r][e]) : o[r][e];
            }
    }
#pragma unroll
    for (int off = R; off < 32; off <<= 1) l += __shfl_xor_sync(~0u, l, off);

    // join the warps: sm = [WARPS][R][D] outputs, then [WARPS][R] maxima and sums
    float *sm_m = sm + WARPS * R * D, *sm_l = sm_m + WARPS * R;
#pragma unroll
    for (int r = 0; r < R; r++)
#pragma unroll
        for (int e = 0; e < NE; e++) {
            const int d = elem_at<NE, VEC>(e);
            if (d < D) sm[(warp * R + r) * D + d] = o[r][e];
        }
    if (lane < R) {
        sm_m[warp * R + lane] = m;
        sm_l[warp * R + lane] = l;
    }
    __syncthreads();

    auto store = [&](int r, int d, float x, float mm, float ll) {
        const int idx = rb * R + r;
        const size_t row = (size_t)s.row0 + idx / v.G;
        const int head = h * v.G + idx % v.G;
        ((T *)a.out)[row * a.out_stride + (size_t)head * D + d] = from_f32<T>(ll == 0.0f ? 0.0f : x / ll);  // a sum that is NaN stays one
        if (d == 0 && a.lse) a.lse[row * v.Hq + head] = ll == 0.0f ? -INFINITY : (mm + log2f(ll)) * LN2;
    };
    const int stride = R * (D + 2);
    float *mine = a.parts + ((size_t)item * splits + split) * stride;
    for (int i = threadIdx.x; i < n_rows * D; i += blockDim.x) {
        const int r = i / D, d = i - r * D;
        float mm = -INFINITY, ll = 0.0f, x = 0.0f;
        for (int w = 0; w < WARPS; w++) mm = fmaxf(mm, sm_m[w * R + r]);
        const float base = mm == -INFINITY ? 0.0f : mm;
        for (int w = 0; w < WARPS; w++) {
            const float c = exp2f(sm_m[w * R + r] - base);
            ll += c * sm_l[w * R + r];
            x += c * sm[(w * R + r) * D + d];
        }
        if (used == 1) {
            store(r, d, x, mm, ll);
        } else {
            mine[r * D + d] = x;
            if (d == 0) {
                mine[R * D + r] = mm;
                mine[R * D + R + r] = ll;
            }
        }
    }
    if (used == 1) return;
    __shared__ int last;
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) last = atomicAdd(a.counters + item, 1u) == (unsigned)used - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
    const float *parts = a.parts + (size_t)item * splits * stride;
    for (int i = threadIdx.x; i < n_rows * D; i += blockDim.x) {
        const int r = i / D, d = i - r * D;
        float mm = -INFINITY, ll = 0.0f, x = 0.0f;
        for (int w = 0; w < used; w++) mm = fmaxf(mm, __ldcg(parts + w * stride + R * D + r));
        const float base = mm == -INFINITY ? 0.0f : mm;
        for (int w = 0; w < used; w++) {
            const float c = exp2f(__ldcg(parts + w * stride + R * D + r) - base);
            ll += c * __ldcg(parts + w * stride + R * D + R + r);
            x += c * __ldcg(parts + w * stride + r * D + d);
        }
        store(r, d, x, mm, ll);
    }
    if (threadIdx.x == 0) a.counters[item] = 0u;
}

template <typename T, int NE, bool VEC>
__global__ void __launch_bounds__(32 * WARPS) weigh_simt_kernel(WeighArgs a) {
    constexpr int R = 8, KS = 4;
    const CacheView &v = a.v;
    const int D = v.D, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int h = blockIdx.y % v.Hkv, b = blockIdx.y / v.Hkv;
    const Seq s = seq_of(v, b);
    const int counted = min(s.nq, a.n_rows ? max(__ldg(a.n_rows + b), 0) : s.nq) * v.G;
    const int my_r = lane % R, my_k = lane / R;
    for (int j0 = (blockIdx.x * WARPS + warp) * KS; j0 < s.L; j0 += gridDim.x * WARPS * KS) {
        const int j = j0 + my_k;
        const size_t row = j < s.L ? page_row(v, b, h, j) : 0;
        float kk[KS][NE];
#pragma unroll
        for (int i = 0; i < KS; i++) {
            const size_t ri = __shfl_sync(~0u, (unsigned long long)row, i * R);
            if (j0 + i < s.L)
                load_part<T, NE, VEC>((const T *)a.k + ri * D, D, kk[i]);
            else
#pragma unroll
                for (int e = 0; e < NE; e++) kk[i][e] = 0.0f;
        }
        float sum = 0.0f;
        for (int r0 = 0; r0 < counted; r0 += R) {
            float part[32];
#pragma unroll
            for (int r = 0; r < R; r++) {
                float q[NE];
                const int idx = min(r0 + r, counted - 1);
                load_part<T, NE, VEC>((const T *)a.q + ((size_t)s.row0 + idx / v.G) * a.q_stride + (size_t)(h * v.G + idx % v.G) * D, D, q);
#pragma unroll
                for (int i = 0; i < KS; i++) {
                    float x = 0.0f;
#pragma unroll
                    for (int e = 0; e < NE; e++) x = fmaf(q[e], kk[i][e], x);
                    part[i * R + r] = x;
                }
            }
            const float dot = transposed_sum(part);
            const int idx = min(r0 + my_r, counted - 1), t = idx / v.G;
            const float ls = __ldg(a.lse + ((size_t)s.row0 + t) * v.Hq + h * v.G + idx % v.G);
            if (r0 + my_r < counted && j < s.L && ls != -INFINITY && sees(v, s.L - s.nq + t, j))
                sum += exp2f(fmaf(dot, a.scale_log2, -ls * LOG2E));
        }
#pragma unroll
        for (int off = 1; off < R; off <<= 1) sum += __shfl_xor_sync(~0u, sum, off);
        if (my_r == 0 && j < s.L) {
            const size_t at = ((size_t)b * v.Hkv + h) * v.cap + j;
            a.weight_out[at] = a.weight[at] + sum;
        }
    }
}

template <typename T, int NE, bool VEC, int R> cudaError_t attend_rows(const AttendArgs &a, int num_sms, cudaStream_t s) {
    const int n_rb = (a.v.n_q * a.v.G + R - 1) / R;
    const long long items = (long long)a.v.B * a.v.Hkv * n_rb;
    // enough pieces that the CTAs of a few waves even out sequences of different length; no piece under 64 slots
    long long splits = (6LL * num_sms + items - 1) / items;
    const long long most = (a.v.cap + 63) / 64;
    splits = splits < 1 ? 1 : splits > most ? most : splits;
    if (splits > SIMT_MAX_SPLITS) splits = SIMT_MAX_SPLITS;
    while (splits > 1 && (size_t)(items * splits) * R * (a.v.D + 2) > a.parts_floats) splits--;
    if (splits > 1 && items > a.n_counters) splits = 1;
    const size_t smem = (size_t)WARPS * R * (a.v.D + 2) * sizeof(float);
    auto kernel = attend_simt_kernel<T, NE, VEC, R>;
    if (smem > 48 * 1024) {
        cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
    }
    kernel<<<dim3((unsigned)items, (unsigned)splits), 32 * WARPS, smem, s>>>(a, n_rb, (int)splits);
    return cudaGetLastError();
}

template <typename T, int NE, bool VEC> cudaError_t attend_any(const AttendArgs &a, int num_sms, cudaStream_t s) {
    return a.v.n_q * a.v.G <= 4 ? attend_rows<T, NE, VEC, 4>(a, num_sms, s) : attend_rows<T, NE, VEC, 8>(a, num_sms, s);
}

template <typename T, int NE, bool VEC> cudaError_t weigh_any(const WeighArgs &a, cudaStream_t s) {
    const int per = WARPS * 4;
    weigh_simt_kernel<T, NE, VEC><<<dim3((unsigned)((a.v.cap + per - 1) / per), a.v.B * a.v.Hkv), 32 * WARPS, 0, s>>>(a);
    return cudaGetLastError();
}

}  // namespace

// The element count per lane is a template argument; rows of exactly 64, 128 or 256 elements load as vectors.
#define AJ_KV_BY_HEAD(T, FN, ...)                                       \
    switch (a.v.D) {                                                    \
        case 64: return FN<T, 2, true>(__VA_ARGS__);                    \
        case 128: return FN<T, 4, true>(__VA_ARGS__);                   \
        default: break;                                                 \
    }                                                                   \
    if (a.v.D <= 64) return FN<T, 2, false>(__VA_ARGS__);               \
    if (a.v.D <= 128) return FN<T, 4, false>(__VA_ARGS__);              \
    return FN<T, 8, false>(__VA_ARGS__);

cudaError_t launch_attend_simt(const AttendArgs &a, bool bf16, int num_sms, cudaStream_t s) {
    if (bf16) {
        AJ_KV_BY_HEAD(__nv_bfloat16, attend_any, a, num_sms, s)
    }
    AJ_KV_BY_HEAD(float, attend_any, a, num_sms, s)
}

cudaError_t launch_weigh_simt(const WeighArgs &a, bool bf16, cudaStream_t s) {
    if (bf16) {
        AJ_KV_BY_HEAD(__nv_bfloat16, weigh_any, a, s)
    }
    AJ_KV_BY_HEAD(float, weigh_any, a, s)
}

}  // namespace kv
}  // namespace aj
