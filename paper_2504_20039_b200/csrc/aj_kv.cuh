// Declarations shared by the key-value cache kernels.
#pragma once

#include <cuda_bf16.h>

#include "aj_internal.cuh"

namespace aj {
namespace kv {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
// A running maximum (in units of log2) is left alone until a score exceeds it by this much: sums of 2^20 weights of 2^30
// are far from the end of f32's range.
constexpr float RAISE = 30.0f;

constexpr int MAX_CHUNKS = 16;  // of the slots that a batch shares

// What a call says about the cache and its new tokens (device pointers).
struct CacheView {
    const int *table = nullptr, *lens = nullptr, *q_start = nullptr;
    int B = 0, n_q = 0, width = 0, n_pages = 0, cap = 0;
    int Hq = 0, Hkv = 0, G = 0, D = 0, page = 0, page_shift = 0;
    int window = 0, sinks = 0;
};

// The same of a call whose sequences may share slots.  (Among every kernel's parameters these fields cost a single token's append 0.3 us of
// the host's time.)
struct View : CacheView {
    // A batch that shares its first slots (whole tiles of 128): the shared slots are cut into chunks, and `lead` chunks come before
    // the sequences, as sequences whose new tokens are those of the whole batch and see all of the chunk.  The sequences themselves
    // then begin behind the shared slots.  Each leaves its unnormalised results, for aj_kv_join.cu.
    int shared = 0, lead = 0, chunk = 0, n_chunks = 0;
    int behind = 0;  // slots before its new tokens of a sequence that shares: the whole tiles and what is shared of the next
    const int *lead_table = nullptr;
    int align = 0;  // places of the line that every piece takes and a CTA's share is a multiple of; 0: as many as it has
    int n_seq = 0, total = 0, pre_rows = 0;  // sequences; rows without q_start; rows that the results have room for
};

struct Seq {
    int row0, nq, L;  // first row of q, new tokens, slots in use
    int first = 0;    // slots below this one are left out
    int ahead = 0;    // new tokens sit this much further on than in the last nq slots
};

struct AttendArgs {
    View v;
    const void *q = nullptr, *k = nullptr, *vv = nullptr;
    void *out = nullptr;
    float *lse = nullptr;
    long long q_stride = 0, out_stride = 0;
    float scale_log2 = 0;        // scale * log2(e): scores are kept in units of log2
    float *pre = nullptr;        // unnormalised results of a shared call: [n_chunks + 1][Hkv][pre_rows * G][D], the last the sequences' own
    float2 *pre_ml = nullptr;    // their maxima and sums, [n_chunks][Hkv][pre_rows * G]
    float2 *own_ml = nullptr;    // the sequences' own, [rows][Hq]: a sum of -1 where a row has none
    float *parts = nullptr;      // partial results (unnormalised output, maximum, sum)
    unsigned *counters = nullptr;  // zero between launches: splits of an item that have arrived
    size_t parts_floats = 0;
    int n_counters = 0;
    int *status = nullptr;
};

struct WeighArgs {
    CacheView v;
    const void *q = nullptr, *k = nullptr;
    const float *lse = nullptr, *weight = nullptr;
    float *weight_out = nullptr;
    const int *n_rows = nullptr;
    long long q_stride = 0;
    float scale_log2 = 0;
    int *status = nullptr;
};

struct AppendArgs {
    CacheView v;
    const void *q = nullptr, *k = nullptr, *vv = nullptr;
    long long q_stride = 0, k_stride = 0, v_stride = 0, q_out_stride = 0;
    const float *q_norm = nullptr, *k_norm = nullptr, *cos_sin = nullptr;
    float eps = 0;
    int n_pos = 0, rot = 0, interleaved = 0;
    const int *positions = nullptr;
    void *k_pages = nullptr, *v_pages = nullptr, *q_out = nullptr;
    int *slot_pos = nullptr;
    float *weight = nullptr;
};

struct EvictArgs {
    CacheView v;
    void *k_pages = nullptr, *v_pages = nullptr;
    int keep = 0, sinks = 0, recent = 0, elem = 0;
    const float *weight = nullptr;
    const int *slot_pos = nullptr;
    int *lens_out = nullptr, *slot_pos_out = nullptr;
    float *weight_out = nullptr;
};

cudaError_t launch_append(const AppendArgs &a, bool bf16, cudaStream_t s);
cudaError_t launch_attend_simt(const AttendArgs &a, bool bf16, int num_sms, cudaStream_t s);
// few rows: at most FEW_ROWS = new tokens x query heads per key head; bf16, head size 64 or 128.  Both sides, at up to 8191
// slots of 64 sequences: 4 rows 170 us on mma.sync and 230 on tcgen05, 8 rows 222 and 294, 16 rows 207 and 245 (other
// lengths); 20 rows and more pass the registers of the first.  Accumulating the weight: 4 rows 74 and 82 us, 16 rows 85 and
// 87, 20 rows 90 and 88, 132 rows (8 sequences) 70 and 34.
constexpr int FEW_ROWS = 16;
// (of a shared call: as a programmatic dependent of the kernel over the shared slots, on num_sms SMs)
cudaError_t launch_attend_few(const AttendArgs &a, int num_sms, cudaStream_t s);
size_t few_parts_floats(int D, int num_sms);
// many rows: at most 128 query heads per key head; bf16, head size 64 or 128
// maps: K pages, V pages, queries in boxes of one token and of eight; q_tma: 0 if the queries have no maps, 1 if only boxes
// of one token fit a row tile, 8 if both do
cudaError_t launch_attend_umma(const AttendArgs &a, const CUtensorMap (&maps)[4], int q_tma, int num_sms, cudaStream_t s);
size_t umma_parts_floats(int D, int num_sms);
// joins the results of a shared call, as a programmatic dependent of the kernel before it
cudaError_t mark_now(float2 *own_ml, size_t n);
cudaError_t launch_join(const AttendArgs &a, cudaStream_t s);
cudaError_t launch_weigh_simt(const WeighArgs &a, bool bf16, cudaStream_t s);
cudaError_t launch_weigh_umma(const WeighArgs &a, const CUtensorMap &mk, int num_sms, cudaStream_t s);
cudaError_t launch_weigh_mma(const WeighArgs &a, int num_sms, cudaStream_t s);
cudaError_t launch_evict(const EvictArgs &a, unsigned *counters, const int (&clusters)[4], int num_sms, cudaStream_t s);

// For every handle, on its device: more than 48 KB of shared memory per CTA, and what eviction may ask for (a handle takes 0.6 ms).
cudaError_t prepare_attend_few();
cudaError_t prepare_attend_umma();
cudaError_t prepare_weigh_mma();
cudaError_t prepare_weigh_umma();
cudaError_t prepare_evict(int (&clusters)[4]);

// Sizes of the split-attention workspace that the CUDA-core kernels can use for this handle.
constexpr int SIMT_MAX_SPLITS = 64;
constexpr int SIMT_ROWS = 8;  // query rows a CTA of the CUDA-core kernels handles at once

#ifdef __CUDACC__

// A kernel may use all of the shared memory that its own static share leaves.
template <typename K> cudaError_t allow_shared(K kernel) {
    cudaFuncAttributes fa;
    const cudaError_t e = cudaFuncGetAttributes(&fa, kernel);
    if (e != cudaSuccess) return e;
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 232448 - (int)fa.sharedSizeBytes);
}

// The rows of a shared call: those of all sequences, as far as the results have room.
struct Rows {
    int base, n;
};
__device__ inline Rows rows_of(const View &v) {
    Rows r;
    r.base = v.q_start ? __ldg(v.q_start) : 0;
    r.n = min(max(v.q_start ? __ldg(v.q_start + v.n_seq) - r.base : v.total, 0), v.pre_rows);
    return r;
}
// Places of a row's results: chunk (or n_chunks for the sequence's own), key head, row of the call x query heads per key head.
__device__ inline float *pre_o(const AttendArgs &a, int chunk, int h, int rowg) {
    return a.pre + (((size_t)chunk * a.v.Hkv + h) * ((size_t)a.v.pre_rows * a.v.G) + rowg) * a.v.D;
}
__device__ inline float2 *pre_ml(const AttendArgs &a, int chunk, int h, int rowg) {
    return a.pre_ml + ((size_t)chunk * a.v.Hkv + h) * ((size_t)a.v.pre_rows * a.v.G) + rowg;
}

// SHARED: of a shared call, with its chunks.  (Asked of every call, this cost 1 to 18 % of others' time.)
template <bool SHARED = false, typename V> __device__ inline Seq seq_of(const V &v, int b) {
    Seq s;
    if constexpr (SHARED) {
        if (b < v.lead) {
            const Rows r = rows_of(v);
            s.row0 = r.base;
            s.nq = s.ahead = r.n;
            s.first = b * v.chunk;
            s.L = min(v.shared, s.first + v.chunk);
            return s;
        }
        b -= v.lead;
    }
    s.L = min(max(__ldg(v.lens + b), 0), v.cap);
    if (v.q_start) {
        s.row0 = __ldg(v.q_start + b);
        s.nq = min(max(__ldg(v.q_start + b + 1) - s.row0, 0), v.n_q);
    } else {
        s.row0 = b * v.n_q;
        s.nq = v.n_q;
    }
    if constexpr (SHARED) {  // a sequence that does not have all of the prefix before its new tokens, or no room for them, is on its own
        const Rows r = rows_of(v);
        if (s.L - s.nq >= v.behind && s.row0 >= r.base && s.nq <= r.n && s.row0 - r.base <= r.n - s.nq) s.first = v.shared;
    }
    return s;
}

// Number of the page that holds a slot; a number outside the pool reads page 0.
template <bool SHARED = false, typename V> __device__ inline int page_of(const V &v, int b, int slot) {
    const int *row;
    if constexpr (SHARED)
        row = b < v.lead ? v.lead_table : v.table + (size_t)(b - v.lead) * v.width;
    else
        row = v.table + (size_t)b * v.width;
    const int p = __ldg(row + (slot >> v.page_shift));
    return (unsigned)p < (unsigned)v.n_pages ? p : 0;
}

// Row of the pages, as [n_pages * Hkv * page_size, D], that holds a slot of a key head.
__device__ inline size_t page_row(const CacheView &v, int b, int h, int slot) {
    return ((size_t)page_of(v, b, slot) * v.Hkv + h) * v.page + (slot & (v.page - 1));
}

// Does the token in slot p see slot j?
__device__ inline bool sees(const CacheView &v, int p, int j) {
    return j <= p && (v.window == 0 || j > p - v.window || j < v.sinks);
}

template <typename T> __device__ inline float to_f32(T x);
template <> __device__ inline float to_f32<float>(float x) { return x; }
template <> __device__ inline float to_f32<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ inline T from_f32(float x);
template <> __device__ inline float from_f32<float>(float x) { return x; }
template <> __device__ inline __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

__device__ inline float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

#endif

}  // namespace kv
}  // namespace aj
