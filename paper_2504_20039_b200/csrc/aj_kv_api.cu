// Host side of the key-value cache operators: argument checks, the handle's workspace, choice of kernel, launches.
// No call synchronises or allocates but aj_kv_create, aj_kv_destroy, aj_kv_reserve_shared and aj_kv_last_status.
#include "../../include/aj_kv.h"

#include <new>

#include "aj_kv.cuh"

using namespace aj;

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                  const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
typedef CUresult (*ReplaceAddressFn)(CUtensorMap *, void *);

struct aj_kv_s {
    int device = 0, num_sms = 0;
    int max_B = 0, max_q = 0, Hq = 0, Hkv = 0, D = 0, page = 0, page_shift = 0, dtype = 0;
    unsigned flags = 0;
    bool tensor = false;           // bf16 and a head size that the tensor-core kernels take
    float *parts = nullptr;
    size_t parts_floats = 0;
    unsigned *counters = nullptr;  // [n_counters] attention items, then [max_B] eviction
    int n_counters = 0;
    int *status = nullptr;
    // aj_kv_reserve_shared: results of a shared call's parts, and partial results and arrivals of the kernel over the shared slots
    float *pre = nullptr, *pre_parts = nullptr;
    float2 *pre_ml = nullptr, *own_ml = nullptr;
    unsigned *pre_counters = nullptr;
    int pre_rows = 0;
    int clusters[4] = {};          // see prepare_evict
    EncodeTiledFn encode = nullptr;
    ReplaceAddressFn replace = nullptr;
    // tensor maps of pages, and of query rows of stride q_stride in boxes of one token and of eight: a call puts its addresses in
    CUtensorMap pages = {}, rows1 = {}, rows8 = {};
    long long q_stride = -1;
    int last_launches = 0;
    const char *last_path = "none";
};

namespace {

class Guard {  // the handle's device for the duration of a call
   public:
    explicit Guard(int dev) {
        if (cudaGetDevice(&prev_) != cudaSuccess) prev_ = -1;
        if (prev_ != dev) ok_ = cudaSetDevice(dev) == cudaSuccess;
        changed_ = ok_ && prev_ != dev;
    }
    ~Guard() {
        if (changed_ && prev_ >= 0) cudaSetDevice(prev_);
    }
    bool ok() const { return ok_; }

   private:
    int prev_ = -1;
    bool ok_ = true, changed_ = false;
};

bool off16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }
bool on128(const void *p, long long stride_bytes = 0) { return ((reinterpret_cast<uintptr_t>(p) | (uintptr_t)stride_bytes) & 127) == 0; }

// What every call has in common.
aj_status check_view(aj_kv h, const void *pages, int n_pages, const int32_t *table, int width, const int32_t *lens, int B,
                     int n_q) {
    if (!h || !pages || !table || !lens) return AJ_ERR_INVALID_ARG;
    if (B < 1 || n_q < 1 || n_pages < 1 || width < 1) return AJ_ERR_INVALID_ARG;
    if ((long long)n_pages * h->Hkv * h->page > 0x7fffffffll || (long long)width * h->page > (1ll << 20)) return AJ_ERR_UNSUPPORTED;
    if (B > h->max_B || n_q > h->max_q) return AJ_ERR_WORKSPACE;
    if (off16(pages)) return AJ_ERR_UNSUPPORTED;
    return AJ_OK;
}

// A row stride: at least the heads, and whole 16-byte pieces.
aj_status check_rows(aj_kv h, const void *p, long long stride, int heads) {
    if (!p || stride < (long long)heads * h->D) return AJ_ERR_INVALID_ARG;
    const int e = h->dtype == AJ_BF16 ? 2 : 4;
    if (off16(p) || (stride * e) % 16 != 0) return AJ_ERR_UNSUPPORTED;
    return AJ_OK;
}

kv::CacheView view_of(aj_kv h, int n_pages, const int32_t *table, int width, const int32_t *lens, const int32_t *q_start, int B,
                 int n_q, int window, int sinks) {
    kv::CacheView v;
    v.table = table;
    v.lens = lens;
    v.q_start = q_start;
    v.B = B;
    v.n_q = n_q;
    v.width = width;
    v.n_pages = n_pages;
    v.cap = width * h->page;
    v.Hq = h->Hq;
    v.Hkv = h->Hkv;
    v.G = h->Hq / h->Hkv;
    v.D = h->D;
    v.page = h->page;
    v.page_shift = h->page_shift;
    // a window as long as the cache hides nothing (positions minus a window must not wrap, below a first slot either)
    v.window = window < v.cap ? window : 0;
    v.sinks = sinks < v.cap ? sinks : v.cap;
    return v;
}

// A tensor map of pages as rows of D elements, boxes of 64 elements x one page, 128-byte swizzle.  Page numbers are checked
// in the kernels, so the map's row count is only an upper bound; the address is put in by each call.
bool encode_pages(aj_kv h, void *any) {
    const cuuint64_t dims[2] = {(cuuint64_t)h->D, 0x7fffffff};
    const cuuint64_t strides[1] = {(cuuint64_t)h->D * 2};
    const cuuint32_t box[2] = {64, (cuuint32_t)h->page}, one[2] = {1, 1};
    return h->encode(&h->pages, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, any, dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                     CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// A tensor map of query rows as [rows, Hq, D], boxes of 64 elements x the heads of one key head x `tokens`.  How many rows
// exist is known on the device only; no copy goes past a sequence's own.
bool encode_rows(aj_kv h, CUtensorMap *m, void *any, long long stride, int tokens) {
    const cuuint64_t dims[3] = {(cuuint64_t)h->D, (cuuint64_t)h->Hq, 1u << 30};
    const cuuint64_t strides[2] = {(cuuint64_t)h->D * 2, (cuuint64_t)stride * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)(h->Hq / h->Hkv), (cuuint32_t)tokens}, one[3] = {1, 1, 1};
    return h->encode(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, any, dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                     CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool at_address(aj_kv h, CUtensorMap *m, const CUtensorMap &from, const void *p) {
    *m = from;
    return h->replace(m, const_cast<void *>(p)) == CUDA_SUCCESS;
}

kv::AttendArgs attend_args(aj_kv h, const void *q, long long q_stride, const void *k_pages, const void *v_pages, float scale, void *out,
                           long long out_stride, float *lse) {
    kv::AttendArgs a;
    a.q = q;
    a.q_stride = q_stride;
    a.k = k_pages;
    a.vv = v_pages;
    a.out = out;
    a.out_stride = out_stride;
    a.lse = lse;
    a.scale_log2 = scale * kv::LOG2E;
    a.parts = h->parts;
    a.parts_floats = h->parts_floats;
    a.counters = h->counters;
    a.n_counters = h->n_counters;
    a.status = h->status;
    return a;
}

// The tensor maps of a call of the tcgen05 kernel.
bool attend_maps(aj_kv h, const kv::AttendArgs &a, CUtensorMap (&maps)[4], int *q_tma) {
    if (!at_address(h, &maps[0], h->pages, a.k) || !at_address(h, &maps[1], h->pages, a.vv)) return false;
    // queries by TMA (boxes of eight tokens where a tile has as many, and of one), or by one warp's 16-byte copies where their
    // rows do not lie on 128 bytes: 64 windows of 33 rows 157 us and 209, a prompt of 8192 490 and 647
    const int tma = *q_tma = !on128(a.q, a.q_stride * 2) ? 0 : 128 / a.v.G >= 8 ? 8 : 1;
    if (tma && a.q_stride != h->q_stride) {
        h->q_stride = -1;
        if (!encode_rows(h, &h->rows1, h->parts, a.q_stride, 1) || (tma == 8 && !encode_rows(h, &h->rows8, h->parts, a.q_stride, 8))) return false;
        h->q_stride = a.q_stride;
    }
    return !tma || (at_address(h, &maps[2], h->rows1, a.q) && (tma != 8 || at_address(h, &maps[3], h->rows8, a.q)));
}

// Into how many chunks the shared slots are cut.  An item is a chunk, a key head and a piece of up to 256 query rows.  With few
// rows per sequence, chunks of six tiles on up to half of the SMs, while the sequences' own slots are attended on the others (64 tokens
// behind 2048 slots: 32 to 38 us, with every SM for one and then the other 62); else as many items as there are SMs, so that hardly
// one spans CTAs, which costs a join by one CTA.  Returns the CTAs for it.
int cut_shared(kv::View &v, int num_sms) {
    const int tiles = v.shared / 128, per_piece = 2 * (128 / v.G);
    const long long items = (long long)v.Hkv * ((v.pre_rows + per_piece - 1) / per_piece);
    const bool few = v.n_q * v.G <= kv::FEW_ROWS;
    const int most = few ? num_sms / 2 : num_sms;
    int n = items < most ? (int)(most / items) : 1;
    if (few && n > (tiles + 5) / 6) n = (tiles + 5) / 6;
    if (n > kv::MAX_CHUNKS) n = kv::MAX_CHUNKS;
    const int each = (tiles + n - 1) / n;
    v.chunk = each * 128;
    v.n_chunks = (tiles + each - 1) / each;
    return (int)(items * v.n_chunks < most ? items * v.n_chunks : most);
}
// Is it worth the parts and their join?  Sequences that share pages read them from L2 when they are attended one by one, so what is
// saved is the stream from L2 (few rows: at 5.9 TB/s, against 8 us and 1.5 for each tile of a chunk, at a head size of 128), or row tiles
// that a window does not fill (more rows: 10 ns a tile, against 4 us and 0.8 ns for each row and head, whose parts go through L2; half of
// that at 64).  Measured, us, together and one by one, 32 query and 8 key heads of 128: 64 tokens behind 2048 slots 32 and 80, behind 512 29 and 35,
// behind 256 26 and 27; 16 behind 4096 24 and 43, behind 1024 19 and 21; 2 behind 32768 61 and 48; 32 windows of 9 rows behind 2048 52 and
// 70, 16 of 33 behind 8192 108 and 134, 32 of 33 behind 1504 86 and 74; heads of 64: 16 tokens behind 4096 22 and 34, 32 windows of 33
// behind 1504 72 and 66; 64 query heads: 32 of 33 behind 1504 147 and 118, 16 behind 8192 188 and 219.  Over 1584 calls of twelve
// head counts, both sizes, 1 to 384 rows, 700 of them not looked at before: within 1 % of the better way on average, more than 8 % above it in 55.
bool worth_sharing(const kv::View &v) {
    const double size = v.D / 128.0;
    if (v.n_q * v.G <= kv::FEW_ROWS) return (double)v.n_seq * v.shared * v.Hkv * v.D * 4 / 5.9e6 > 8 + 1.5 * (v.chunk / 128) * size;
    const long long per_piece = 2 * (128 / v.G), together = (v.pre_rows + per_piece - 1) / per_piece;
    // (of a ragged batch the host knows the sum at most: half a piece more for each sequence)
    const long long one_by_one = v.q_start ? together + v.n_seq / 2 : v.n_seq * ((v.n_q + per_piece - 1) / per_piece);
    return 0.010 * (double)((one_by_one - together) * v.Hkv * (v.shared / 128)) > 4 + 0.0008 * (double)v.pre_rows * v.Hq * size;
}
// Rows x chunks that a workspace for max_rows rows must hold.
int pre_capacity(aj_kv h, int max_rows) {
    const int few = 2 * (128 * h->Hkv / h->Hq) * (h->num_sms / h->Hkv + 1);
    return max_rows > few ? max_rows : few;
}

void free_shared(aj_kv h) {
    cudaFree(h->pre);
    cudaFree(h->pre_ml);
    cudaFree(h->own_ml);
    cudaFree(h->pre_parts);
    cudaFree(h->pre_counters);
    h->pre = h->pre_parts = nullptr;
    h->pre_ml = h->own_ml = nullptr;
    h->pre_counters = nullptr;
    h->pre_rows = 0;
}

// What the tcgen05 kernels need beside the handle's workspace.
bool prepare_maps(aj_kv h) {
    void *fn = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess || !fn)
        return false;
    h->encode = reinterpret_cast<EncodeTiledFn>(fn);
    if (cudaGetDriverEntryPointByVersion("cuTensorMapReplaceAddress", &fn, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess || !fn)
        return false;
    h->replace = reinterpret_cast<ReplaceAddressFn>(fn);
    return true;
}

aj_status done(cudaError_t e) {
    if (e == cudaSuccess) return AJ_OK;
    cudaGetLastError();
    return AJ_ERR_CUDA;
}

}  // namespace

extern "C" {

aj_status aj_kv_create(aj_kv *out, int device, int max_B, int max_q, int Hq, int Hkv, int D, int page_size, aj_dtype dtype,
                       unsigned flags) {
    if (!out) return AJ_ERR_INVALID_ARG;
    *out = nullptr;
    if (device < 0 || max_B < 1 || max_B > 4096 || max_q < 1 || max_q > (1 << 20) || Hq < 1 || Hkv < 1 || Hq % Hkv != 0 || D < 1)
        return AJ_ERR_INVALID_ARG;
    if (dtype != AJ_BF16 && dtype != AJ_F32) return AJ_ERR_INVALID_ARG;
    if (flags & ~(AJ_KV_FLAG_FORCE_SIMT | AJ_KV_FLAG_FORCE_SHARED)) return AJ_ERR_INVALID_ARG;
    if (D % 8 != 0 || D > 256 || Hq > 1024 || (long long)max_B * Hkv > 65535) return AJ_ERR_UNSUPPORTED;
    if (page_size != 16 && page_size != 32 && page_size != 64 && page_size != 128) return AJ_ERR_UNSUPPORTED;
    if ((long long)max_B * max_q * Hq > (1ll << 30)) return AJ_ERR_UNSUPPORTED;

    int count = 0;
    if (cudaGetDeviceCount(&count) != cudaSuccess || device >= count) {
        cudaGetLastError();
        return AJ_ERR_CUDA;
    }
    int major = 0, sms = 0;
    if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, device) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess) {
        cudaGetLastError();
        return AJ_ERR_CUDA;
    }
    if (major != 10) return AJ_ERR_NOT_SM100;
    Guard guard(device);
    if (!guard.ok()) return AJ_ERR_CUDA;
    aj_kv h = new (std::nothrow) aj_kv_s;
    if (!h) return AJ_ERR_CUDA;
    h->device = device;
    h->num_sms = sms;
    h->max_B = max_B;
    h->max_q = max_q;
    h->Hq = Hq;
    h->Hkv = Hkv;
    h->D = D;
    h->page = page_size;
    for (h->page_shift = 0; (1 << h->page_shift) < page_size;) h->page_shift++;
    h->dtype = dtype;
    h->flags = flags;
    if (kv::prepare_attend_few() != cudaSuccess || kv::prepare_attend_umma() != cudaSuccess || kv::prepare_weigh_mma() != cudaSuccess ||
        kv::prepare_weigh_umma() != cudaSuccess || kv::prepare_evict(h->clusters) != cudaSuccess) {
        cudaGetLastError();
        delete h;
        return AJ_ERR_CUDA;
    }
    // CUDA-core kernels: 6 waves of pieces, or two per item if that is more, up to 64 MB
    const int G = Hq / Hkv;
    const long long items = (long long)max_B * Hkv * (((long long)max_q * G + kv::SIMT_ROWS - 1) / kv::SIMT_ROWS);
    h->n_counters = (int)(items < 65536 ? items : 65536);
    if (h->n_counters < 2 * sms) h->n_counters = 2 * sms;  // tcgen05 kernel: two streams of the item that spans on from a CTA
    h->parts_floats = (size_t)(7 * sms) * kv::SIMT_ROWS * (D + 2);
    h->tensor = dtype == AJ_BF16 && (D == 64 || D == 128) && !(flags & AJ_KV_FLAG_FORCE_SIMT);
    if (h->tensor && kv::few_parts_floats(D, sms) > h->parts_floats) h->parts_floats = kv::few_parts_floats(D, sms);
    const bool many = h->tensor && (long long)max_q * G > kv::FEW_ROWS;  // calls for the tcgen05 kernels
    if (many && G <= 128 && kv::umma_parts_floats(D, sms) > h->parts_floats) h->parts_floats = kv::umma_parts_floats(D, sms);
    if (many && !prepare_maps(h)) {
        cudaGetLastError();
        delete h;
        return AJ_ERR_CUDA;
    }
    const size_t n = (size_t)h->n_counters + max_B;
    if (cudaMalloc(&h->parts, h->parts_floats * 4) != cudaSuccess || cudaMalloc(&h->counters, n * 4) != cudaSuccess ||
        cudaMalloc(&h->status, 256) != cudaSuccess || zero_now(h->counters, n * 4) != cudaSuccess ||
        zero_now(h->status, 256) != cudaSuccess) {
        cudaGetLastError();
        aj_kv_destroy(h);
        return AJ_ERR_CUDA;
    }
    if (many && !encode_pages(h, h->parts)) {
        aj_kv_destroy(h);
        return AJ_ERR_CUDA;
    }
    *out = h;
    return AJ_OK;
}

aj_status aj_kv_destroy(aj_kv h) {
    if (!h) return AJ_ERR_INVALID_ARG;
    Guard guard(h->device);
    cudaFree(h->parts);
    cudaFree(h->counters);
    cudaFree(h->status);
    free_shared(h);
    delete h;
    return AJ_OK;
}

aj_status aj_kv_append(aj_kv h, const void *q, long long q_stride, const void *k, long long k_stride, const void *v,
                       long long v_stride, const float *q_norm, const float *k_norm, float eps, const float *cos_sin,
                       int n_pos, int rot_dim, int interleaved, const int32_t *positions, void *k_pages, void *v_pages,
                       int n_pages, const int32_t *block_table, int table_width, const int32_t *seq_lens,
                       const int32_t *q_start, int B, int n_q, void *q_out, long long q_out_stride, int32_t *slot_pos,
                       float *weight, void *cuda_stream) {
    aj_status st = check_view(h, k_pages, n_pages, block_table, table_width, seq_lens, B, n_q);
    if (st != AJ_OK) return st;
    if (!v_pages || rot_dim < 0 || rot_dim > h->D || rot_dim % 2 != 0 || (rot_dim > 0 && (!cos_sin || n_pos < 1)) || !(eps >= 0.0f))
        return AJ_ERR_INVALID_ARG;
    if ((st = check_rows(h, q, q_stride, h->Hq)) != AJ_OK || (st = check_rows(h, k, k_stride, h->Hkv)) != AJ_OK ||
        (st = check_rows(h, v, v_stride, h->Hkv)) != AJ_OK || (st = check_rows(h, q_out, q_out_stride, h->Hq)) != AJ_OK)
        return st;
    if (off16(v_pages) || off16(cos_sin) || off16(q_norm) || off16(k_norm)) return AJ_ERR_UNSUPPORTED;
    Guard guard(h->device);
    if (!guard.ok()) return AJ_ERR_CUDA;
    kv::AppendArgs a;
    a.v = view_of(h, n_pages, block_table, table_width, seq_lens, q_start, B, n_q, 0, 0);
    a.q = q;
    a.k = k;
    a.vv = v;
    a.q_stride = q_stride;
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.q_out = q_out;
    a.q_out_stride = q_out_stride;
    a.q_norm = q_norm;
    a.k_norm = k_norm;
    a.eps = eps;
    a.cos_sin = cos_sin;
    a.n_pos = n_pos;
    a.rot = rot_dim;
    a.interleaved = interleaved != 0;
    a.positions = positions;
    a.k_pages = k_pages;
    a.v_pages = v_pages;
    a.slot_pos = slot_pos;
    a.weight = weight;
    h->last_launches = 1;
    return done(kv::launch_append(a, h->dtype == AJ_BF16, (cudaStream_t)cuda_stream));
}

aj_status aj_kv_attend(aj_kv h, const void *q, long long q_stride, const void *k_pages, const void *v_pages, int n_pages,
                       const int32_t *block_table, int table_width, const int32_t *seq_lens, const int32_t *q_start, int B,
                       int n_q, float scale, int window, int sinks, void *out, long long out_stride, float *lse,
                       void *cuda_stream) {
    aj_status st = check_view(h, k_pages, n_pages, block_table, table_width, seq_lens, B, n_q);
    if (st != AJ_OK) return st;
    if (!v_pages || !(scale > 0.0f) || !(scale < 1e30f) || window < 0 || sinks < 0) return AJ_ERR_INVALID_ARG;
    if ((st = check_rows(h, q, q_stride, h->Hq)) != AJ_OK || (st = check_rows(h, out, out_stride, h->Hq)) != AJ_OK) return st;
    if (off16(v_pages)) return AJ_ERR_UNSUPPORTED;
    Guard guard(h->device);
    if (!guard.ok()) return AJ_ERR_CUDA;
    kv::AttendArgs a = attend_args(h, q, q_stride, k_pages, v_pages, scale, out, out_stride, lse);
    static_cast<kv::CacheView &>(a.v) = view_of(h, n_pages, block_table, table_width, seq_lens, q_start, B, n_q, window, sinks);
    h->last_launches = 1;
    if (h->tensor && n_q * a.v.G <= kv::FEW_ROWS) {
        h->last_path = "few";
        return done(kv::launch_attend_few(a, h->num_sms, (cudaStream_t)cuda_stream));
    }
    if (h->tensor && a.v.G <= 128 && on128(k_pages) && on128(v_pages)) {  // (swizzled boxes want 128-byte rows; else the CUDA cores)
        h->last_path = "umma";
        CUtensorMap maps[4];
        int q_tma;
        if (!attend_maps(h, a, maps, &q_tma)) return AJ_ERR_CUDA;
        return done(kv::launch_attend_umma(a, maps, q_tma, h->num_sms, (cudaStream_t)cuda_stream));
    }
    h->last_path = "simt";
    return done(kv::launch_attend_simt(a, h->dtype == AJ_BF16, h->num_sms, (cudaStream_t)cuda_stream));
}

aj_status aj_kv_reserve_shared(aj_kv h, int max_rows) {
    if (!h || max_rows < 0 || (long long)max_rows * h->Hq > (1ll << 30)) return AJ_ERR_INVALID_ARG;
    Guard guard(h->device);
    if (!guard.ok()) return AJ_ERR_CUDA;
    if (!h->tensor || h->Hq / h->Hkv > 128 || max_rows == 0) {  // nothing to reserve: calls attend sequence by sequence
        free_shared(h);
        return AJ_OK;
    }
    if (max_rows <= h->pre_rows) return AJ_OK;
    // the shared slots always go to the tcgen05 kernel, which a handle for single tokens was not made for
    if (!h->encode) {
        if (!prepare_maps(h) || !encode_pages(h, h->parts)) {
            h->encode = nullptr;
            cudaGetLastError();
            return AJ_ERR_CUDA;
        }
    }
    const size_t heads = (size_t)pre_capacity(h, max_rows) * h->Hq, own = (size_t)max_rows * h->Hq;
    aj_kv_s n;  // the new workspace
    n.pre_rows = max_rows;
    if (cudaMalloc(&n.pre, (heads + own) * h->D * 4) != cudaSuccess || cudaMalloc(&n.pre_ml, heads * 8) != cudaSuccess ||
        cudaMalloc(&n.own_ml, own * 8) != cudaSuccess || cudaMalloc(&n.pre_parts, kv::umma_parts_floats(h->D, h->num_sms) * 4) != cudaSuccess ||
        cudaMalloc(&n.pre_counters, (size_t)h->num_sms * 8) != cudaSuccess || zero_now(n.pre_counters, (size_t)h->num_sms * 8) != cudaSuccess ||
        kv::mark_now(n.own_ml, own) != cudaSuccess) {
        cudaGetLastError();
        free_shared(&n);
        return AJ_ERR_CUDA;
    }
    free_shared(h);
    h->pre = n.pre;
    h->pre_ml = n.pre_ml;
    h->own_ml = n.own_ml;
    h->pre_parts = n.pre_parts;
    h->pre_counters = n.pre_counters;
    h->pre_rows = max_rows;
    return AJ_OK;
}

aj_status aj_kv_attend_shared(aj_kv h, const void *q, long long q_stride, const void *k_pages, const void *v_pages, int n_pages,
                              const int32_t *shared_table, int shared, const int32_t *block_table, int table_width, const int32_t *seq_lens,
                              const int32_t *q_start, int B, int n_q, float scale, void *out, long long out_stride, float *lse,
                              void *cuda_stream) {
    aj_status st = check_view(h, k_pages, n_pages, block_table, table_width, seq_lens, B, n_q);
    if (st != AJ_OK) return st;
    if (shared < 0 || shared > (long long)table_width * h->page || (shared > 0 && !shared_table)) return AJ_ERR_INVALID_ARG;
    const int whole = shared / 128 * 128;  // tiles that are shared to their end
    if (!h->tensor || h->Hq / h->Hkv > 128 || !on128(k_pages) || !on128(v_pages) || whole == 0 || B == 1)
        return aj_kv_attend(h, q, q_stride, k_pages, v_pages, n_pages, block_table, table_width, seq_lens, q_start, B, n_q, scale, 0, 0, out, out_stride,
                            lse, cuda_stream);
    if (!v_pages || !(scale > 0.0f) || !(scale < 1e30f)) return AJ_ERR_INVALID_ARG;
    if ((st = check_rows(h, q, q_stride, h->Hq)) != AJ_OK || (st = check_rows(h, out, out_stride, h->Hq)) != AJ_OK) return st;
    if (h->pre_rows == 0 || (!q_start && (long long)B * n_q > h->pre_rows)) return AJ_ERR_WORKSPACE;
    Guard guard(h->device);
    if (!guard.ok()) return AJ_ERR_CUDA;
    kv::AttendArgs a = attend_args(h, q, q_stride, k_pages, v_pages, scale, out, out_stride, lse);
    static_cast<kv::CacheView &>(a.v) = view_of(h, n_pages, block_table, table_width, seq_lens, q_start, B, n_q, 0, 0);
    a.v.shared = whole;
    a.v.behind = shared;
    a.v.lead_table = shared_table;
    a.v.n_seq = B;
    a.v.total = B * n_q;
    a.v.pre_rows = a.v.total < h->pre_rows ? a.v.total : h->pre_rows;
    const int ctas = cut_shared(a.v, h->num_sms);
    if (!(h->flags & AJ_KV_FLAG_FORCE_SHARED) && !worth_sharing(a.v))
        return aj_kv_attend(h, q, q_stride, k_pages, v_pages, n_pages, block_table, table_width, seq_lens, q_start, B, n_q, scale, 0, 0, out, out_stride,
                            lse, cuda_stream);
    a.pre = h->pre;
    a.pre_ml = h->pre_ml;
    a.own_ml = h->own_ml;
    CUtensorMap maps[4];
    int q_tma;
    if (!attend_maps(h, a, maps, &q_tma)) return AJ_ERR_CUDA;
    const cudaStream_t s = (cudaStream_t)cuda_stream;
    cudaError_t e;
    kv::AttendArgs p = a;
    p.v.lead = a.v.n_chunks;
    if (n_q * a.v.G <= kv::FEW_ROWS) {
        // the shared slots on the tcgen05 kernel, the sequences' own on the one for few rows, side by side: each with a workspace
        h->last_path = "shared_few";
        h->last_launches = 3;
        p.v.B = p.v.lead;
        p.v.align = p.v.chunk / 128 + 2;  // whole items
        p.v.n_q = p.v.pre_rows;
        p.parts = h->pre_parts;
        p.counters = h->pre_counters;
        e = kv::launch_attend_umma(p, maps, q_tma, ctas, s);
        if (e == cudaSuccess) e = kv::launch_attend_few(a, h->num_sms - ctas, s);
    } else {
        h->last_path = "shared_umma";
        h->last_launches = 2;
        p.v.B = p.v.lead + B;
        e = kv::launch_attend_umma(p, maps, q_tma, h->num_sms, s);
    }
    if (e == cudaSuccess) e = kv::launch_join(a, s);
    return done(e);
}

aj_status aj_kv_weigh(aj_kv h, const void *q, long long q_stride, const float *lse, const void *k_pages, int n_pages,
                      const int32_t *block_table, int table_width, const int32_t *seq_lens, const int32_t *q_start,
                      const int32_t *n_rows, int B, int n_q, float scale, int window, int sinks, const float *weight,
                      float *weight_out, void *cuda_stream) {
    aj_status st = check_view(h, k_pages, n_pages, block_table, table_width, seq_lens, B, n_q);
    if (st != AJ_OK) return st;
    if (!lse || !weight || !weight_out || !(scale > 0.0f) || !(scale < 1e30f) || window < 0 || sinks < 0) return AJ_ERR_INVALID_ARG;
    if ((st = check_rows(h, q, q_stride, h->Hq)) != AJ_OK) return st;
    Guard guard(h->device);
    if (!guard.ok()) return AJ_ERR_CUDA;
    kv::WeighArgs a;
    a.v = view_of(h, n_pages, block_table, table_width, seq_lens, q_start, B, n_q, window, sinks);
    a.q = q;
    a.q_stride = q_stride;
    a.k = k_pages;
    a.lse = lse;
    a.n_rows = n_rows;
    a.weight = weight;
    a.weight_out = weight_out;
    a.scale_log2 = scale * kv::LOG2E;
    a.status = h->status;
    h->last_launches = 1;
    if (h->tensor && n_q * a.v.G > kv::FEW_ROWS && on128(k_pages)) {
        h->last_path = "umma";
        CUtensorMap mk;
        if (!at_address(h, &mk, h->pages, k_pages)) return AJ_ERR_CUDA;
        return done(kv::launch_weigh_umma(a, mk, h->num_sms, (cudaStream_t)cuda_stream));
    }
    if (h->tensor) {
        h->last_path = "mma";
        return done(kv::launch_weigh_mma(a, h->num_sms, (cudaStream_t)cuda_stream));
    }
    h->last_path = "simt";
    return done(kv::launch_weigh_simt(a, h->dtype == AJ_BF16, (cudaStream_t)cuda_stream));
}

aj_status aj_kv_evict(aj_kv h, void *k_pages, void *v_pages, int n_pages, const int32_t *block_table, int table_width,
                      const int32_t *seq_lens, int B, int keep, int sinks, int recent, const float *weight,
                      const int32_t *slot_pos, int32_t *lens_out, float *weight_out, int32_t *slot_pos_out,
                      void *cuda_stream) {
    aj_status st = check_view(h, k_pages, n_pages, block_table, table_width, seq_lens, B, 1);
    if (st != AJ_OK) return st;
    if (!v_pages || !weight || !slot_pos || !lens_out || !weight_out || !slot_pos_out || keep < 1 || sinks < 0 || recent < 0 ||
        (long long)sinks + recent > keep)
        return AJ_ERR_INVALID_ARG;
    if (off16(v_pages)) return AJ_ERR_UNSUPPORTED;
    Guard guard(h->device);
    if (!guard.ok()) return AJ_ERR_CUDA;
    kv::EvictArgs a;
    a.v = view_of(h, n_pages, block_table, table_width, seq_lens, nullptr, B, 1, 0, 0);
    a.k_pages = k_pages;
    a.v_pages = v_pages;
    a.keep = keep;
    a.sinks = sinks;
    a.recent = recent;
    a.elem = h->dtype == AJ_BF16 ? 2 : 4;
    a.weight = weight;
    a.slot_pos = slot_pos;
    a.lens_out = lens_out;
    a.weight_out = weight_out;
    a.slot_pos_out = slot_pos_out;
    h->last_launches = 1;
    return done(kv::launch_evict(a, h->counters + h->n_counters, h->clusters, h->num_sms, (cudaStream_t)cuda_stream));
}

aj_status aj_kv_last_status(aj_kv h) {
    if (!h) return AJ_ERR_INVALID_ARG;
    Guard guard(h->device);
    int s = 0;
    if (!guard.ok() || cudaDeviceSynchronize() != cudaSuccess || cudaMemcpy(&s, h->status, 4, cudaMemcpyDeviceToHost) != cudaSuccess) {
        cudaGetLastError();
        return AJ_ERR_CUDA;
    }
    // a call that gave up may have left items without their last arrival: the counts of later calls begin at zero again
    if (s != 0 && (zero_now(h->counters, ((size_t)h->n_counters + h->max_B) * 4) != cudaSuccess || zero_now(h->status, 4) != cudaSuccess))
        return AJ_ERR_CUDA;
    if (s != 0 && h->pre && (zero_now(h->pre_counters, (size_t)h->num_sms * 8) != cudaSuccess || kv::mark_now(h->own_ml, (size_t)h->pre_rows * h->Hq) != cudaSuccess))
        return AJ_ERR_CUDA;
    return s == DEV_TIMEOUT ? AJ_ERR_TIMEOUT : AJ_OK;
}

int aj_kv_last_launch_count(aj_kv h) { return h ? h->last_launches : 0; }
const char *aj_kv_last_path(aj_kv h) { return h ? h->last_path : "none"; }

}  // extern "C"
