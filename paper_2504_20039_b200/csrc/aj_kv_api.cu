// Host side of the key-value cache operators: argument checks, the handle's workspace, choice of kernel, launches.
// No call synchronises or allocates but aj_kv_create, aj_kv_destroy and aj_kv_last_status.
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

kv::View view_of(aj_kv h, int n_pages, const int32_t *table, int width, const int32_t *lens, const int32_t *q_start, int B,
                 int n_q, int window, int sinks) {
    kv::View v;
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
    if (flags & ~AJ_KV_FLAG_FORCE_SIMT) return AJ_ERR_INVALID_ARG;
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
    if (many) {
        void *fn = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess || !fn) {
            cudaGetLastError();
            delete h;
            return AJ_ERR_CUDA;
        }
        h->encode = reinterpret_cast<EncodeTiledFn>(fn);
        if (cudaGetDriverEntryPointByVersion("cuTensorMapReplaceAddress", &fn, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess || !fn) {
            cudaGetLastError();
            delete h;
            return AJ_ERR_CUDA;
        }
        h->replace = reinterpret_cast<ReplaceAddressFn>(fn);
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
    kv::AttendArgs a;
    a.v = view_of(h, n_pages, block_table, table_width, seq_lens, q_start, B, n_q, window, sinks);
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
    h->last_launches = 1;
    if (h->tensor && n_q * a.v.G <= kv::FEW_ROWS) {
        h->last_path = "few";
        return done(kv::launch_attend_few(a, h->num_sms, (cudaStream_t)cuda_stream));
    }
    if (h->tensor && a.v.G <= 128 && on128(k_pages) && on128(v_pages)) {  // (swizzled boxes want 128-byte rows; else the CUDA cores)
        h->last_path = "umma";
        CUtensorMap maps[4];
        if (!at_address(h, &maps[0], h->pages, k_pages) || !at_address(h, &maps[1], h->pages, v_pages)) return AJ_ERR_CUDA;
        // queries by TMA (boxes of eight tokens where a tile has as many, and of one), or by one warp's 16-byte copies where their
        // rows do not lie on 128 bytes: 64 windows of 33 rows 157 us and 209, a prompt of 8192 490 and 647
        const int q_tma = !on128(q, q_stride * 2) ? 0 : 128 / a.v.G >= 8 ? 8 : 1;
        if (q_tma && q_stride != h->q_stride) {
            h->q_stride = -1;
            if (!encode_rows(h, &h->rows1, h->parts, q_stride, 1) || (q_tma == 8 && !encode_rows(h, &h->rows8, h->parts, q_stride, 8))) return AJ_ERR_CUDA;
            h->q_stride = q_stride;
        }
        if (q_tma && (!at_address(h, &maps[2], h->rows1, q) || (q_tma == 8 && !at_address(h, &maps[3], h->rows8, q)))) return AJ_ERR_CUDA;
        h->last_launches = 1;
        return done(kv::launch_attend_umma(a, maps, q_tma, h->num_sms, (cudaStream_t)cuda_stream));
    }
    h->last_path = "simt";
    return done(kv::launch_attend_simt(a, h->dtype == AJ_BF16, h->num_sms, (cudaStream_t)cuda_stream));
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
    return s == DEV_TIMEOUT ? AJ_ERR_TIMEOUT : AJ_OK;
}

int aj_kv_last_launch_count(aj_kv h) { return h ? h->last_launches : 0; }
const char *aj_kv_last_path(aj_kv h) { return h ? h->last_path : "none"; }

}  // extern "C"
