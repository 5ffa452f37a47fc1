// aj_kv_attend for many query rows per key head (verification windows and prompts), bf16, on tcgen05.
//
//   S = Q K^T   128 rows (token, query head) x 128 slots, f32 in tensor memory
//   P = exp2(scale * S - m)   one thread per row, bf16, written back over S in tensor memory
//   O += P V    P from tensor memory, V from shared memory as it lies in the pages (head elements contiguous)
//
// A CTA per SM holds two such row tiles ("streams").  A piece of work of more than 128 rows gives each stream half of
// the tokens, and both read the same K and V tiles; a piece of at most 128 rows (a verification window) gives
// both streams the same rows and every other tile of 128 slots, so that in either case one stream's softmax runs
// under the other's matrix products.  Tensor memory: S0 S1 (128 columns each), O0 O1 (D columns each).
//
//   warps 0-3, 4-7  softmax of stream 0 and 1 (thread = row = TMEM lane); they store the results
//   warps 8, 10     issue tcgen05.mma for stream 0 and 1: PV of half a tile, then QK^T of that half of the stream's next tile
//   warp 9          TMA: 64-column x page-row boxes (128-byte swizzle) of the pages into a ring of K and V tiles, in the
//                   order K0 K1 V0 K2 V1 ... in which they are consumed
//   warp 11         the queries of both streams, by TMA where they lie on 128 bytes, else by 16-byte copies
//
// Scores go to the softmax in halves of 64 slots with barriers of their own: while one half is in the softmax, the other
// half's products run.
//
// The tiles of all (sequence, key head, row piece) items of the batch form one line, cut into equal pieces, one per
// CTA: causal prompts and ragged caches are balanced alike.  Items that span CTAs leave unnormalised partial results
// (f32) in the workspace, and the CTA that arrives last joins them, in the order of the CTAs (a second kernel for that cost 11
// to 16 us a call, most of it in finding its place on the line).
//
// What bounds it, and what it measured (8 key heads, 32 query heads):
//   windows of 33 rows, 64 sequences of 129 .. 4100 slots, D = 128: 162 us, 3.8 TB/s; 6 us go by before the first scores, 3 us
//   between two items, 5 us in the last join.  132 rows, four more than a tile holds, make two tiles of 68 and 64: their
//   products keep the tensor pipe 47 % busy in what should be a stream of pages
//   a prompt of 8192, D = 128: 510 us alone, 1.08 PFLOP/s; back to back the card's power limit lowers the clock (570 us)
//   four prompts with a window of 1024, D = 64: half the products for as many exponentials, and ten tiles an item, two of
//   them partly masked; 174 us
//   In both, a pair of tiles (256 x 128 scores) takes some 3500 cycles, where its exponentials take 1536 of their unit (16 per
//   clock and SM, a quarter of them on the multiply-add pipe) and its four products 2048 (D = 128) or 1024 of the
//   tensor pipe: with two softmax warps per scheduler it is their latencies that are left over (an instruction in 35 to 47 % of the
//   issue slots; waits for tensor memory first, then for results of fixed latency, then for instructions)
//
// The running maximum is a reference that is raised only when a score exceeds it by more than RAISE, so the rescaling of
// O (a round trip through tensor memory) is rare; weights far above 1 are as exact as weights up to 1 (raised from 8 on: 192 us
// for the prompts with a window, from 30 on: 183 us, at that stage).
// Every wait is bounded (aj_ptx.cuh); one that runs out sets the status word and the CTA leaves by the normal way out.
#include "aj_kv.cuh"
#include "aj_kv_line.cuh"
#include "aj_kv_tc.cuh"
#include "aj_ptx.cuh"

namespace aj {
namespace kv {

namespace {

constexpr int THREADS = 384;
// Registers: launched with 168 a thread; the two softmax warpgroups, which hold a row of 128 scores, take 200 and leave
// 104 to the third (2 x 200 + 104 = 3 x 168).  Each branch sets its own share: before that no code is shared.
constexpr int REGS_SOFTMAX = 200, REGS_OTHER = 104;
constexpr uint32_t B_MN_MAJOR = 1u << 16;

template <int D> struct Cfg {
    static constexpr int TILE_BYTES = TILE * D * 2;            // a K or V tile, and a query tile
    static constexpr int STAGES = D == 128 ? 5 : 8;
    static constexpr int BARS = 2 * STAGES + 24;
    static constexpr int ML_AT = (2 + STAGES) * TILE_BYTES + BARS * 8 + 16;  // maxima and sums of both streams' rows
    static constexpr int SMEM = ML_AT + 4 * 128 * 4;
    static_assert(SMEM <= 232448 && STAGES * TILE_BYTES >= (4096 + 1) * 8, "the prefix sums of the largest batch fit the ring");
    static constexpr int PART = 256 * (D + 2);                 // floats of one partial result
};

// Prefix sums over the sequences of their tiles, by all threads; returns the total.
__device__ inline long long build_line(const View &v, int tpt, long long *pre) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (v.n_q <= 16 * tpt) {  // few pieces: a thread per sequence; else a warp
        for (int b = threadIdx.x; b < v.B; b += blockDim.x) pre[b + 1] = units_of(v, pieces_of(seq_of(v, b), tpt), tpt, 0, 1) * v.Hkv;
    } else {
        for (int b = warp; b < v.B; b += blockDim.x >> 5) {
            long long u = units_of(v, pieces_of(seq_of(v, b), tpt), tpt, lane, 32);
#pragma unroll
            for (int o = 16; o; o >>= 1) u += __shfl_xor_sync(~0u, u, o);
            if (lane == 0) pre[b + 1] = u * v.Hkv;
        }
    }
    if (threadIdx.x == 0) pre[0] = 0;
    __syncthreads();
    if (warp == 0) {
        long long carry = 0;
        for (int b0 = 1; b0 <= v.B; b0 += 32) {
            long long x = b0 + lane <= v.B ? pre[b0 + lane] : 0;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long y = __shfl_up_sync(~0u, x, o);
                if (lane >= o) x += y;
            }
            if (b0 + lane <= v.B) pre[b0 + lane] = carry + x;
            carry += __shfl_sync(~0u, x, 31);
        }
    }
    __syncthreads();
    return pre[v.B];
}

// By a whole warp.
__device__ inline Line seek(const View &v, int tpt, const long long *pre, long long u) {
    Line c;
    const int lane = threadIdx.x & 31;
    int lo = 0, hi = v.B;  // pre[lo] <= u < pre[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (pre[mid] <= u) lo = mid; else hi = mid;
    }
    c.b = lo;
    c.q = pieces_of(seq_of(v, lo), tpt);
    const long long per_head = (pre[lo + 1] - pre[lo]) / v.Hkv;
    long long r = u - pre[lo];
    c.h = (int)(r / per_head);
    r -= c.h * per_head;
    for (int q0 = 0;; q0 += 32) {
        const int n = q0 + lane < c.q.n ? CHARGE + piece_of(v, c.q, q0 + lane, tpt).units : 0;
        int x = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(~0u, x, o);
            if (lane >= o) x += y;
        }
        const int all = __shfl_sync(~0u, x, 31);
        if (r < all) {
            const int at = __ffs(__ballot_sync(~0u, r < x)) - 1;
            c.qt = q0 + at;
            c.unit = (int)r - __shfl_sync(~0u, x - n, at) - CHARGE;
            break;
        }
        r -= all;
    }
    c.p = piece_of(v, c.q, c.qt, tpt);
    return c;
}

// To the first tile of the next item.
__device__ inline void next_item(const View &v, int tpt, Line &c) {
    c.unit = -CHARGE;
    if (++c.qt == c.q.n) {
        c.qt = 0;
        if (++c.h == v.Hkv) {
            c.h = 0;
            do {
                if (++c.b >= v.B) return;
                c.q = pieces_of(seq_of(v, c.b), tpt);
            } while (c.q.n == 0);
        }
    }
    c.p = piece_of(v, c.q, c.qt, tpt);
}

// Order of the K and V tiles of a segment of n tiles in the ring: K0 K1 V0 K2 V1 ... V(n-1).
__device__ inline int pos_k(int t) { return t == 0 ? 0 : 2 * t - 1; }
__device__ inline int pos_v(int t, int n) { return t + 1 < n ? 2 * t + 2 : 2 * n - 1; }

__device__ inline void umma_ts(uint32_t d, uint32_t a, unsigned long long bdesc, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d), "r"(a), "l"(bdesc), "r"(idesc), "r"(acc)
        : "memory");
}
// V as it lies in the pages: element blocks of 64 (128 bytes per slot), 128 slots each, 16 KB apart.
__device__ inline unsigned long long desc_v(uint32_t addr) {
    return (unsigned long long)((addr & 0x3FFFF) >> 4) | (unsigned long long)(16384 >> 4) << 16 |
           (unsigned long long)(1024 >> 4) << 32 | (unsigned long long)1 << 46 | (unsigned long long)2 << 61;
}

#define I8(r, i) "r"(r[i]), "r"(r[i + 1]), "r"(r[i + 2]), "r"(r[i + 3]), "r"(r[i + 4]), "r"(r[i + 5]), "r"(r[i + 6]), "r"(r[i + 7])

// x *= c for 16 columns of this thread's lane
__device__ inline void tmem_scale16(uint32_t addr, float c) {
    uint32_t r[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : R8(r, 0), R8(r, 8)
        : "r"(addr)
        : "memory");
#pragma unroll
    for (int i = 0; i < 16; i++) r[i] = __float_as_uint(__uint_as_float(r[i]) * c);
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
        ::I8(r, 0), I8(r, 8), "r"(addr)
        : "memory");
}
__device__ inline void tmem_st32(uint32_t addr, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};"
        ::I8(r, 0), I8(r, 8), I8(r, 16), I8(r, 24), "r"(addr)
        : "memory");
}
__device__ inline void tma_load_3d(uint32_t dst, const CUtensorMap *tmap, int c0, int c1, int c2, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
        ::"r"(dst), "l"(tmap), "r"(bar), "r"(c0), "r"(c1), "r"(c2)
        : "memory");
}
__device__ inline void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// 2^x for a pair on the multiply-add pipe, for x <= RAISE (which is far inside its range): x = n + f with n the nearest
// integer, 2^f by the polynomial that interpolates it at the five Chebyshev nodes of [-1/2, 1/2] (relative error below 4e-6, of
// either sign: a thousandth of what rounding a weight to bf16 takes, and as much in lse at most), 2^n by adding to the exponent.
// Arguments of -127 and below (masked slots) give zero, those up to -126 less than 2^-126, NaN gives zero too.
constexpr float P0 = 1.0f, P1 = 0.6931210527f, P2 = 0.2402234922f, P3 = 0.05592198042f, P4 = 0.009666368369f;
__device__ inline uint64_t ex2_poly(uint64_t x) {
    const uint64_t y = f2(fmaxf(lo(x), -127.0f), fmaxf(hi(x), -127.0f));
    const float big = 12582912.0f;  // 1.5 * 2^23: the sum's last bits are the nearest integer
    const uint64_t t = add2(y, f2(big, big)), f = fma2(add2(t, f2(-big, -big)), f2(-1.0f, -1.0f), y);
    uint64_t p = fma2(f2(P4, P4), f, f2(P3, P3));
    p = fma2(p, f, f2(P2, P2));
    p = fma2(p, f, f2(P1, P1));
    p = fma2(p, f, f2(P0, P0));
    return f2(__int_as_float(__float_as_int(lo(p)) + (__float_as_int(lo(t)) << 23)), __int_as_float(__float_as_int(hi(p)) + (__float_as_int(hi(t)) << 23)));
}

__device__ inline uint32_t pack2(float lo, float hi) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&p);
}

template <int D>
__global__ void __launch_bounds__(THREADS, 1)
attend_umma_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v, const __grid_constant__ CUtensorMap tmap_q1,
                   const __grid_constant__ CUtensorMap tmap_q8, AttendArgs a, int tpt, int g_shift, int q_tma) {
    using C = Cfg<D>;
    constexpr int NS = C::STAGES, HALVES = D / 64;
    extern __shared__ __align__(1024) uint8_t smem[];  // swizzled tiles need 1024-byte alignment
    const uint32_t base = smem_u32(smem);
    const uint32_t q_at = base, ring = base + 2 * C::TILE_BYTES, bars = ring + NS * C::TILE_BYTES;
    auto full = [&](int s) { return bars + 8u * s; };
    auto empty = [&](int s) { return bars + 8u * (NS + s); };
    auto s_full = [&](int x, int hf) { return bars + 8u * (2 * NS + 2 * x + hf); };
    auto p_ready = [&](int x, int hf) { return bars + 8u * (2 * NS + 4 + 2 * x + hf); };
    auto pv_done = [&](int x, uint32_t half) { return bars + 8u * (2 * NS + 8 + 4 * x + (half & 3u)); };
    auto q_ready = [&](int x) { return bars + 8u * (2 * NS + 16 + x); };
    auto drained = [&](int x) { return bars + 8u * (2 * NS + 18 + x); };
    auto o_done = [&](int x) { return bars + 8u * (2 * NS + 20 + x); };
    auto q_free = [&](int x) { return bars + 8u * (2 * NS + 22 + x); };
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(smem + (2 + NS) * C::TILE_BYTES + C::BARS * 8);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
    long long *pre = reinterpret_cast<long long *>(smem + 2 * C::TILE_BYTES);  // the line's prefix sums lie in the ring until the first copy
    const View &v = a.v;
    const int warp = __shfl_sync(~0u, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;  // warp: uniform

    if (threadIdx.x == 0) {
        for (int s = 0; s < NS; s++) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), 2);  // both streams
        }
        for (int x = 0; x < 2; x++) {
            for (int hf = 0; hf < 2; hf++) {
                mbar_init(s_full(x, hf), 1);
                mbar_init(p_ready(x, hf), 128);
            }
            for (uint32_t i = 0; i < 4; i++) mbar_init(pv_done(x, i), 1);
            mbar_init(q_ready(x), 1);
            mbar_init(q_free(x), 1);
            mbar_init(drained(x), 1);
            mbar_init(o_done(x), 1);
        }
        *abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == 8) tmem_alloc(smem_u32(const_cast<uint32_t *>(tmem_slot)), 512);
    const long long total = build_line(v, tpt, pre);  // synchronises the CTA
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    // a piece of less than four tiles costs more in the join than its tiles (one window of 17 rows: 35 -> 28 us)
    // (a CTA's places fit an int, the line's need not; see the bounds at units_of)
    const int per = (int)max(4ll, (total + gridDim.x - 1) / gridDim.x);
    const long long u0 = min(total, (long long)blockIdx.x * per);
    const int u1 = (int)(min(total, u0 + per) - u0);  // from here on places are counted from u0
    auto give_up = [&]() {
        *abort_flag = 1;
        atomicCAS(a.status, DEV_OK, DEV_TIMEOUT);
    };

    if (u1 > 0) {
        if (warp >= 8) {
          asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_OTHER));
          Line c = seek(v, tpt, pre, u0);
          fence_async_shared();
          __syncthreads();  // the prefix sums are read: the ring may be filled
          if (warp == 9) {
            // ---------------------------------------------------------------- TMA
            const unsigned long long pol = policy_evict_normal();
            const int per_tile = TILE >> v.page_shift;  // pages of a tile: at most 8
            const uint32_t box_bytes = (uint32_t)v.page * 128u;
            uint32_t g = 0;
            bool ok = true;
            for (int u = 0; ok && u < u1; next_item(v, tpt, c)) {
                const Part pt = part_of(c, u1 - u);
                const int n = pt.n;
                u += pt.line;
                for (int i = 0; ok && i < 2 * n; i++) {
                    // position i holds K of tile t, or V of tile t
                    const bool is_v = i == 2 * n - 1 || (i >= 2 && (i & 1) == 0);
                    const int t = is_v ? (i == 2 * n - 1 ? n - 1 : (i - 2) >> 1) : (i == 0 ? 0 : (i + 1) >> 1);
                    const int s = g % NS;
                    // lane i looks up the tile's i-th page; one elected lane issues all copies.  Pages past the
                    // length and pages that no row of the item sees are not fetched.
                    const int slot0 = tile_of(c.p, pt.first + t) * TILE, slot = slot0 + (lane << v.page_shift);
                    const bool on = lane < per_tile && slot < c.q.s.L && (slot + v.page > c.p.first || slot < v.sinks);
                    const int row = on ? (page_of(v, c.b, slot) * v.Hkv + c.h) << v.page_shift : 0;
                    const unsigned which = __ballot_sync(~0u, on);
                    ok = __all_sync(~0u, mbar_wait(empty(s), ((g / NS) & 1u) ^ 1u, abort_flag));
                    if (!ok) {
                        give_up();
                        break;
                    }
                    const bool leader = elect_one();
                    if (leader) mbar_expect_tx(full(s), __popc(which) * (uint32_t)HALVES * box_bytes);
                    for (int p = 0; p < per_tile; p++) {
                        const int r = __shfl_sync(~0u, row, p);
                        if (which >> p & 1) {
                            const uint32_t dst = ring + s * C::TILE_BYTES + (uint32_t)(p << v.page_shift) * 128u;
                            if (leader) {
                                if (is_v) {
#pragma unroll
                                    for (int hf = 0; hf < HALVES; hf++) tma_load_2d(dst + hf * 16384, &tmap_v, hf * 64, r, full(s), pol);
                                } else {
#pragma unroll
                                    for (int hf = 0; hf < HALVES; hf++) tma_load_2d(dst + hf * 16384, &tmap_k, hf * 64, r, full(s), pol);
                                }
                            }
                        }
                    }
                    __syncwarp();
                    g++;
                }
            }
            // Before the CTA may leave, every copy has landed (after a time-out too) and every stage has been released:
            // a commit that is still on its way must not arrive in shared memory that belongs to the next CTA.
            int never = 0;
            for (uint32_t i = g > NS ? g - NS : 0; i < g; i++) {
                mbar_wait(full(i % NS), (i / NS) & 1u, &never);
                if (ok && !__all_sync(~0u, mbar_wait(empty(i % NS), (i / NS) & 1u, abort_flag))) {
                    give_up();
                    ok = false;
                }
            }
          } else if (warp == 11) {
            // ---------------------------------------------------------------- queries
            // A stream's queries of an item into the swizzled K-major layout (row = token x query heads + head), by TMA in
            // boxes of eight tokens and of one, or with 16-byte copies if their rows do not lie on 128 bytes (that takes one warp some
            // 10,000 cycles per item where TMA takes 1,500).  Rows past its tokens keep what they held: no other row
            // depends on them.  The next item's come in while the softmax and the last product of this one run.
            uint32_t n_q[2] = {0, 0};  // items whose queries have been asked for
            for (int u = 0; u < u1; next_item(v, tpt, c)) {
                const Part pt = part_of(c, u1 - u);
                u += pt.line;
                for (int x = 0; x < 2 && pt.n > 0; x++) {
                    if (!has_tile(c.p, x, pt.n)) continue;
                    if (!__all_sync(~0u, mbar_wait(q_free(x), (n_q[x] & 1u) ^ 1u, abort_flag))) {
                        give_up();
                        u = u1;
                        break;
                    }
                    n_q[x]++;
                    if (q_tma) {
                        const bool lead = x == 0 || c.p.tok0 == c.p.n_tok;
                        const int tok = lead ? c.p.tok0 : c.p.n_tok - c.p.tok0, r0 = c.q.s.row0 + c.p.ta + (lead ? 0 : c.p.tok0);
                        if (elect_one()) {
                            mbar_expect_tx(q_ready(x), (uint32_t)(tok * v.G) * 128u * HALVES);
                            for (int t = 0; t < tok;) {
                                const bool eight = q_tma == 8 && t + 8 <= tok;
#pragma unroll
                                for (int hf = 0; hf < HALVES; hf++)
                                    tma_load_3d(q_at + x * C::TILE_BYTES + hf * 16384 + (uint32_t)(t * v.G) * 128u, eight ? &tmap_q8 : &tmap_q1, hf * 64, c.h * v.G, r0 + t, q_ready(x));
                                t += eight ? 8 : 1;
                            }
                        }
                        __syncwarp();
                        continue;
                    }
                    constexpr int CPR = D / 8;
                    const bool lead = x == 0 || c.p.tok0 == c.p.n_tok;
                    const int n_rows = (lead ? c.p.tok0 : c.p.n_tok - c.p.tok0) * v.G;
                    const __nv_bfloat16 *qp = (const __nv_bfloat16 *)a.q + ((size_t)c.q.s.row0 + c.p.ta + (lead ? 0 : c.p.tok0)) * a.q_stride + (size_t)c.h * v.G * D;
#pragma unroll 4
                    for (int i = lane; i < 128 * CPR; i += 32) {
                        const int r = i / CPR, cc = i % CPR, t = g_shift >= 0 ? r >> g_shift : r / v.G;
                        const uint32_t dst = q_at + x * C::TILE_BYTES + (cc >> 3) * 16384 + r * 128 + (((cc & 7) ^ (r & 7)) << 4);
                        const int bytes = r < n_rows ? 16 : 0;
                        const void *src = r < n_rows ? (const void *)(qp + (size_t)t * a.q_stride + (size_t)(r - t * v.G) * D + cc * 8) : a.q;
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
                    }
                    asm volatile("cp.async.wait_all;" ::: "memory");
                    fence_async_shared();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(q_ready(x));
                }
            }
            int never = 0;  // every copy has landed before the CTA may leave, after a time-out too
            for (int x = 0; x < 2; x++)
                if (n_q[x] > 0) mbar_wait(q_ready(x), (n_q[x] - 1) & 1u, &never);
          } else if (warp <= 10) {
            // ---------------------------------------------------------------- MMA: warp 8 stream 0, warp 10 stream 1
            // The whole warp walks the loop and waits, one elected lane issues.
            const int x = warp == 8 ? 0 : 1;
            constexpr uint32_t idesc_s = instr_desc(128, 64), idesc_o = instr_desc(128, D) | B_MN_MAJOR;
            const uint32_t t_s = tmem + x * 128, t_o = tmem + 256 + x * D;
            const unsigned long long qd = smem_desc_sw128(q_at + x * C::TILE_BYTES);
            uint32_t g = 0, n_p = 0, n_q = 0;
            bool ok = true;
            auto wait = [&](uint32_t bar, uint32_t parity) {
                if (ok && !__all_sync(~0u, mbar_wait(bar, parity & 1u, abort_flag))) {
                    give_up();
                    ok = false;
                }
                tc_fence_after();
                return ok;
            };
            // Both warps walk over every tile and both release it: a warp that skipped the other stream's tiles could wait
            // for a stage's next phase while the previous one is still loading, and a parity wait would let it through.
            for (int u = 0; ok && u < u1; next_item(v, tpt, c)) {
                const Part pt = part_of(c, u1 - u);
                const int n = pt.n;
                u += pt.line;
                const bool shared_rows = c.p.tok0 == c.p.n_tok;
                const int ahead = shared_rows ? 2 : 1;  // K tiles in front of V tiles
                auto mine = [&](int t) { return !shared_rows || (t & 1) == x; };
                bool begun = false;
                auto issue_qk = [&](int t, int hf) {  // QK^T of one half of tile t, into the columns of that half
                    const unsigned long long kd = smem_desc_sw128(ring + ((g + pos_k(t)) % NS) * C::TILE_BYTES + hf * 8192);
#pragma unroll
                    for (int k = 0; k < D / 16; k++)
                        umma_bf16(t_s + hf * 64, qd + (k / 4) * (16384 >> 4) + 2 * (k % 4), kd + (k / 4) * (16384 >> 4) + 2 * (k % 4), idesc_s, k != 0);
                    umma_commit(s_full(x, hf));
                    if (hf == 1) {
                        umma_commit(empty((g + pos_k(t)) % NS));
                        if (t + ahead >= n) umma_commit(q_free(x));  // the stream's last product with these queries
                    }
                };
                auto qk = [&](int t, int hf) {
                    if (!begun) {
                        if (!wait(q_ready(x), n_q)) return;
                        n_q++;
                    }
                    begun = true;
                    if (elect_one()) issue_qk(t, hf);
                    __syncwarp();
                };
                // P V of one half of tile t, and right behind it the scores of the stream's next tile into the same columns.
                // The softmax waits for a product by a one-bit phase when it raises its reference, so it must know that the phase
                // before has passed.  Four barriers take turns over the halves, and this warp sees the product of two halves ago done
                // (long since: its scores have been through the softmax) before it issues the next half: when the scores of half m
                // are there, product m - 5, the one before m - 1 on its barrier, has been seen.
                auto pv_qk = [&](int t, int hf, bool more) {
                    const uint32_t s = (g + pos_v(t, n)) % NS;
                    const uint32_t half = 2 * n_p + hf;
                    const unsigned long long vd = desc_v(ring + s * C::TILE_BYTES + hf * 8192);
                    if (!wait(p_ready(x, hf), n_p)) return;
                    if (elect_one()) {
#pragma unroll
                        for (int k = 0; k < 4; k++)
                            umma_ts(t_o, t_s + hf * 64 + k * 8, vd + (unsigned long long)k * (2048 >> 4), idesc_o, hf == 0 && k == 0 ? t >= ahead : 1);
                        umma_commit(pv_done(x, half));  // the product alone, not the scores behind it
                        if (more) issue_qk(t + ahead, hf);
                        if (hf == 1) umma_commit(empty(s));
                        if (hf == 1 && t + ahead >= n) umma_commit(o_done(x));
                    }
                    __syncwarp();
                    if (half >= 2) wait(pv_done(x, half - 2), (half - 2) >> 2);
                };
                auto arrived = [&](uint32_t at) { return wait(full(at % NS), at / NS); };
                auto release = [&](uint32_t at) {
                    if (elect_one()) mbar_arrive(empty(at % NS));
                    __syncwarp();
                };
                for (int t = 0; ok && t < ahead && t < n; t++) {
                    if (!arrived(g + pos_k(t))) break;
                    if (mine(t)) {
                        qk(t, 0);
                        qk(t, 1);
                    } else {
                        release(g + pos_k(t));
                    }
                }
                for (int t = 0; ok && t < n; t++) {
                    const bool more = t + ahead < n;
                    if (!arrived(g + pos_v(t, n))) break;
                    if (mine(t)) {
                        if (more && !arrived(g + pos_k(t + ahead))) break;
                        pv_qk(t, 0, more);
                        if (ok) pv_qk(t, 1, more);
                        n_p++;
                    } else {
                        release(g + pos_v(t, n));
                        if (more) {
                            if (!arrived(g + pos_k(t + ahead))) break;
                            release(g + pos_k(t + ahead));
                        }
                    }
                }
                g += 2 * n;
            }
            // nothing that this warp issued is in flight when the CTA leaves, after a time-out either
            int never = 0;
            if (elect_one()) umma_commit(drained(x));
            __syncwarp();
            mbar_wait(drained(x), 0, &never);
            for (uint32_t i = 1; ok && i <= 2 && n_p > 0; i++) mbar_wait(pv_done(x, 2 * n_p - i), ((2 * n_p - i) >> 2) & 1u, &never);
          }
        } else {
            // ---------------------------------------------------------------- softmax of stream x
            asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS_SOFTMAX));
            Line c = seek(v, tpt, pre, u0);
            // rows of a query tile without a token stay zero (or what an item before had there): the tensor cores draw less
            // power on zeros, and power is what limits the clock
            for (int i = threadIdx.x; i < 2 * C::TILE_BYTES / 16; i += 256) reinterpret_cast<uint4 *>(smem)[i] = make_uint4(0, 0, 0, 0);
            fence_async_shared();
            __syncthreads();  // the prefix sums are read
            const int x = warp >> 2, row = threadIdx.x & 127, wq = warp & 3;
            const uint32_t lanes = (uint32_t)(wq * 32) << 16;
            const uint32_t t_s = tmem + x * 128 + lanes, t_o = tmem + 256 + x * D + lanes;
            uint32_t n_h = 0, n_o = 0, g = 0;  // halves of tiles and segments with a tile so far; places in the ring
            bool dead = false;
            auto wait = [&](uint32_t bar, uint32_t parity) {
                if (!dead && !mbar_wait(bar, parity & 1u, abort_flag)) {
                    give_up();
                    dead = true;  // go through the motions, so that the barriers below stay matched
                }
                __syncwarp();
                tc_fence_after();
            };
            const float scale = a.scale_log2;
            const bool wide_out = ((reinterpret_cast<uintptr_t>(a.out) | (uintptr_t)(a.out_stride * 2)) & 31) == 0;  // rows on 32 bytes
            auto token = [&](int r) { return g_shift >= 0 ? r >> g_shift : r / v.G; };
            for (int u = 0; u < u1; next_item(v, tpt, c)) {
                const Part pt = part_of(c, u1 - u);
                const int n = pt.n, unit = c.unit;
                u += pt.line;
                if (n == 0) continue;
                const bool shared_rows = c.p.tok0 == c.p.n_tok;
                const int tok = shared_rows || x == 0 ? c.p.tok0 : c.p.n_tok - c.p.tok0;
                const int ta = c.p.ta + (shared_rows || x == 0 ? 0 : c.p.tok0);
                const int n_rows = tok * v.G;
                const int p_first = c.q.s.L - c.q.s.nq + ta;           // slot of the stream's first token
                const int my_p = p_first + token(min(row, n_rows - 1)), p_last = p_first + tok - 1;
                float m = -INFINITY, l = 0.0f;
                const int step = shared_rows ? 2 : 1;
                bool first = true;
                // slots that nobody sees may hold anything: the values of a half's are cleared before its product, after its
                // softmax, because the values arrive one tile behind the keys (before it: 4 us more per item)
                auto clear_hidden = [&](int t, int j0, int hf) {
                    const int jh = j0 + hf * 64;
                    if (c.q.s.L - jh >= 64 && (jh >= c.p.first || jh + 64 <= v.sinks || c.p.first <= v.sinks)) return;
                    const uint32_t at = g + pos_v(t, n), s = at % NS;
                    wait(full(s), at / NS);
                    const int r = hf * 64 + (row & 63), j = j0 + r;
                    if (j >= c.q.s.L || (j < c.p.first && j >= v.sinks)) {
                        // half a row per thread; neighbouring rows begin at different 16 bytes, so they meet on no bank
#pragma unroll 1
                        for (int i = 0; i < 4 * HALVES; i++)
                            *reinterpret_cast<uint4 *>(smem + (2 + s) * C::TILE_BYTES + (HALVES == 2 ? (row >> 6) * 16384 : 0) + r * 128 +
                                                       (HALVES == 2 ? (i + r) & 7 : ((row >> 6) * 4 + ((i + r) & 3))) * 16) = make_uint4(0, 0, 0, 0);
                    }
                    fence_async_shared();
                    __syncwarp();
                };
                for (int t = shared_rows ? x : 0; t < n; t += step) {
                    const int j0 = tile_of(c.p, pt.first + t) * TILE;
                    const bool masked = j0 + TILE > p_first + 1 || (v.window && j0 <= p_last - v.window);
#pragma unroll 1
                    for (int hf = 0; hf < 2; hf++, n_h++) {
                        wait(s_full(x, hf), n_h >> 1);
                        if (wq * 32 >= n_rows) {  // a warp without a row: zero queries have left zeros where its weights go
                            first = false;
                            clear_hidden(t, j0, hf);
                            mbar_arrive(p_ready(x, hf));
                            continue;
                        }
                        uint32_t sr[64];
                        tmem_ld64(t_s + hf * 64, sr);
                        if (masked) {
                            // one bit per slot; no branch per element
                            const int jh = j0 + hf * 64, hi = my_p - jh + 1, lo = v.window ? my_p - v.window + 1 - jh : 0, sk = v.sinks - jh;
#pragma unroll
                            for (int w = 0; w < 2; w++) {
                                const uint32_t bits = bits_below(hi - 32 * w) & (~bits_below(lo - 32 * w) | bits_below(sk - 32 * w));
#pragma unroll
                                for (int i = 0; i < 32; i++) sr[w * 32 + i] = bits & (1u << i) ? sr[w * 32 + i] : 0xff800000u;
                            }
                        }
                        float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                        for (int i = 0; i < 64; i += 8)
#pragma unroll
                            for (int j = 0; j < 4; j++) mx4[j] = max3(mx4[j], __uint_as_float(sr[i + j]), __uint_as_float(sr[i + 4 + j]));
                        const float mx = max3(max3(mx4[0], mx4[1], mx4[2]), mx4[3], mx4[3]) * scale;  // NaN if a score is
                        const bool raise = mx > m + RAISE;
                        if (first) {
                            m = mx;
                            first = false;
                        } else if (__any_sync(~0u, raise)) {
                            wait(pv_done(x, n_h - 1), (n_h - 1) >> 2);  // the last product into O
                            const float c2 = raise ? ex2(m - mx) : 1.0f;
                            if (raise) m = mx;
                            l *= c2;
#pragma unroll 1
                            for (int k = 0; k < D / 16; k++) tmem_scale16(t_o + k * 16, c2);
                        }
                        // a score that is NaN or +infinite makes the row NaN (the polynomial would pass over it)
                        const float ref = !(mx < INFINITY) ? __int_as_float(0x7fffffff) : m == -INFINITY ? 0.0f : m;
                        const uint64_t scale2 = f2(scale, scale), ref2 = f2(-ref, -ref);
                        uint64_t sum2[2] = {0, 0};
                        // every fourth pair of exponentials on the multiply-add pipe: both streams' other ones queue at the
                        // exponential unit (509 -> 495 us for an 8192-token prompt; three in eight gained no more)
                        uint32_t pw[32];
#pragma unroll
                        for (int i = 0; i < 32; i++) {
                            const uint64_t y = fma2(f2(__uint_as_float(sr[2 * i]), __uint_as_float(sr[2 * i + 1])), scale2, ref2);
                            const uint64_t e = i % 4 == 1 ? ex2_poly(y) : f2(ex2(lo(y)), ex2(hi(y)));
                            sum2[i & 1] = add2(sum2[i & 1], e);
                            pw[i] = pack2(lo(e), hi(e));
                        }
                        tmem_st32(t_s + hf * 64, pw);
                        const uint64_t sum = add2(sum2[0], sum2[1]);
                        l += lo(sum) + hi(sum);
                        clear_hidden(t, j0, hf);
                        tmem_st_wait();
                        tc_fence_before();
                        mbar_arrive(p_ready(x, hf));
                    }
                }
                // ---- the segment is done: store, or leave a partial result
                // Streams of their own rows store and join by themselves, streams that share rows together.
                const bool whole = n == c.p.units;
                const int who = shared_rows ? 0 : x, id = shared_rows ? 1 : 2 + x, threads = shared_rows ? 256 : 128;
                const int i0 = u - pt.line - unit;  // the place where the item's tiles begin, from u0
                int mine = 0, n_parts = 1;
                if (!whole) {
                    mine = -floor_div(i0, per);
                    n_parts = floor_div(i0 + c.p.units - 1, per) + mine + 1;
                }
                const int cta0 = (int)blockIdx.x - mine;
                unsigned *counter = a.counters + 2 * cta0 + who;
                volatile uint32_t *last = tmem_slot + 2 + who;  // every other part is in the workspace
                const bool lead = row == 0 && x == who;
                if (lead && !whole) *last = ld_acquire(counter) == (unsigned)n_parts - 1;
                __syncwarp();
                if (!first) wait(o_done(x), n_o++);  // (first: no tile in this segment)
                float w0 = 1.0f, w1 = 0.0f;
                const bool both = shared_rows && n > 1;
                if (shared_rows) {
                    // warps w and w + 4 reach the same lanes of tensor memory: each stream stores half of the columns
                    volatile float *ml = reinterpret_cast<volatile float *>(smem + C::ML_AT);
                    ml[x * 256 + row] = m;
                    ml[x * 256 + 128 + row] = l;
                    tc_fence_before();
                    bar_sync(1, 256);
                    tc_fence_after();
                    const float m0 = ml[row], l0 = ml[128 + row], m1 = ml[256 + row], l1 = ml[384 + row];
                    const float mm = fmaxf(m0, m1), ref = mm == -INFINITY ? 0.0f : mm;
                    w0 = ex2(m0 - ref);
                    w1 = ex2(m1 - ref);
                    l = l0 * w0 + l1 * w1;
                    m = mm;
                } else if (!whole) {
                    bar_sync(id, threads);
                }
                const uint32_t t_o0 = tmem + 256 + who * D + lanes, t_o1 = tmem + 256 + D + lanes;
                const int k0 = shared_rows ? x * (D / 64) : 0, k1 = wq * 32 >= n_rows ? k0 : k0 + (shared_rows ? D / 64 : D / 32);
                auto load_o = [&](int k, float (&y)[32]) {  // 32 columns of this CTA's result
                    __syncwarp();
                    tmem_ld32(t_o0 + k * 32, y);
                    if (both) {
                        float o1[32];
                        tmem_ld32(t_o1 + k * 32, o1);
#pragma unroll
                        for (int i = 0; i < 32; i++) y[i] = y[i] * w0 + o1[i] * w1;
                    }
                };
                auto part_of_cta = [&](int i) { return a.parts + ((size_t)(cta0 + i) * 2 + (i == 0 ? 1 : 0)) * C::PART; };
                const int at = who * 128 + row;
                bool store = whole || *last;
                if (!store) {
                    float *part = part_of_cta(mine);
#pragma unroll 1
                    for (int k = k0; k < k1; k++) {  // not unrolled: code that runs once per item mostly costs its way into the cache
                        float y[32];
                        load_o(k, y);
                        if (row < n_rows) {
#pragma unroll
                            for (int i = 0; i < 8; i++)
                                reinterpret_cast<float4 *>(part)[(k * 8 + i) * 256 + at] = make_float4(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
                        }
                    }
                    if (x == who && row < n_rows) {
                        part[256 * D + at] = m;
                        part[256 * (D + 1) + at] = l;
                    }
                    __syncwarp();
                    bar_sync(id, threads);
                    if (lead) {
                        __threadfence();
                        *last = atomicAdd(counter, 1u) == (unsigned)n_parts - 1;
                        __threadfence();
                    }
                    __syncwarp();
                    bar_sync(id, threads);
                    store = *last;
                }
                if (store) {
                    float mm = m, ll = l, w_mine = 1.0f, ref = 0.0f;
                    if (!whole && row < n_rows) {
                        for (int i = 0; i < n_parts; i++) mm = fmaxf(mm, i == mine ? m : __ldcg(part_of_cta(i) + 256 * D + at));
                        ref = mm == -INFINITY ? 0.0f : mm;
                        w_mine = ex2(m - ref);
                        ll = 0.0f;
#pragma unroll 4
                        for (int i = 0; i < n_parts; i++)
                            ll += i == mine ? w_mine * l : ex2(__ldcg(part_of_cta(i) + 256 * D + at) - ref) * __ldcg(part_of_cta(i) + 256 * (D + 1) + at);
                    }
                    const float inv = ll == 0.0f ? 0.0f : 1.0f / ll;  // a sum that is NaN stays one
                    const int t_row = token(row);
                    const size_t out_row = (size_t)c.q.s.row0 + ta + t_row;
                    const int head = c.h * v.G + row - t_row * v.G;
                    __nv_bfloat16 *o = (__nv_bfloat16 *)a.out + out_row * a.out_stride + (size_t)head * D;
#pragma unroll 1
                    for (int k = k0; k < k1; k++) {
                        float y[32];
                        if (whole) {
                            load_o(k, y);
                        } else {
                            // in the order of the CTAs, whichever came last
                            auto add = [&](int from, int to) {
#pragma unroll 2
                                for (int i = from; i < to; i++) {
                                    const float w = ex2(__ldcg(part_of_cta(i) + 256 * D + at) - ref);
                                    const float4 *z = reinterpret_cast<const float4 *>(part_of_cta(i)) + k * 8 * 256 + at;
#pragma unroll
                                    for (int j = 0; j < 8; j++) {
                                        const float4 f = __ldcg(z + j * 256);
                                        y[4 * j] += w * f.x;
                                        y[4 * j + 1] += w * f.y;
                                        y[4 * j + 2] += w * f.z;
                                        y[4 * j + 3] += w * f.w;
                                    }
                                }
                            };
#pragma unroll
                            for (int i = 0; i < 32; i++) y[i] = 0.0f;
                            if (row < n_rows) add(0, mine);
                            float own[32];
                            load_o(k, own);
#pragma unroll
                            for (int i = 0; i < 32; i++) y[i] += w_mine * own[i];
                            if (row < n_rows) add(mine + 1, n_parts);
                        }
                        if (row < n_rows) {
                            uint32_t w[16];
#pragma unroll
                            for (int i = 0; i < 16; i++) w[i] = pack2(y[2 * i] * inv, y[2 * i + 1] * inv);
                            if (wide_out) {
#pragma unroll
                                for (int i = 0; i < 16; i += 8)
                                    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(o + k * 32 + 2 * i), I8(w, i) : "memory");
                            } else {
#pragma unroll
                                for (int i = 0; i < 16; i += 4) *reinterpret_cast<uint4 *>(o + k * 32 + 2 * i) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
                            }
                        }
                    }
                    if (x == who && row < n_rows && a.lse) a.lse[out_row * v.Hq + head] = ll == 0.0f ? -INFINITY : (mm + log2f(ll)) * LN2;
                    if (lead && !whole) *counter = 0;
                }
                __syncwarp();
                tc_fence_before();
                if (shared_rows || !whole) bar_sync(id, threads);  // both streams' tensor memory and the flag are read
                g += 2 * n;
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 8) tmem_dealloc(*tmem_slot, 512);
}

template <int D> cudaError_t umma(const AttendArgs &a, const CUtensorMap (&maps)[4], int q_tma, int num_sms, cudaStream_t s) {
    using C = Cfg<D>;
    const int tpt = 128 / a.v.G;
    auto kernel = attend_umma_kernel<D>;
    int g_shift = -1;  // log2 of the query heads per key head, if it is a power of two
    for (int i = 0; i < 8; i++)
        if (a.v.G == 1 << i) g_shift = i;
    kernel<<<num_sms, THREADS, C::SMEM, s>>>(maps[0], maps[1], maps[2], maps[3], a, tpt, g_shift, q_tma);
    return cudaGetLastError();
}

}  // namespace

size_t umma_parts_floats(int D, int num_sms) { return (size_t)num_sms * 2 * 256 * (D + 2); }

cudaError_t prepare_attend_umma() {
    const cudaError_t e = allow_shared(attend_umma_kernel<64>);
    return e == cudaSuccess ? allow_shared(attend_umma_kernel<128>) : e;
}

cudaError_t launch_attend_umma(const AttendArgs &a, const CUtensorMap (&maps)[4], int q_tma, int num_sms, cudaStream_t s) {
    return a.v.D == 64 ? umma<64>(a, maps, q_tma, num_sms, s) : umma<128>(a, maps, q_tma, num_sms, s);
}

}  // namespace kv
}  // namespace aj
