// Product of rows in 8 bits:  y[t][n] = (sum_k xq[t][k] * wq[n][k]) * xscale[t] * wscale[n] + bias[n].
// The sum is exact in int32 (at most 2^17 - 1 products of at most 2^14 each), so any order and any split of it gives
// the same bits.
//
// Four kernels, chosen by the number of tokens and the work there is for the SMs (choose() below), and one for no columns:
//   k_linear_rows   one token: bound by reading the weights once; int8 dot products in the ordinary pipes
//   k_linear_few    up to 32 tokens: the same, with warp-wide products
//   k_linear_tile   one CTA a tile of 128 channels by up to 256 tokens; the columns of a tile may be split over the CTAs of a
//                   cluster, whose int32 partial sums meet in distributed shared memory
//   k_linear_pair   two CTAs a tile of 256 channels by up to 256 tokens, persistent, accumulators double-buffered in tensor memory
// The tile kernels put the WEIGHTS on the rows of the tensor cores' tile (the lanes of tensor memory) and the tokens on its
// columns: a tile is then never wider in tokens than there are tokens to a multiple of 32, and a warp that reads one
// accumulator column holds 32 neighbouring channels of one token, which it stores as one contiguous piece of y - no
// staging in shared memory, no alignment asked of y or ldy.
#include <cuda.h>

#include <algorithm>
#include <cmath>

#include "dnns_internal.cuh"

namespace dnns {

namespace {

struct LinearArgs {
    const int8_t *xq, *wq;
    const float *xscale, *wscale, *bias;  // bias nullable
    void* y;
    uint32_t* status;
    int64_t ldx, ldw, ldy;
    int32_t rows, k, n;
};

constexpr uint32_t kFullMask = 0xFFFFFFFFu;

template <int DT>
__device__ __forceinline__ void store_out(void* y, int64_t at, float v) {
    if (DT == DNNS_F32) {
        static_cast<float*>(y)[at] = v;
    } else {
        uint32_t d;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(0.0f), "f"(v));
        static_cast<uint16_t*>(y)[at] = (uint16_t)d;
    }
}

// What a sum becomes.  The int32 sum is rounded to fp32 here (24 bits: half a unit of the last place of an fp32 result).
__device__ __forceinline__ float scaled(int32_t acc, float xs, float ws, float bias) { return fmaf((float)acc * ws, xs, bias); }

// ================= few tokens =================
// Bound by reading the weights once, so what counts is that enough of them are on their way: a warp has R channels, its lanes
// 16 bytes of each at a time, several loads deep; `parts` warps share a channel's columns where there are few channels.
// The tokens are read beside them, from the L1 cache but for a block's first warp (the weights pass it by).
constexpr int kRowsWarps = 8;

// (Not the read-only path, here and for the tokens: a chained kernel begins while the one that writes them may still run.)
__device__ __forceinline__ int4 stream16(const int8_t* p) {
    int4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ int4 token16(const int8_t* p) { return *reinterpret_cast<const int4*>(p); }
__device__ __forceinline__ int32_t dot16(const int4& a, const int4& b, int32_t c) { return __dp4a(a.x, b.x, __dp4a(a.y, b.y, __dp4a(a.z, b.z, __dp4a(a.w, b.w, c)))); }

// M tokens at most (a.rows of them), blockIdx.y the token group.  Launched for one token: with two and more, k_linear_few or a tile reads
// the weights no more often and multiplies faster.
// 1 x 4096 x 4096 (tokens, columns, channels): 3.0 us with the weights in L2, 4.6 with them in HBM (floor 2.6, and 1.7 of that time is
// what any kernel of this size takes); 1 x 4096 x 14336 11.2 (5.2 TB/s, floor 9.0); 1 x 1024 x 1024 1.8.
template <int M, int R, int DT>
__global__ void __launch_bounds__(32 * kRowsWarps) k_linear_rows(const LinearArgs a, int32_t parts) {
    chain_go();
    chain_wait();
    constexpr int U = 4;  // loads deep
    __shared__ int32_t s_part[kRowsWarps][R * M];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int group = warp / parts, part = warp - group * parts;
    const int32_t n0 = (int32_t)(((int64_t)blockIdx.x * (kRowsWarps / parts) + group) * R);
    const int32_t t0 = blockIdx.y * M, vecs = a.k >> 4, step = 32 * parts;
    int32_t acc[R][M];
    const int8_t *w[R], *x[M];
#pragma unroll
    for (int i = 0; i < R; ++i) w[i] = a.wq + (int64_t)min(n0 + i, a.n - 1) * a.ldw;  // (rows past the end repeat the last)
#pragma unroll
    for (int t = 0; t < M; ++t) x[t] = a.xq + (int64_t)min(t0 + t, a.rows - 1) * a.ldx;
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
        for (int t = 0; t < M; ++t) acc[i][t] = 0;
    int32_t v = part * 32 + lane;
    for (; v + (U - 1) * step < vecs; v += U * step) {
        int4 wv[U][R];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < R; ++i) wv[u][i] = stream16(w[i] + 16 * (v + u * step));
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int t = 0; t < M; ++t) {
                const int4 xv = token16(x[t] + 16 * (v + u * step));
#pragma unroll
                for (int i = 0; i < R; ++i) acc[i][t] = dot16(wv[u][i], xv, acc[i][t]);
            }
    }
    for (; v < vecs; v += step) {
        int4 wv[R];
#pragma unroll
        for (int i = 0; i < R; ++i) wv[i] = stream16(w[i] + 16 * v);
#pragma unroll
        for (int t = 0; t < M; ++t) {
            const int4 xv = token16(x[t] + 16 * v);
#pragma unroll
            for (int i = 0; i < R; ++i) acc[i][t] = dot16(wv[i], xv, acc[i][t]);
        }
    }
    // the last columns, fewer than 16: a lane each
    if (const int32_t c = (vecs << 4) + lane; part == 0 && c < a.k) {
#pragma unroll
        for (int t = 0; t < M; ++t)
#pragma unroll
            for (int i = 0; i < R; ++i) acc[i][t] += (int32_t)w[i][c] * (int32_t)x[t][c];
    }
    // lane l ends up with the l-th of the R * M sums (32 at a time)
    constexpr int kSums = R * M;
    int32_t mine[(kSums + 31) / 32];
#pragma unroll
    for (int q = 0; q < kSums; ++q) {
        const int32_t sum = __reduce_add_sync(kFullMask, acc[q / M][q % M]);
        if (lane == (q & 31)) mine[q >> 5] = sum;
    }
    if (parts > 1) {
#pragma unroll
        for (int b = 0; b < (kSums + 31) / 32; ++b)
            if (b * 32 + lane < kSums) s_part[warp][b * 32 + lane] = mine[b];
        __syncthreads();
        if (part) return;
#pragma unroll
        for (int b = 0; b < (kSums + 31) / 32; ++b)
            if (b * 32 + lane < kSums)
                for (int i = 1; i < parts; ++i) mine[b] += s_part[warp + i][b * 32 + lane];
    }
#pragma unroll
    for (int b = 0; b < (kSums + 31) / 32; ++b) {
        const int q = b * 32 + lane, n = n0 + q / M, t = t0 + q % M;
        if (q < kSums && n < a.n && t < a.rows)
            store_out<DT>(a.y, (int64_t)t * a.ldy + n, scaled(mine[b], a.xscale[t], a.wscale[n], a.bias ? a.bias[n] : 0.0f));
    }
}

// No columns: all sums are 0.  (Not a copy of the bias: a scale that is NaN still gives NaN.)
template <int DT>
__global__ void __launch_bounds__(256) k_linear_empty(const LinearArgs a) {
    chain_go();
    chain_wait();
    const int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (n >= a.n) return;
    for (int64_t t = blockIdx.y; t < a.rows; t += gridDim.y) store_out<DT>(a.y, t * a.ldy + n, scaled(0, a.xscale[t], a.wscale[n], a.bias ? a.bias[n] : 0.0f));
}

// ================= a few more tokens: warp-wide products =================
// Still bound by reading the weights once, but with dot products lane by lane the tokens, read once a channel, become the larger
// traffic (L1).  A warp-wide product of 16 channels x 32 columns by 8 tokens reads them once for 16 channels.  The sum over the
// columns may go in any order, so a lane feeds the product with 16 neighbouring bytes of a row at a time: lane (g, q) has
// bytes 16 q .. of 64 of channels g and g + 8 and of token g, words 0, 1 for one product and 2, 3 for the next.  `parts` warps
// share the columns of a group of 16 channels and meet in shared memory.
__device__ __forceinline__ void warp_product(int32_t (&d)[4], int32_t a0, int32_t a1, int32_t a2, int32_t a3, int32_t b0, int32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void lane_product(int32_t (&d)[4], const int4& lo, const int4& hi, const int4& x) {
    warp_product(d, lo.x, hi.x, lo.y, hi.y, x.x, x.y);
    warp_product(d, lo.z, hi.z, lo.w, hi.w, x.z, x.w);
}
// Bytes c .. c + 15 of a row of k bytes, those past the end as 0 (never read).
__device__ __forceinline__ int4 row16(const int8_t* row, int32_t c, int32_t k) {
    if (c + 16 <= k) return *reinterpret_cast<const int4*>(row + c);
    uint32_t b[16], w[4];
#pragma unroll
    for (int i = 0; i < 16; ++i) b[i] = c + i < k ? (uint32_t)(uint8_t)row[c + i] : 0u;  // (all on their way together)
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = b[4 * i] | b[4 * i + 1] << 8 | b[4 * i + 2] << 16 | b[4 * i + 3] << 24;
    return make_int4((int)w[0], (int)w[1], (int)w[2], (int)w[3]);
}

// 8 * TB tokens at most (a.rows of them): a warp has 16 channels, on the rows of its products, and all the tokens on the columns.
// Bound by the weights' way like the kernel above, and for more tokens by the products' issue and the tokens read from L1 for each
// 16 channels: 16 x 4096 x 4096 5.9 us (floor 2.6), 5 x 700 x 3000 4.4.
template <int TB, int DT>
__global__ void __launch_bounds__(32 * kRowsWarps, 2) k_linear_few(const LinearArgs a, int32_t parts) {
    chain_go();
    chain_wait();
    constexpr int U = 4, kSums = 16 * 8 * TB;  // loads deep; results of a group
    __shared__ int32_t s_part[kRowsWarps][kSums];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, q = lane & 3;
    const int groups = kRowsWarps / parts, group = warp / parts, part = warp - group * parts;
    const int32_t n0 = (int32_t)(((int64_t)blockIdx.x * groups + group) * 16);
    const int8_t* lo = a.wq + (int64_t)min(n0 + g, a.n - 1) * a.ldw;  // (rows and tokens past the end repeat the last)
    const int8_t* hi = a.wq + (int64_t)min(n0 + g + 8, a.n - 1) * a.ldw;
    const int8_t* x[TB];
#pragma unroll
    for (int t = 0; t < TB; ++t) x[t] = a.xq + (int64_t)min(8 * t + g, a.rows - 1) * a.ldx;
    int32_t acc[TB][4];
#pragma unroll
    for (int t = 0; t < TB; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[t][i] = 0;
    const int32_t whole = a.k >> 6, step = parts;  // pieces of 64 columns
    int32_t b = part;
    for (; b + (U - 1) * step < whole; b += U * step) {
        int4 wl[U], wh[U];
#pragma unroll
        for (int u = 0; u < U; ++u) wl[u] = stream16(lo + 64 * (b + u * step) + 16 * q), wh[u] = stream16(hi + 64 * (b + u * step) + 16 * q);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int t = 0; t < TB; ++t) lane_product(acc[t], wl[u], wh[u], token16(x[t] + 64 * (b + u * step) + 16 * q));
    }
    for (; b < whole; b += step) {
        const int4 wl = stream16(lo + 64 * b + 16 * q), wh = stream16(hi + 64 * b + 16 * q);
#pragma unroll
        for (int t = 0; t < TB; ++t) lane_product(acc[t], wl, wh, token16(x[t] + 64 * b + 16 * q));
    }
    if (part == parts - 1 && (a.k & 63)) {
        const int32_t c = 64 * whole + 16 * q;
        const int4 wl = row16(lo, c, a.k), wh = row16(hi, c, a.k);
#pragma unroll
        for (int t = 0; t < TB; ++t) lane_product(acc[t], wl, wh, row16(x[t], c, a.k));
    }
    // sum [token][channel] of the group
#pragma unroll
    for (int t = 0; t < TB; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) s_part[warp][(8 * t + 2 * q + (i & 1)) * 16 + g + 8 * (i >> 1)] = acc[t][i];
    __syncthreads();
    for (int i = threadIdx.x; i < groups * kSums; i += 32 * kRowsWarps) {
        const int grp = i / kSums, at = i - grp * kSums, t = at >> 4;
        const int32_t n = (int32_t)(((int64_t)blockIdx.x * groups + grp) * 16) + (at & 15);
        if (t >= a.rows || n >= a.n) continue;
        int32_t sum = 0;
        for (int p = 0; p < parts; ++p) sum += s_part[grp * parts + p][at];
        store_out<DT>(a.y, (int64_t)t * a.ldy + n, scaled(sum, a.xscale[t], a.wscale[n], a.bias ? a.bias[n] : 0.0f));
    }
}

// ================= tensor cores: the pieces both tile kernels are made of =================
constexpr int kBlockK = 128;                   // columns of a stage: one 128-byte swizzle row of int8
constexpr int kTileRows = 128;                 // channels of a CTA
constexpr uint32_t kWeightBytes = kTileRows * kBlockK;
constexpr uint64_t kWaitLimitNs = 500ull * 1000ull * 1000ull;  // a wait that lasts this long is given up (status TIMEOUT)

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// The address, in the cluster's shared window, of what `local` is in CTA `rank`.
__device__ __forceinline__ uint32_t in_cta(uint32_t local, uint32_t rank) {
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(local), "r"(rank));
    return a;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void mbar_init(uint64_t* bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_addr(bar)), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_expect(uint64_t* bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_addr(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive_at(uint32_t cluster_addr) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
__device__ __forceinline__ bool mbar_try(uint64_t* bar, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"  // may sleep up to the hint (ns) before it answers
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(smem_addr(bar)), "r"(parity), "r"(20000u)
        : "memory");
    return done != 0;
}
__device__ __forceinline__ uint64_t global_ns() {
    uint64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}
#ifdef DNNS_BOUNDS_CHECK
// Checked build only: where set, a wait that does not find its phase complete at once is given up, so that the tests reach what follows.
__device__ uint32_t g_hurry = 0;
__device__ __forceinline__ bool mbar_test(uint64_t* bar, uint32_t parity) {
    uint32_t done;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(done) : "r"(smem_addr(bar)), "r"(parity) : "memory");
    return done != 0;
}
#endif
// Wait for a phase of an mbarrier, but not for ever: false when the wait was given up, or another thread of the CTA gave
// up before.  (The timer takes long to read: it is looked at only after many tries.)
__device__ __forceinline__ bool mbar_wait(uint64_t* bar, uint32_t parity, volatile uint32_t* gave_up) {
#ifdef DNNS_BOUNDS_CHECK
    if (*(volatile uint32_t*)&g_hurry) {
        if (mbar_test(bar, parity)) return true;
        *gave_up = 1;
        return false;
    }
#endif
    if (mbar_try(bar, parity)) return true;
    uint64_t since = 0;
    for (uint32_t spin = 1;; ++spin) {
        if (mbar_try(bar, parity)) return true;
        if ((spin & 15u) == 0) {
            const uint64_t now = global_ns();
            if (since == 0) since = now;
            if (*gave_up || now - since > kWaitLimitNs) {
                *gave_up = 1;
                return false;
            }
        }
    }
}
// The wait for what is in flight when a kernel gives up: it ends by itself, so the limit is only the last resort.
__device__ __forceinline__ void mbar_drain(uint64_t* bar, uint32_t parity) {
    const uint64_t since = global_ns();
    while (!mbar_try(bar, parity) && global_ns() - since < kWaitLimitNs) {
    }
}
// Counts `bytes` at a barrier of this CTA as if a copy had brought them.
__device__ __forceinline__ void mbar_count(uint64_t* bar, uint32_t bytes) {
    asm volatile("mbarrier.complete_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(smem_addr(bar)), "r"(bytes) : "memory");
}
// Box of a tensor map into this CTA's shared memory; `bar` counts its bytes (PAIR: may be the pair's first CTA's barrier).
template <bool PAIR>
__device__ __forceinline__ void tile_load(uint32_t dst, const CUtensorMap* map, int32_t x, int32_t y, uint32_t bar) {
    if (PAIR)
        asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
                     "l"(map), "r"(x), "r"(y), "r"(bar)
                     : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"(map), "r"(x),
                     "r"(y), "r"(bar)
                     : "memory");
}
// Shared-memory operand: rows of 128 bytes in the 128-byte swizzle, groups of 8 rows 1024 bytes apart, columns contiguous.
__device__ __forceinline__ uint64_t operand(uint32_t addr) {
    return (uint64_t)((addr >> 4) & 0x3FFFu) | (1ull << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
// Instruction descriptor: int32 accumulators, signed 8-bit operands, both with contiguous columns, M x N.
__host__ __device__ constexpr uint32_t mma_shape(uint32_t m, uint32_t n) { return (2u << 4) | (1u << 7) | (1u << 10) | ((n >> 3) << 17) | ((m >> 4) << 24); }
template <bool PAIR>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t shape, bool add) {
    if (PAIR)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b),
                     "r"(shape), "r"((uint32_t)add)
                     : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b),
                     "r"(shape), "r"((uint32_t)add)
                     : "memory");
}
// Arrive at `bar` (PAIR: of both CTAs) once all products issued so far are done.
template <bool PAIR>
__device__ __forceinline__ void mma_commit(uint64_t* bar) {
    if (PAIR)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_addr(bar)), "h"((uint16_t)3)
                     : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ void mma_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void mma_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
template <bool PAIR>
__device__ __forceinline__ void tmem_alloc(uint32_t* where, uint32_t columns) {
    if (PAIR) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(where)), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    } else {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(where)), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
}
template <bool PAIR>
__device__ __forceinline__ void tmem_free(uint32_t at, uint32_t columns) {
    if (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns));
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns));
}
// 32 accumulator columns of this warp's 32 lanes.
__device__ __forceinline__ void tmem_load32(uint32_t at, int32_t (&v)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]),
          "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]),
          "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
        : "r"(at));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

// Up to 32 columns (tokens t0 .. t0 + left - 1) of one channel a lane: scale and store.  The tokens' scales: a lane fetches one and
// they go round by shuffles, or (SHARED) they are in shared memory.  Measured: in shared memory, fetched beside the
// products, 200 x 4096 x 4096 over clusters of two 11.4 -> 10.2 us; but a whole tile's 128 to 256 columns stored without the shuffles'
// pace between them take longer (4000 x 300 x 300 5.8 -> 7.6), so tiles of one CTA or a pair keep the shuffles.
template <int DT, bool SHARED = false>
__device__ __forceinline__ void store_columns(const LinearArgs& a, const int32_t (&v)[32], int32_t t0, int32_t left, int32_t n, float ws, float bias,
                                              const float4* scales = nullptr) {
    typedef typename std::conditional<DT == DNNS_F32, float, uint16_t>::type T;
    const int lane = threadIdx.x & 31;
    const float mine = !SHARED && lane < left ? a.xscale[t0 + lane] : 0.0f;
    T* y = static_cast<T*>(a.y) + (int64_t)t0 * a.ldy + n;
    const bool in = n < a.n;
#pragma unroll
    for (int j = 0; j < 32; ++j) {
        float xs;
        if constexpr (SHARED) {
            const float4 four = scales[j / 4];
            xs = j & 2 ? (j & 1 ? four.w : four.z) : (j & 1 ? four.y : four.x);
        } else {
            xs = __shfl_sync(kFullMask, mine, j);
        }
        if (in && j < left) store_out<DT>(y, 0, scaled(v[j], xs, ws, bias));
        y += a.ldy;
    }
}

constexpr int kMaxStages = 10;
struct TileShared {  // in front of the stages
    uint64_t full[kMaxStages], empty[kMaxStages], done[2], taken[2], drain;
    uint32_t tmem, gave_up, issued[2];  // (pair: stages that the CTAs had copied when they gave up)
    alignas(16) float scales[128];  // of the tokens that a CTA of a cluster stores
};
constexpr uint32_t kSharedHead = 2048;
static_assert(sizeof(TileShared) <= kSharedHead, "head of the shared memory");

__device__ __forceinline__ unsigned char* shared_base() {
    extern __shared__ unsigned char raw[];
    return raw + ((1024u - (smem_addr(raw) & 1023u)) & 1023u);  // (the swizzle repeats every 1024 bytes)
}

// ================= one CTA a tile, its columns split over a cluster =================
// Bound by what comes from L2 into an SM, about 60 bytes a clock, and by 3 us that do not depend on the size: the tensor maps, the
// first stage's way, the accumulators' way out and the cluster's barrier.  A tile's columns are split so that every SM has a share of
// them: 64 x 4096 x 4096 is 32 tiles, 9.9 us unsplit and 7.6 in four.  The CTAs of a cluster exchange partial sums so that each ends
// with a share of the tokens: the sums cross once, and all of them scale, convert and store.  24 x 4096 x 14336 13.7 us (4.3 TB/s of
// weights, floor 9.1; 112 of the SMs have a tile), 128 x 4096 x 4096 8.3, 200 x 4096 x 4096 9.3, 333 x 5003 x 2741 (fp32 result) 11.0.
constexpr int kTileThreads2 = 192;  // warp 0 loads, warp 1 issues the products, warps 2 .. 5 read the accumulators

// How a product is cut: tiles of `tokens` (a multiple of 32 up to 256), each over `split` CTAs of a cluster; a share of the
// tokens, tokens / split, is a multiple of 4.
struct TilePlan {
    int32_t tokens, t_tiles, split, stages;
    __host__ __device__ uint32_t stage_bytes() const { return kWeightBytes + (uint32_t)tokens * kBlockK; }
    // the stages, then (split) the partial sums that the other CTAs send
    __host__ __device__ uint32_t sums_at() const { return kSharedHead + (uint32_t)stages * stage_bytes(); }
    uint32_t shared_bytes() const { return sums_at() + (split > 1 ? (uint32_t)tokens * kTileRows * 4 : 0) + 1024; }
};
// Given up, here or in another warp: what is in flight ends before this CTA leaves its memory.  `it`: stages copied (warp 0).  (Not
// inlined, as pair_gave_up: inside the kernels this code cost calls that never reach it 0.1 to 0.3 us.)
__device__ __noinline__ void tile_gave_up(TileShared& s, int warp, int lane, int32_t it, int32_t stages, uint32_t* status) {
    if (lane == 0) {
        atomicCAS(status, 0u, (uint32_t)DNNS_ERR_TIMEOUT);
        if (warp == 0)
            for (int32_t u = max(0, it - stages); u < it; ++u) mbar_drain(&s.full[u % stages], (u / stages) & 1);
        if (warp == 1) mma_commit<false>(&s.drain), mbar_drain(&s.drain, 0);
    }
    __syncwarp();
}
template <int DT>
__global__ void __launch_bounds__(kTileThreads2) k_linear_tile(const LinearArgs a, const __grid_constant__ CUtensorMap wmap,
                                                               const __grid_constant__ CUtensorMap xmap, const TilePlan plan) {
    unsigned char* base = shared_base();
    TileShared& s = *reinterpret_cast<TileShared*>(base);
    const uint32_t stages = smem_addr(base) + kSharedHead, stage_bytes = plan.stage_bytes();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int32_t split = plan.split, tile = blockIdx.x / split, slice = blockIdx.x - tile * split;
    const int32_t t_tile = tile % plan.t_tiles, t0 = t_tile * plan.tokens, n0 = tile / plan.t_tiles * kTileRows;
    const int32_t blocks = (a.k + kBlockK - 1) / kBlockK;
    const int32_t kb0 = (int32_t)((int64_t)blocks * slice / split), kbs = (int32_t)((int64_t)blocks * (slice + 1) / split) - kb0;
    const uint32_t columns = plan.tokens <= 32 ? 32 : plan.tokens <= 64 ? 64 : plan.tokens <= 128 ? 128 : 256;  // of tensor memory

    if (threadIdx.x == 0) {
        for (int i = 0; i < plan.stages; ++i) mbar_init(&s.full[i], 1), mbar_init(&s.empty[i], 1);
        mbar_init(&s.done[0], 1);
        mbar_init(&s.drain, 1);
        s.gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&wmap) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&xmap) : "memory");
    }
    if (warp == 1) {
        __syncwarp();
        tmem_alloc<false>(&s.tmem, columns);
        mma_fence_before();
    }
    __syncthreads();
    mma_fence_after();
    // (the cluster's CTAs are all there before one of them sends its sums to another: waited for below)
    if (split > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    chain_go();  // (not before this CTA has its tensor memory: the next kernel's CTAs would take it and wait for this one's end)
    chain_wait();
    const uint32_t tmem = s.tmem;
    volatile uint32_t* gave_up = &s.gave_up;

    int32_t it = 0;  // lane 0 of warps 0 and 1: stages copied, and multiplied
    if (warp == 0) {
        if (lane == 0) {
            int32_t st = 0;
            uint32_t turn = 1;
            for (; it < kbs; ++it) {
                if (!mbar_wait(&s.empty[st], turn, gave_up)) break;
                const uint32_t at = stages + st * stage_bytes, bar = smem_addr(&s.full[st]);
                mbar_expect(&s.full[st], stage_bytes);
                tile_load<false>(at, &wmap, (kb0 + it) * kBlockK, n0, bar);
                tile_load<false>(at + kWeightBytes, &xmap, (kb0 + it) * kBlockK, t0, bar);
                if (++st == plan.stages) st = 0, turn ^= 1;
            }
        }
    } else if (warp == 1) {
        if (lane == 0) {
            const uint32_t shape = mma_shape(kTileRows, plan.tokens);
            int32_t st = 0;
            uint32_t turn = 0;
            for (; it < kbs; ++it) {
                if (!mbar_wait(&s.full[st], turn, gave_up)) break;
                mma_fence_after();
                const uint32_t at = stages + st * stage_bytes;
                const uint64_t w = operand(at), x = operand(at + kWeightBytes);
#pragma unroll
                for (int q = 0; q < kBlockK / 32; ++q) mma<false>(tmem, w + 2 * q, x + 2 * q, shape, it > 0 || q > 0);
                mma_commit<false>(&s.empty[st]);
                if (++st == plan.stages) st = 0, turn ^= 1;
            }
            if (it == kbs) mma_commit<false>(&s.done[0]);
        }
    }
    const int quarter = warp & 3;  // tensor memory lanes a warp may read: 32 * (its index mod 4) ..
    const int32_t n = n0 + 32 * quarter + lane;
    const float ws = warp >= 2 && n < a.n ? a.wscale[n] : 0.0f, bias = warp >= 2 && a.bias && n < a.n ? a.bias[n] : 0.0f;
    const int share = plan.tokens / split, t1 = t0 + slice * share;  // the tokens that this CTA stores
    if (split > 1)
        for (int i = threadIdx.x; i < share; i += kTileThreads2) s.scales[i] = t1 + i < a.rows ? a.xscale[t1 + i] : 0.0f;
    // everybody waits for the sums: once they are there, no copy and no product of this CTA is in flight
    __syncwarp();
    const bool ok = __shfl_sync(kFullMask, (int)(lane == 0 && mbar_wait(&s.done[0], 0, gave_up)), 0);
    mma_fence_after();
    const uint32_t row = tmem + ((uint32_t)(32 * quarter) << 16);
    if (!ok) tile_gave_up(s, warp, lane, it, plan.stages, a.status);
    __syncwarp();
    if (split == 1) {
        if (warp >= 2 && ok) {
#pragma unroll 1
            for (int c = 0; c < plan.tokens && t0 + c < a.rows; c += 32) {
                int32_t v[32];
                tmem_load32(row + c, v);
                store_columns<DT>(a, v, t0 + c, a.rows - t0 - c, n, ws, bias);
            }
        }
    } else {
        // the cluster's CTAs share the columns out: CTA r gets everybody's sums of columns r * share .., four columns of a channel
        // in 16 bytes
        const uint32_t sums = smem_addr(base) + plan.sums_at();
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");  // (the barrier arrived at above)
        if (warp >= 2 && ok) {
            int to = 0, slot = slice * (share / 4);  // of the next four columns: the CTA they go to, and their place there
            uint32_t dest = in_cta(sums, 0);
#pragma unroll 1
            for (int c = 0; c < plan.tokens && t0 + c < a.rows; c += 32) {
                int32_t v[32];
                tmem_load32(row + c, v);
#pragma unroll
                for (int j = 0; j < 32; j += 4) {
                    asm volatile("st.shared::cluster.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(dest + (uint32_t)(slot * kTileRows + 32 * quarter + lane) * 16), "r"(v[j]),
                                 "r"(v[j + 1]), "r"(v[j + 2]), "r"(v[j + 3])
                                 : "memory");
                    if (++slot == (slice + 1) * (share / 4)) {
                        slot = slice * (share / 4);
                        ++to;
                        dest = in_cta(sums, (uint32_t)min(to, split - 1));
                    }
                }
            }
        }
        cluster_sync();
        if (warp >= 2 && ok) {
            const int4* part = reinterpret_cast<const int4*>(base + plan.sums_at()) + 32 * quarter + lane;
            const int32_t have = min(share, a.rows - t1);
#pragma unroll 1
            for (int c = 0; c < have; c += 32) {
                int32_t v[32];
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = 0;
#pragma unroll 1
                for (int r = 0; r < split; ++r) {
                    const int4* from = part + (r * share + c) / 4 * kTileRows;
#pragma unroll
                    for (int j = 0; j < 32; j += 4) {
                        if (c + j >= have) break;
                        const int4 p = from[j / 4 * kTileRows];
                        v[j] += p.x, v[j + 1] += p.y, v[j + 2] += p.z, v[j + 3] += p.w;
                    }
                }
                store_columns<DT, true>(a, v, t1 + c, have - c, n, ws, bias, reinterpret_cast<const float4*>(s.scales + c));
            }
        }
    }
    __syncwarp();
    mma_fence_before();
    __syncthreads();
    if (warp == 1) {
        mma_fence_after();
        tmem_free<false>(tmem, columns);
    }
}

// ================= two CTAs a tile, persistent =================
// A pair of SMs shares each operand (half of the tokens in either's memory), which halves what comes from L2 for a product; while
// the products of one tile run, the last one's accumulators are read out of the other half of tensor memory.  Bound by the tensor
// cores, and for seconds on end by the board's power: 8192 x 8192 x 14336 577 us at its best (3335 TOP/s), 650 to 677 in a long
// run under the power cap (450 with operands of zeros, which take less power).  2048 x 4096 x 4096 27.0 us (2545 TOP/s): 128 tiles
// over 74 pairs are two turns, the second of them three quarters full.  512 x 4096 x 4096 12.2, 1024 17.3, 4096 49.
constexpr int kPairThreads = 320;  // warp 0 loads, warp 1 issues the products, warps 2 .. 9 read the accumulators
constexpr int kPairReaders = 8;
constexpr int kRaster = 8;         // channel tiles that are walked together, so that what runs at a time shares its operands in L2

constexpr uint32_t kPairColumns = 512;  // of tensor memory: two sets of accumulators

__device__ __forceinline__ void tell_pair(uint32_t* where, uint32_t what) {  // both CTAs
    for (uint32_t r = 0; r < 2; ++r) asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(in_cta(smem_addr(where), r)), "r"(what) : "memory");
}
// Given up, in either CTA: what is in flight ends before the pair leaves its memory.
__device__ __noinline__ void pair_gave_up(TileShared& s, uint32_t rank, uint32_t n, uint32_t stage_bytes) {
    if (threadIdx.x == 0) tell_pair(&s.issued[rank], s.issued[rank]);
    __syncwarp();
    __syncthreads();
    cluster_sync();
    // The first CTA's barriers count the copies of both; a stage that only one of them had come to is counted full by hand.
    if (rank == 0 && threadIdx.x == 0) {
        const uint32_t most = max(s.issued[0], s.issued[1]);
        for (uint32_t u = most - min(most, n); u < most; ++u) {
            uint64_t* bar = &s.full[u % n];
            if (u >= s.issued[0]) mbar_expect(bar, 2 * stage_bytes);
            if (u >= s.issued[0] || u >= s.issued[1]) mbar_count(bar, stage_bytes);
            mbar_drain(bar, (u / n) & 1);
        }
    }
    if (threadIdx.x == 32) {  // (behind all that the products' thread had arrive in either CTA)
        if (rank == 0) mma_commit<true>(&s.drain);
        mbar_drain(&s.drain, 0);
    }
    __syncwarp();
    __syncthreads();
    cluster_sync();
}
template <int DT>
__global__ void __launch_bounds__(kPairThreads)
    k_linear_pair(const LinearArgs a, const __grid_constant__ CUtensorMap wmap, const __grid_constant__ CUtensorMap xmap, int32_t tokens, int32_t n_stages) {
    // a CTA holds its 128 channels and half of the tile's tokens
    const uint32_t stage_bytes = kWeightBytes + (uint32_t)tokens / 2 * kBlockK;
    unsigned char* base = shared_base();
    TileShared& s = *reinterpret_cast<TileShared*>(base);
    const uint32_t stages = smem_addr(base) + kSharedHead;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t rank = cluster_rank();
    const int32_t n_tiles = (a.n + 2 * kTileRows - 1) / (2 * kTileRows), t_tiles = (a.rows + tokens - 1) / tokens;
    const int64_t tiles = (int64_t)n_tiles * t_tiles;
    const int32_t blocks = (a.k + kBlockK - 1) / kBlockK;
    const int64_t first = blockIdx.x >> 1, step = gridDim.x >> 1;
    // tiles in groups of kRaster channel tiles; inside a group channel tiles run fastest
    auto place = [&](int64_t tile, int32_t& n0, int32_t& t0) {
        const int64_t per = (int64_t)kRaster * t_tiles, group = tile / per, in = tile - group * per;
        const int32_t wide = min(kRaster, n_tiles - (int32_t)group * kRaster);
        const int32_t t = (int32_t)(in / wide);
        n0 = ((int32_t)group * kRaster + (int32_t)(in - (int64_t)t * wide)) * 2 * kTileRows;
        t0 = t * tokens;
    };

    if (threadIdx.x == 0) {
        for (int i = 0; i < n_stages; ++i) mbar_init(&s.full[i], 1), mbar_init(&s.empty[i], 1);
        for (int i = 0; i < 2; ++i) mbar_init(&s.done[i], 1), mbar_init(&s.taken[i], 2 * kPairReaders);
        mbar_init(&s.drain, 1);
        s.gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&wmap) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&xmap) : "memory");
    }
    if (warp == 1) {
        __syncwarp();
        tmem_alloc<true>(&s.tmem, kPairColumns);
        mma_fence_before();
    }
    __syncthreads();
    cluster_sync();  // the other CTA's barriers are ready
    mma_fence_after();
    chain_go();  // (not before this CTA has its tensor memory: the next kernel's CTAs would take it and wait for this one's end)
    chain_wait();
    const uint32_t tmem = s.tmem;
    volatile uint32_t* gave_up = &s.gave_up;
    bool lost = false;

    if (warp == 0) {
        if (lane == 0) {
            uint32_t it = 0, st = 0, turn = 1;
            for (int64_t tile = first; tile < tiles && !lost; tile += step) {
                int32_t n0, t0;
                place(tile, n0, t0);
                for (int32_t kb = 0; kb < blocks; ++kb, ++it) {
                    if (!mbar_wait(&s.empty[st], turn, gave_up)) {
                        lost = true;
                        break;
                    }
                    const uint32_t at = stages + st * stage_bytes, bar = in_cta(smem_addr(&s.full[st]), 0);
                    if (rank == 0) mbar_expect(&s.full[st], 2 * stage_bytes);
                    tile_load<true>(at, &wmap, kb * kBlockK, n0 + (int32_t)rank * kTileRows, bar);
                    tile_load<true>(at + kWeightBytes, &xmap, kb * kBlockK, t0 + (int32_t)rank * (tokens / 2), bar);
                    if (++st == (uint32_t)n_stages) st = 0, turn ^= 1;
                }
            }
            // the products that read this CTA's stages are done once their stages are free again
            for (uint32_t u = it - min(it, (uint32_t)n_stages); u < it && !lost; ++u) lost = !mbar_wait(&s.empty[u % n_stages], (u / n_stages) & 1, gave_up);
            s.issued[rank] = it;
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            const uint32_t shape = mma_shape(2 * kTileRows, tokens);
            uint32_t st = 0, turn = 0, local = 0;
            for (int64_t tile = first; tile < tiles && !lost; tile += step, ++local) {
                const uint32_t side = local & 1;
                if (!mbar_wait(&s.taken[side], ((local >> 1) & 1) ^ 1, gave_up)) {
                    lost = true;
                    break;
                }
                mma_fence_after();
                for (int32_t kb = 0; kb < blocks; ++kb) {
                    if (!mbar_wait(&s.full[st], turn, gave_up)) {
                        lost = true;
                        break;
                    }
                    mma_fence_after();
                    const uint32_t at = stages + st * stage_bytes;
                    const uint64_t w = operand(at), x = operand(at + kWeightBytes);
#pragma unroll
                    for (int q = 0; q < kBlockK / 32; ++q) mma<true>(tmem + side * 256, w + 2 * q, x + 2 * q, shape, kb > 0 || q > 0);
                    mma_commit<true>(&s.empty[st]);
                    if (++st == (uint32_t)n_stages) st = 0, turn ^= 1;
                }
                if (!lost) mma_commit<true>(&s.done[side]);
            }
        }
    } else {
        const int quarter = warp & 3, half = (warp - 2) >> 2;  // lanes 32 * quarter .., every other 32 columns
        uint32_t local = 0;
        for (int64_t tile = first; tile < tiles; tile += step, ++local) {
            int32_t n0, t0;
            place(tile, n0, t0);
            const uint32_t side = local & 1;
            const int32_t n = n0 + (int32_t)rank * kTileRows + 32 * quarter + lane;
            const float ws = n < a.n ? a.wscale[n] : 0.0f, bias = a.bias && n < a.n ? a.bias[n] : 0.0f;
            if (lane == 0 && !mbar_wait(&s.done[side], (local >> 1) & 1, gave_up)) lost = true;
            lost = __any_sync(kFullMask, lost);
            if (lost) break;
            mma_fence_after();
            const uint32_t row = tmem + ((uint32_t)(32 * quarter) << 16) + side * 256;
#pragma unroll 1
            for (int c = 32 * half; c < tokens; c += 64) {
                if (t0 + c >= a.rows) break;
                int32_t v[32];
                tmem_load32(row + c, v);
                store_columns<DT>(a, v, t0 + c, a.rows - t0 - c, n, ws, bias);
            }
            mma_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_at(in_cta(smem_addr(&s.taken[side]), 0));
        }
    }
    if (lost) {
        atomicCAS(a.status, 0u, (uint32_t)DNNS_ERR_TIMEOUT);
        tell_pair(&s.gave_up, 1);
    }
    __syncwarp();
    mma_fence_before();
    __syncthreads();
    cluster_sync();  // unless the pair gave up, nothing of it is in flight any more
    if (*gave_up) pair_gave_up(s, rank, (uint32_t)n_stages, stage_bytes);
    mma_fence_after();
    if (warp == 1) tmem_free<true>(tmem, kPairColumns);
}

// ================= host side =================
typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled() {
    static const EncodeTiled fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (!succeeded(cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found)) ||
            found != cudaDriverEntryPointSuccess)
            p = nullptr;
        return reinterpret_cast<EncodeTiled>(p);
    }();
    return fn;
}

// Rows of k bytes, ld apart, fetched in boxes of box_rows rows of 128 bytes; what lies past k or past the rows reads as 0.
bool make_map(CUtensorMap* map, const int8_t* p, int64_t rows, int64_t k, int64_t ld, uint32_t box_rows) {
    const EncodeTiled encode = encode_tiled();
    if (!encode) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)k, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)(rows > 1 ? ld : (k + 15) / 16 * 16)};
    const cuuint32_t box[2] = {kBlockK, box_rows}, steps[2] = {1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<int8_t*>(p), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

constexpr uint32_t kSharedLimit = 227 * 1024;

TilePlan tile_plan(int32_t rows, int tokens, int split) {
    TilePlan plan{tokens, (rows + tokens - 1) / tokens, split, kMaxStages};
    // Small tiles leave room for two CTAs an SM, whether or not the grid has two: where it has not, they go without half of their stages (64
    // x 4096 x 4096 in four 7.6 us; a tile of 96 tokens, with all of them, took 6.8).
    const uint32_t room = tokens <= 64 ? kSharedLimit / 2 - 1024 : kSharedLimit;
    while (plan.stages > 2 && plan.shared_bytes() > room) --plan.stages;
    return plan;
}

template <int DT>
bool launch_tile(const LinearArgs& a, int tokens, int split, int dev, cudaStream_t st) {
    static std::atomic<uint64_t> done{0};
    if (!allow_shared(k_linear_tile<DT>, kSharedLimit, done, dev)) return false;
    CUtensorMap wmap, xmap;
    if (!make_map(&wmap, a.wq, a.n, a.k, a.ldw, kTileRows) || !make_map(&xmap, a.xq, a.rows, a.k, a.ldx, (uint32_t)tokens)) return false;
    const TilePlan plan = tile_plan(a.rows, tokens, split);
    const int32_t n_tiles = (a.n + kTileRows - 1) / kTileRows;
    return launch_chained(k_linear_tile<DT>, (unsigned)((int64_t)plan.t_tiles * n_tiles * split), kTileThreads2, plan.shared_bytes(), st, (unsigned)split, a, wmap,
                          xmap, plan);
}

template <int DT>
bool launch_pair(const LinearArgs& a, int tokens, int n_sm, int dev, cudaStream_t st) {
    static std::atomic<uint64_t> done{0};
    if (!allow_shared(k_linear_pair<DT>, kSharedLimit, done, dev)) return false;
    CUtensorMap wmap, xmap;
    if (!make_map(&wmap, a.wq, a.n, a.k, a.ldw, kTileRows) || !make_map(&xmap, a.xq, a.rows, a.k, a.ldx, (uint32_t)tokens / 2)) return false;
    const int64_t tiles = (int64_t)((a.rows + tokens - 1) / tokens) * ((a.n + 2 * kTileRows - 1) / (2 * kTileRows));
    const unsigned grid = 2 * (unsigned)std::min<int64_t>(tiles, n_sm / 2);
    const uint32_t stage = kWeightBytes + (uint32_t)tokens / 2 * kBlockK;
    const int stages = std::min<int>(kMaxStages, (int)((kSharedLimit - kSharedHead - 1024) / stage));
    return launch_chained(k_linear_pair<DT>, grid, kPairThreads, kSharedHead + stages * stage + 1024, st, 2, a, wmap, xmap, (int32_t)tokens, (int32_t)stages);
}

template <int DT>
bool launch_rows(const LinearArgs& a, int n_sm, cudaStream_t st) {
    // two channels a warp where that still leaves a dozen warps an SM (each then has more loads on their way); warps share a
    // channel, down to four loads a lane of each, until there are enough blocks for the SMs to finish together
    const bool two = a.n >= 24 * n_sm;
    int parts = 1;
    while (parts < kRowsWarps && (int64_t)a.n * parts < 6 * (two ? 2 : 1) * kRowsWarps * (int64_t)n_sm && a.k >= 4 * 512 * 2 * parts) parts *= 2;
    const int64_t step = kRowsWarps / parts * (two ? 2 : 1);
    return launch_chained(two ? k_linear_rows<1, 2, DT> : k_linear_rows<1, 1, DT>, (unsigned)((a.n + step - 1) / step), 32 * kRowsWarps, 0, st, 1, a, parts);
}

template <int DT>
bool launch_empty(const LinearArgs& a, cudaStream_t st) {
    return launch_chained(k_linear_empty<DT>, dim3((unsigned)(((int64_t)a.n + 255) / 256), (unsigned)std::min(a.rows, 65535)), 256, 0, st, 1, a);
}

// Warps that share the columns of 16 channels: as long as the 16 warps an SM that fit at a time are not passed (17 x 3000 x 5000 in
// two turns of blocks 11.9 us, in one 8.6), down to four loads a lane.
int few_parts(int64_t n, int64_t k, int n_sm) {
    int parts = 1;
    while (parts < kRowsWarps && (n + 15) / 16 * parts * 2 <= 16 * (int64_t)n_sm && k >= 4 * 64 * 2 * parts) parts *= 2;
    return parts;
}

template <int DT>
bool launch_few(const LinearArgs& a, int n_sm, cudaStream_t st) {
    const int64_t groups = ((int64_t)a.n + 15) / 16;
    const int parts = few_parts(a.n, a.k, n_sm);
    const unsigned grid = (unsigned)((groups * parts + kRowsWarps - 1) / kRowsWarps);
    const int blocks = (a.rows + 7) / 8;
    const auto kernel = blocks == 1 ? k_linear_few<1, DT> : blocks == 2 ? k_linear_few<2, DT> : blocks == 3 ? k_linear_few<3, DT> : k_linear_few<4, DT>;
    return launch_chained(kernel, grid, 32 * kRowsWarps, 0, st, 1, a, parts);
}

// Which kernel: `tokens` of a tile (0: k_linear_rows, 8: k_linear_few), over one CTA or a pair, columns split so many ways.
struct Choice {
    int tokens, pair, split;
};

// The cheapest by a model of the kernels' time in clocks at 1.9 GHz, fitted to sweeps of every tile and split over 37 shapes of 1 ..
// 8192 tokens and 250 .. 14336 columns and channels (what it takes is within 1.15 of the best of each but for four, 1.2 to 1.45).  What it
// says, with both sides measured (us):
//   - a tile kernel's stage costs what its bytes take from L2, about 60 B a clock into one SM (k_linear_tile, up to 148 of them) or 44
//     (k_linear_pair, all SMs at once); rows that do not start on 128 bytes cost more: 333 x 5003 x 2741 (tokens, columns, channels) at a row
//     distance of 5008 14.2, of 5120 11.3.  Hence large tiles for many tokens (2048 x 4096 x 4096: a pair with 256 tokens 27.0, with
//     128 39.8), and hence splits, which put every SM to work where there are few tiles (64 x 4096 x 4096: one CTA a tile 9.9,
//     its columns over four 7.6).  With few stages a stage costs its way from L2 to the product and back instead.
//   - k_linear_few pays for each 8 tokens in warp-wide products: 16 x 4096 x 4096 5.9 against 7.4 in tiles, 24 x 4096 x 14336 19.9
//     against 13.4; and for loads one after the other where the columns are not whole batches: 5 x 700 x 3000 4.4 against 3.7.
Choice choose(const LinearArgs& a, int n_sm) {
    if (a.rows <= 1) return {0, 0, 1};
    const double bytes = (double)a.n * a.k, memory = bytes / 3400.0;  // 6.5 TB/s
    const double blocks = (a.k + kBlockK - 1) / kBlockK, rough_w = a.ldw % 128 ? 1.2 : 1.0, rough_x = a.ldx % 128 ? 1.2 : 1.0;
    Choice best{8, 0, 1};
    double least = 1e300;
    if (a.rows <= 32) {
        // a warp's loads one after the other: four pieces at a time, then one by one, then the ragged one
        const int pieces = a.k / 64 / few_parts(a.n, a.k, n_sm), turns = pieces / 4 + pieces % 4 + (a.k % 64 ? 2 : 0);
        least = 3300.0 + std::max(bytes * 1e-6 * 1900.0 * (0.15 + 0.052 * ((a.rows + 7) / 8)), turns * 2300.0);
    }
    const int64_t channels = (a.n + kTileRows - 1) / kTileRows, pairs = (a.n + 2 * kTileRows - 1) / (2 * kTileRows);
    const int most = std::min(256, (a.rows + 31) / 32 * 32);
    for (int tokens = 32; tokens <= most; tokens += 32) {
        const int64_t t_tiles = (a.rows + tokens - 1) / tokens, tiles = channels * t_tiles;
        const double stage = std::max(std::max((rough_w * 16384.0 + rough_x * 128.0 * tokens) / 60.0, 2.0 * tokens), 430.0);
        static const int splits[] = {1, 2, 3, 4, 6, 8};
        for (int split : splits) {
            const int64_t turns = (tiles * split + n_sm - 1) / n_sm;
            if (tokens % (4 * split)) continue;
            if (split > 1 && (tiles * split > (tokens <= 64 ? 2 : 1) * (int64_t)n_sm || blocks < 2 * split)) break;
            const double late = 2600.0 / tile_plan(a.rows, tokens, split).stages;  // a stage's way from L2 to the product and back
            const double cost = 4000.0 + std::max(memory, turns * (std::ceil(blocks / split) * std::max(stage, late))) + 30.0 * turns * tokens / split +
                                (split > 1 ? 2500.0 + 10.0 * tokens + 350.0 * split : 0.0);
            if (cost < least) least = cost, best = {tokens, 0, split};
            if (tiles >= n_sm) break;
        }
        if (tokens < 64) continue;
        const int64_t turns = (pairs * t_tiles + n_sm / 2 - 1) / (n_sm / 2);
        const double pair_stage = std::max((rough_w * 16384.0 + rough_x * 64.0 * tokens) / 44.0, 2.0 * tokens);
        const double cost = 6500.0 + std::max(memory, turns * blocks * pair_stage) + 15.0 * tokens;
        if (cost < least) least = cost, best = {tokens, 1, 1};
    }
    return best;
}

template <int DT>
bool launch_linear(const LinearArgs& a, const Choice& c, int n_sm, int dev, cudaStream_t st) {
    if (c.tokens == 0) return launch_rows<DT>(a, n_sm, st);
    if (c.tokens == 8) return launch_few<DT>(a, n_sm, st);
    return c.pair ? launch_pair<DT>(a, c.tokens, n_sm, dev, st) : launch_tile<DT>(a, c.tokens, c.split, dev, st);
}

}  // namespace

}  // namespace dnns

extern "C" dnns_status dnns_linear_quantized(const int8_t* xq, int64_t ldx, const float* xscale, const int8_t* wq, int64_t ldw,
                                             const float* wscale, const float* bias, int64_t rows, int64_t in_cols, int64_t out_cols,
                                             int32_t dtype, void* y, int64_t ldy, uint32_t* status_dev, void* stream) {
    using namespace dnns;
    auto address = [](const void* p) { return reinterpret_cast<uintptr_t>(p); };
    if (rows < 0 || in_cols < 0 || out_cols < 0) return DNNS_ERR_INVALID_ARG;
    if (dtype != DNNS_F32 && dtype != DNNS_BF16) return DNNS_ERR_UNSUPPORTED;
    const int64_t limit = ((int64_t)1 << 30) + 1, span = (int64_t)1 << 60;
    if (rows >= limit || out_cols >= limit || in_cols > DNNS_LINEAR_MAX_IN) return DNNS_ERR_UNSUPPORTED;
    if (!status_dev || address(status_dev) % 4) return DNNS_ERR_INVALID_ARG;
    if (rows == 0 || out_cols == 0) return DNNS_OK;
    if (in_cols && (!xq || !wq || address(xq) % 16 || address(wq) % 16 || ldx % 16 || ldw % 16 || ldx < in_cols || ldw < in_cols))
        return DNNS_ERR_INVALID_ARG;
    if (!xscale || !wscale || address(xscale) % 4 || address(wscale) % 4 || address(bias) % 4) return DNNS_ERR_INVALID_ARG;
    if (!y || address(y) % (dtype == DNNS_F32 ? 4 : 2) || ldy < out_cols) return DNNS_ERR_INVALID_ARG;
    if (ldy > span / rows || (in_cols && (ldx > span / rows || ldw > span / out_cols))) return DNNS_ERR_UNSUPPORTED;
    const LinearArgs a{xq, wq, xscale, wscale, bias, y, status_dev, ldx, ldw, ldy, (int32_t)rows, (int32_t)in_cols, (int32_t)out_cols};
    int dev = 0, n_sm = 0;
    if (!succeeded(cudaGetDevice(&dev)) || !succeeded(cudaDeviceGetAttribute(&n_sm, cudaDevAttrMultiProcessorCount, dev))) return DNNS_ERR_CUDA;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (in_cols == 0) return (dtype == DNNS_F32 ? launch_empty<DNNS_F32>(a, st) : launch_empty<DNNS_BF16>(a, st)) ? DNNS_OK : DNNS_ERR_CUDA;
    const Choice c = choose(a, n_sm);
    const bool launched = dtype == DNNS_F32 ? launch_linear<DNNS_F32>(a, c, n_sm, dev, st) : launch_linear<DNNS_BF16>(a, c, n_sm, dev, st);
    return launched ? DNNS_OK : DNNS_ERR_CUDA;
}

#ifdef DNNS_BOUNDS_CHECK
// Checked build only: waits of the product's kernels are given up at once (on the current device) while `on` is not 0.
extern "C" dnns_status dnns_check_hurry(unsigned int on) {
    return cudaDeviceSynchronize() == cudaSuccess && cudaMemcpyToSymbol(dnns::g_hurry, &on, sizeof(on)) == cudaSuccess ? DNNS_OK : DNNS_ERR_CUDA;
}
#endif
