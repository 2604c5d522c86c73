// Product of rows in 8 bits:  y[t][n] = (sum_k xq[t][k] * wq[n][k]) * xscale[t] * wscale[n] + bias[n].
// The sum is exact in int32 (at most 2^17 - 1 products of at most 2^14 each), so any order and any split of it gives
// the same bits.
//
// Three kernels, chosen by the number of tokens and the work there is for the SMs (choose() below):
//   k_linear_rows   few tokens: bound by reading the weights once; int8 dot products in the ordinary pipes
//   k_linear_tile   one CTA a tile of 128 channels x BT tokens; the columns of a tile may be split over the CTAs of a cluster,
//                   whose int32 partial sums meet in distributed shared memory
//   k_linear_pair   two CTAs a tile of 256 channels x BT tokens, persistent, accumulators double-buffered in tensor memory
// The tile kernels put the WEIGHTS on the rows of the tensor cores' tile (the lanes of tensor memory) and the tokens on its
// columns: a tile is then never wider in tokens than there are tokens to a multiple of 32, and a warp that reads one
// accumulator column holds 32 neighbouring channels of one token, which it stores as one contiguous piece of y - no
// staging in shared memory, no alignment asked of y or ldy.
#include <cuda.h>

#include <algorithm>

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

__device__ __forceinline__ int4 stream16(const int8_t* p) {
    int4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ int32_t dot16(const int4& a, const int4& b, int32_t c) { return __dp4a(a.x, b.x, __dp4a(a.y, b.y, __dp4a(a.z, b.z, __dp4a(a.w, b.w, c)))); }

// M tokens at most (a.rows of them), blockIdx.y the token group.
template <int M, int R, int DT>
__global__ void __launch_bounds__(32 * kRowsWarps) k_linear_rows(const LinearArgs a, int32_t parts) {
    chain_go();
    chain_wait();
    constexpr int U = M <= 4 ? 4 : 2;  // loads deep
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
                const int4 xv = __ldg(reinterpret_cast<const int4*>(x[t] + 16 * (v + u * step)));
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
            const int4 xv = __ldg(reinterpret_cast<const int4*>(x[t] + 16 * v));
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
    uint32_t w[4] = {0, 0, 0, 0};
    for (int i = 0; c + i < k; ++i) w[i >> 2] |= (uint32_t)(uint8_t)row[c + i] << (8 * (i & 3));
    return make_int4((int)w[0], (int)w[1], (int)w[2], (int)w[3]);
}

// 8 * TB tokens at most (a.rows of them)
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
            for (int t = 0; t < TB; ++t) lane_product(acc[t], wl[u], wh[u], __ldg(reinterpret_cast<const int4*>(x[t] + 64 * (b + u * step) + 16 * q)));
    }
    for (; b < whole; b += step) {
        const int4 wl = stream16(lo + 64 * b + 16 * q), wh = stream16(hi + 64 * b + 16 * q);
#pragma unroll
        for (int t = 0; t < TB; ++t) lane_product(acc[t], wl, wh, __ldg(reinterpret_cast<const int4*>(x[t] + 64 * b + 16 * q)));
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
// Wait for a phase of an mbarrier, but not for ever: false when the wait was given up, or another thread of the CTA gave
// up before.  (The timer takes long to read: it is looked at only after many tries.)
__device__ __forceinline__ bool mbar_wait(uint64_t* bar, uint32_t parity, volatile uint32_t* gave_up) {
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

// 32 columns (tokens t0 ..) of one channel a lane: scale and store.
template <int DT>
__device__ __forceinline__ void store_columns(const LinearArgs& a, const int32_t (&v)[32], int32_t t0, int32_t n, float ws, float bias) {
    typedef typename std::conditional<DT == DNNS_F32, float, uint16_t>::type T;
    const int lane = threadIdx.x & 31;
    const float mine = t0 + lane < a.rows ? a.xscale[t0 + lane] : 0.0f;
    T* y = static_cast<T*>(a.y) + (int64_t)t0 * a.ldy + n;
    const int32_t left = a.rows - t0;
    const bool in = n < a.n;
#pragma unroll
    for (int j = 0; j < 32; ++j) {
        const float xs = __shfl_sync(kFullMask, mine, j);
        if (in && j < left) store_out<DT>(y, 0, scaled(v[j], xs, ws, bias));
        y += a.ldy;
    }
}

struct TileShared {  // in front of the stages
    uint64_t full[10], empty[10], done[2], taken[2], drain;
    uint32_t tmem, gave_up;
};
constexpr uint32_t kSharedHead = 1024;
static_assert(sizeof(TileShared) <= kSharedHead, "head of the shared memory");

__device__ __forceinline__ unsigned char* shared_base() {
    extern __shared__ unsigned char raw[];
    return raw + ((1024u - (smem_addr(raw) & 1023u)) & 1023u);  // (the swizzle repeats every 1024 bytes)
}

// ================= one CTA a tile, its columns split over a cluster =================
constexpr int kTileThreads2 = 192;  // warp 0 loads, warp 1 issues the products, warps 2 .. 5 read the accumulators

template <int BT>
struct TileCfg {
    static constexpr uint32_t kStage = kWeightBytes + BT * kBlockK;
    #ifndef ST32
#define ST32 5
#endif
    static constexpr int kStages = BT <= 32 ? ST32 : BT <= 64 ? 4 : 6;
    static constexpr uint32_t kShared = kSharedHead + kStages * kStage + 1024;
    static constexpr uint32_t kColumns = BT;
    static_assert(kStages <= 10 && kStages * kStage >= BT * kTileRows * 4, "the partial sums of a cluster reuse the stages");
};

template <int BT, int DT>
__global__ void __launch_bounds__(kTileThreads2) k_linear_tile(const LinearArgs a, const __grid_constant__ CUtensorMap wmap,
                                                               const __grid_constant__ CUtensorMap xmap, int32_t t_tiles, int32_t split) {
    typedef TileCfg<BT> Cfg;
    unsigned char* base = shared_base();
    TileShared& s = *reinterpret_cast<TileShared*>(base);
    const uint32_t stages = smem_addr(base) + kSharedHead;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int32_t tile = blockIdx.x / split, slice = blockIdx.x - tile * split;
    const int32_t t0 = (tile % t_tiles) * BT, n0 = (tile / t_tiles) * kTileRows;
    const int32_t blocks = (a.k + kBlockK - 1) / kBlockK;
    const int32_t kb0 = (int32_t)((int64_t)blocks * slice / split), kbs = (int32_t)((int64_t)blocks * (slice + 1) / split) - kb0;

    if (threadIdx.x == 0) {
        for (int i = 0; i < Cfg::kStages; ++i) mbar_init(&s.full[i], 1), mbar_init(&s.empty[i], 1);
        mbar_init(&s.done[0], 1);
        mbar_init(&s.drain, 1);
        s.gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&wmap) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&xmap) : "memory");
    }
    if (warp == 1) {
        __syncwarp();
        tmem_alloc<false>(&s.tmem, Cfg::kColumns);
        mma_fence_before();
    }
    __syncthreads();
    mma_fence_after();
    chain_go();  // (not before this CTA has its tensor memory: the next kernel's CTAs would take it and wait for this one's end)
    chain_wait();
    const uint32_t tmem = s.tmem;
    volatile uint32_t* gave_up = &s.gave_up;

    if (warp == 0) {
        if (lane == 0) {
            int32_t it = 0;
            for (; it < kbs; ++it) {
                const int st = it % Cfg::kStages;
                if (!mbar_wait(&s.empty[st], ((it / Cfg::kStages) & 1) ^ 1, gave_up)) break;
                const uint32_t at = stages + st * Cfg::kStage, bar = smem_addr(&s.full[st]);
                mbar_expect(&s.full[st], Cfg::kStage);
                tile_load<false>(at, &wmap, (kb0 + it) * kBlockK, n0, bar);
                tile_load<false>(at + kWeightBytes, &xmap, (kb0 + it) * kBlockK, t0, bar);
            }
            // a wait that was given up: copies in flight are waited for (again with a limit) before the memory is left
            if (it < kbs) {
                atomicCAS(a.status, 0u, (uint32_t)DNNS_ERR_TIMEOUT);
                const uint64_t since = global_ns();
                for (int32_t u = max(0, it - Cfg::kStages); u < it; ++u)
                    while (!mbar_try(&s.full[u % Cfg::kStages], (u / Cfg::kStages) & 1) && global_ns() - since < kWaitLimitNs) {
                    }
            }
        }
    } else if (warp == 1) {
        if (lane == 0) {
            int32_t it = 0;
            for (; it < kbs; ++it) {
                const int st = it % Cfg::kStages;
                if (!mbar_wait(&s.full[st], (it / Cfg::kStages) & 1, gave_up)) break;
                mma_fence_after();
                const uint32_t at = stages + st * Cfg::kStage;
                const uint64_t w = operand(at), x = operand(at + kWeightBytes);
#pragma unroll
                for (int q = 0; q < kBlockK / 32; ++q) mma<false>(tmem, w + 2 * q, x + 2 * q, mma_shape(kTileRows, BT), it > 0 || q > 0);
                mma_commit<false>(&s.empty[st]);
            }
            if (it == kbs) {
                mma_commit<false>(&s.done[0]);
            } else {
                atomicCAS(a.status, 0u, (uint32_t)DNNS_ERR_TIMEOUT);
                mma_commit<false>(&s.drain);
                const uint64_t since = global_ns();
                while (!mbar_try(&s.drain, 0) && global_ns() - since < kWaitLimitNs) {
                }
            }
        }
    }
    // everybody waits for the sums: after this no copy and no product of this CTA is in flight
    __syncwarp();
    const bool ok = __shfl_sync(kFullMask, (int)(lane == 0 && mbar_wait(&s.done[0], 0, gave_up)), 0);
    mma_fence_after();
    const int quarter = warp & 3;  // tensor memory lanes a warp may read: 32 * (its index mod 4) ..
    const int32_t n = n0 + 32 * quarter + lane;
    const float ws = warp >= 2 && n < a.n ? a.wscale[n] : 0.0f, bias = warp >= 2 && a.bias && n < a.n ? a.bias[n] : 0.0f;
    const uint32_t row = tmem + ((uint32_t)(32 * quarter) << 16);
    if (!ok && threadIdx.x == 64) atomicCAS(a.status, 0u, (uint32_t)DNNS_ERR_TIMEOUT);
    __syncwarp();
    if (split == 1) {
        if (warp >= 2 && ok) {
#pragma unroll 1
            for (int c = 0; c < BT; c += 32) {
                if (t0 + c >= a.rows) break;
                int32_t v[32];
                tmem_load32(row + c, v);
                store_columns<DT>(a, v, t0 + c, n, ws, bias);
            }
        }
    } else {
        // the cluster's CTAs share the columns out: CTA r gets everybody's sums of columns r * share .., four columns of a channel
        // in 16 bytes
        const int share = BT / split, by = __ffs(share) - 1;  // (powers of two, share at least 4)
        cluster_sync();  // every CTA is done with its stages
        if (warp >= 2) {
#pragma unroll 1
            for (int c = 0; c < BT && t0 + c < a.rows; c += 32) {
                int32_t v[32];
                tmem_load32(row + c, v);
#pragma unroll
                for (int j = 0; j < 32; j += 4) {
                    const int to = (c + j) >> by, slot = (slice * share + (c + j) - to * share) / 4;
                    const uint32_t at = in_cta(stages + (uint32_t)(slot * kTileRows + 32 * quarter + lane) * 16, (uint32_t)to);
                    asm volatile("st.shared::cluster.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v[j]), "r"(v[j + 1]), "r"(v[j + 2]), "r"(v[j + 3]) : "memory");
                }
            }
        }
        const int32_t t1 = t0 + slice * share;
        const float xs = lane < share && t1 + lane < a.rows ? a.xscale[t1 + lane] : 0.0f;
        const float xs2 = share > 32 && t1 + 32 + lane < a.rows ? a.xscale[t1 + 32 + lane] : 0.0f;
        cluster_sync();
        if (warp >= 2 && ok) {
            const int4* part = reinterpret_cast<const int4*>(base + kSharedHead) + 32 * quarter + lane;
            for (int c = 0; c < share && t1 + c < a.rows; c += 4) {
                int32_t sum[4] = {0, 0, 0, 0};
#pragma unroll 4
                for (int r = 0; r < split; ++r) {
                    const int4 p = part[(r * share + c) / 4 * kTileRows];
                    sum[0] += p.x, sum[1] += p.y, sum[2] += p.z, sum[3] += p.w;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float scale = __shfl_sync(kFullMask, c + i < 32 ? xs : xs2, (c + i) & 31);
                    if (t1 + c + i < a.rows && n < a.n) store_out<DT>(a.y, (int64_t)(t1 + c + i) * a.ldy + n, scaled(sum[i], scale, ws, bias));
                }
            }
        }
    }
    __syncwarp();
    mma_fence_before();
    __syncthreads();
    if (warp == 1) {
        mma_fence_after();
        tmem_free<false>(tmem, Cfg::kColumns);
    }
}

// ================= two CTAs a tile, persistent =================
constexpr int kPairThreads = 320;  // warp 0 loads, warp 1 issues the products, warps 2 .. 9 read the accumulators
constexpr int kPairReaders = 8;
constexpr int kRaster = 8;         // channel tiles that are walked together, so that what runs at a time shares its operands in L2

template <int BT>
struct PairCfg {
    static constexpr uint32_t kTokenBytes = BT / 2 * kBlockK;  // a CTA holds half of the tile's tokens
    static constexpr uint32_t kStage = kWeightBytes + kTokenBytes;
    static constexpr int kStages = BT == 256 ? 6 : 8;
    static constexpr uint32_t kShared = kSharedHead + kStages * kStage + 1024;
    static constexpr uint32_t kColumns = 2 * BT;
};

template <int BT, int DT>
__global__ void __launch_bounds__(kPairThreads)
    k_linear_pair(const LinearArgs a, const __grid_constant__ CUtensorMap wmap, const __grid_constant__ CUtensorMap xmap) {
    typedef PairCfg<BT> Cfg;
    unsigned char* base = shared_base();
    TileShared& s = *reinterpret_cast<TileShared*>(base);
    const uint32_t stages = smem_addr(base) + kSharedHead;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t rank = cluster_rank();
    const int32_t n_tiles = (a.n + 2 * kTileRows - 1) / (2 * kTileRows), t_tiles = (a.rows + BT - 1) / BT;
    const int64_t tiles = (int64_t)n_tiles * t_tiles;
    const int32_t blocks = (a.k + kBlockK - 1) / kBlockK;
    const int64_t first = blockIdx.x >> 1, step = gridDim.x >> 1;
    // tiles in groups of kRaster channel tiles; inside a group channel tiles run fastest
    auto place = [&](int64_t tile, int32_t& n0, int32_t& t0) {
        const int64_t per = (int64_t)kRaster * t_tiles, group = tile / per, in = tile - group * per;
        const int32_t wide = min(kRaster, n_tiles - (int32_t)group * kRaster);
        const int32_t t = (int32_t)(in / wide);
        n0 = ((int32_t)group * kRaster + (int32_t)(in - (int64_t)t * wide)) * 2 * kTileRows;
        t0 = t * BT;
    };

    if (threadIdx.x == 0) {
        for (int i = 0; i < Cfg::kStages; ++i) mbar_init(&s.full[i], 1), mbar_init(&s.empty[i], 1);
        for (int i = 0; i < 2; ++i) mbar_init(&s.done[i], 1), mbar_init(&s.taken[i], 2 * kPairReaders);
        mbar_init(&s.drain, 1);
        s.gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&wmap) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&xmap) : "memory");
    }
    if (warp == 1) {
        __syncwarp();
        tmem_alloc<true>(&s.tmem, Cfg::kColumns);
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
            uint32_t it = 0;
            for (int64_t tile = first; tile < tiles && !lost; tile += step) {
                int32_t n0, t0;
                place(tile, n0, t0);
                for (int32_t kb = 0; kb < blocks; ++kb, ++it) {
                    const uint32_t st = it % Cfg::kStages;
                    if (!mbar_wait(&s.empty[st], ((it / Cfg::kStages) & 1) ^ 1, gave_up)) {
                        lost = true;
                        break;
                    }
                    const uint32_t at = stages + st * Cfg::kStage, bar = in_cta(smem_addr(&s.full[st]), 0);
                    if (rank == 0) mbar_expect(&s.full[st], 2 * Cfg::kStage);
                    tile_load<true>(at, &wmap, kb * kBlockK, n0 + (int32_t)rank * kTileRows, bar);
                    tile_load<true>(at + kWeightBytes, &xmap, kb * kBlockK, t0 + (int32_t)rank * (BT / 2), bar);
                }
            }
            // the products that read this CTA's stages are done once their stages are free again; after a wait that was
            // given up, copies in flight are waited for (again with a limit)
            const uint32_t n = min(it, (uint32_t)Cfg::kStages);
            if (!lost) {
                for (uint32_t u = it - n; u < it && !lost; ++u) lost = !mbar_wait(&s.empty[u % Cfg::kStages], (u / Cfg::kStages) & 1, gave_up);
            } else if (rank == 0) {
                const uint64_t since = global_ns();
                for (uint32_t u = it - n; u < it; ++u)
                    while (!mbar_try(&s.full[u % Cfg::kStages], (u / Cfg::kStages) & 1) && global_ns() - since < kWaitLimitNs) {
                    }
            }
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            uint32_t it = 0, local = 0;
            for (int64_t tile = first; tile < tiles && !lost; tile += step, ++local) {
                const uint32_t side = local & 1;
                if (!mbar_wait(&s.taken[side], ((local >> 1) & 1) ^ 1, gave_up)) {
                    lost = true;
                    break;
                }
                mma_fence_after();
                for (int32_t kb = 0; kb < blocks; ++kb, ++it) {
                    const uint32_t st = it % Cfg::kStages;
                    if (!mbar_wait(&s.full[st], (it / Cfg::kStages) & 1, gave_up)) {
                        lost = true;
                        break;
                    }
                    mma_fence_after();
                    const uint32_t at = stages + st * Cfg::kStage;
                    const uint64_t w = operand(at), x = operand(at + kWeightBytes);
#pragma unroll
                    for (int q = 0; q < kBlockK / 32; ++q) mma<true>(tmem + side * BT, w + 2 * q, x + 2 * q, mma_shape(2 * kTileRows, BT), kb > 0 || q > 0);
                    mma_commit<true>(&s.empty[st]);
                }
                if (!lost) mma_commit<true>(&s.done[side]);
            }
            if (lost) {
                mma_commit<true>(&s.drain);
                const uint64_t since = global_ns();
                while (!mbar_try(&s.drain, 0) && global_ns() - since < kWaitLimitNs) {
                }
            }
        }
    } else {
        const int quarter = warp & 3, half = (warp - 2) >> 2;  // lanes 32 * quarter .., columns half * BT / 2 ..
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
            const uint32_t row = tmem + ((uint32_t)(32 * quarter) << 16) + side * BT;
#pragma unroll 1
            for (int c = half * (BT / 2); c < (half + 1) * (BT / 2); c += 32) {
                if (t0 + c >= a.rows) break;
                int32_t v[32];
                tmem_load32(row + c, v);
                store_columns<DT>(a, v, t0 + c, n, ws, bias);
            }
            mma_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_at(in_cta(smem_addr(&s.taken[side]), 0));
        }
    }
    if (lost) atomicCAS(a.status, 0u, (uint32_t)DNNS_ERR_TIMEOUT);
    __syncwarp();
    mma_fence_before();
    __syncthreads();
    cluster_sync();  // nothing of the pair is in flight any more
    mma_fence_after();
    if (warp == 1) tmem_free<true>(tmem, Cfg::kColumns);
}

// ================= host side =================
typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled() {
    static const EncodeTiled fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
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

template <int BT, int DT>
bool launch_tile(const LinearArgs& a, int split, int dev, cudaStream_t st) {
    static std::atomic<uint64_t> done{0};
    typedef TileCfg<BT> Cfg;
    if (!allow_shared(k_linear_tile<BT, DT>, Cfg::kShared, done, dev)) return false;
    CUtensorMap wmap, xmap;
    if (!make_map(&wmap, a.wq, a.n, a.k, a.ldw, kTileRows) || !make_map(&xmap, a.xq, a.rows, a.k, a.ldx, BT)) return false;
    const int32_t t_tiles = (a.rows + BT - 1) / BT, n_tiles = (a.n + kTileRows - 1) / kTileRows;
    return launch_chained(k_linear_tile<BT, DT>, (unsigned)((int64_t)t_tiles * n_tiles * split), kTileThreads2, Cfg::kShared, st, (unsigned)split, a, wmap, xmap, t_tiles,
                          (int32_t)split);
}

template <int BT, int DT>
bool launch_pair(const LinearArgs& a, int n_sm, int dev, cudaStream_t st) {
    static std::atomic<uint64_t> done{0};
    typedef PairCfg<BT> Cfg;
    if (!allow_shared(k_linear_pair<BT, DT>, Cfg::kShared, done, dev)) return false;
    CUtensorMap wmap, xmap;
    if (!make_map(&wmap, a.wq, a.n, a.k, a.ldw, kTileRows) || !make_map(&xmap, a.xq, a.rows, a.k, a.ldx, BT / 2)) return false;
    const int64_t tiles = (int64_t)((a.rows + BT - 1) / BT) * ((a.n + 2 * kTileRows - 1) / (2 * kTileRows));
    const unsigned grid = 2 * (unsigned)std::min<int64_t>(tiles, n_sm / 2);
    return launch_chained(k_linear_pair<BT, DT>, grid, kPairThreads, Cfg::kShared, st, 2, a, wmap, xmap);
}

template <int M, int DT>
bool launch_rows_of(const LinearArgs& a, int n_sm, cudaStream_t st) {
    // two channels a warp where that still leaves a dozen warps an SM (each then has more loads on their way); warps share a
    // channel, down to four loads a lane of each, until there are enough blocks for the SMs to finish together
    const bool two = a.n >= 24 * n_sm;
    int parts = 1;
    while (parts < kRowsWarps && (int64_t)a.n * parts < 6 * (two ? 2 : 1) * kRowsWarps * (int64_t)n_sm && a.k >= 4 * 512 * 2 * parts) parts *= 2;
    const int64_t step = kRowsWarps / parts * (two ? 2 : 1), most = 65535 * (int64_t)M;  // (the grid's second extent)
    for (int64_t t0 = 0; t0 < a.rows; t0 += most) {
        LinearArgs part = a;
        part.rows = (int32_t)std::min<int64_t>(a.rows - t0, most);
        part.xq += t0 * a.ldx, part.xscale += t0;
        part.y = static_cast<char*>(a.y) + t0 * a.ldy * (DT == DNNS_F32 ? 4 : 2);
        const dim3 grid((unsigned)((a.n + step - 1) / step), (unsigned)((part.rows + M - 1) / M));
        if (!launch_chained(two ? k_linear_rows<M, 2, DT> : k_linear_rows<M, 1, DT>, grid, 32 * kRowsWarps, 0, st, 1, part, parts)) return false;
    }
    return true;
}

template <int DT>
bool launch_rows(const LinearArgs& a, int n_sm, cudaStream_t st) {
    if (a.rows <= 1) return launch_rows_of<1, DT>(a, n_sm, st);
    return a.rows <= 2 ? launch_rows_of<2, DT>(a, n_sm, st) : launch_rows_of<4, DT>(a, n_sm, st);
}

template <int DT>
bool launch_few(const LinearArgs& a, int n_sm, cudaStream_t st) {
    const int64_t groups = ((int64_t)a.n + 15) / 16;
    int parts = 1;
    while (parts < kRowsWarps && groups * parts < 16 * (int64_t)n_sm && a.k >= 4 * 64 * 2 * parts) parts *= 2;
    const unsigned grid = (unsigned)((groups * parts + kRowsWarps - 1) / kRowsWarps);
    const int blocks = (a.rows + 7) / 8;
    const auto kernel = blocks == 1 ? k_linear_few<1, DT> : blocks == 2 ? k_linear_few<2, DT> : blocks == 3 ? k_linear_few<3, DT> : k_linear_few<4, DT>;
    return launch_chained(kernel, grid, 32 * kRowsWarps, 0, st, 1, a, parts);
}

// Which kernel: `tokens` of a tile (0: k_linear_rows), over one CTA or a pair, columns split so many ways.
struct Choice {
    int tokens, pair, split;
};

Choice choose(const LinearArgs& a, int n_sm) {
    if (a.k == 0 || a.rows <= 1) return {0, 0, 1};
    if (a.rows <= 32) return {8, 0, 1};
    const int64_t channels = (a.n + kTileRows - 1) / kTileRows, blocks = (a.k + kBlockK - 1) / kBlockK;
    auto tiles = [&](int bt) { return channels * ((a.rows + bt - 1) / bt); };
    if (a.rows > 128 && tiles(256) >= n_sm) return {256, 1, 1};
    const int bt = a.rows <= 32 ? 32 : a.rows <= 64 ? 64 : 128;
    int split = 1;
    while (split < 8 && tiles(bt) * split * 2 <= n_sm + n_sm / 2 && blocks >= 4 * split) split *= 2;
    return {bt, 0, split};
}

template <int DT>
bool launch_linear(const LinearArgs& a, const Choice& c, int n_sm, int dev, cudaStream_t st) {
    if (c.tokens == 0) return launch_rows<DT>(a, n_sm, st);
    if (c.tokens == 8) return launch_few<DT>(a, n_sm, st);
    if (c.pair) return c.tokens == 256 ? launch_pair<256, DT>(a, n_sm, dev, st) : launch_pair<128, DT>(a, n_sm, dev, st);
    switch (c.tokens) {
        case 32: return launch_tile<32, DT>(a, c.split, dev, st);
        case 64: return launch_tile<64, DT>(a, c.split, dev, st);
        default: return launch_tile<128, DT>(a, c.split, dev, st);
    }
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
    const int64_t limit = (int64_t)1 << 31, span = (int64_t)1 << 60;
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
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n_sm, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return DNNS_ERR_CUDA;
    const Choice c = choose(a, n_sm);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool launched = dtype == DNNS_F32 ? launch_linear<DNNS_F32>(a, c, n_sm, dev, st) : launch_linear<DNNS_BF16>(a, c, n_sm, dev, st);
    return launched && cudaGetLastError() == cudaSuccess ? DNNS_OK : DNNS_ERR_CUDA;
}
