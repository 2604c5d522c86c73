// Rows in 8 bits: quantisation of a matrix's rows, fused with what produces them in a language model's block - the
// root-mean-square norm with the residual's addition, and the gated activation - and the gradients of those two.
//   Q(y): a = max |y|, scale = a / 127, q = rint(y * 127 / a).
//
// All five are bound by memory: a few operations an element against 5 to 9 bytes of traffic.  So each row is read
// once and kept in registers (fp32) between the reduction that its scale needs and the stores.  For the norm the
// reduction is a single one, because q does not depend on the row's root mean square: with v = h * weight and
// r = 1 / sqrt(mean(h^2) + eps), q = rint(v * 127 / max|v|) and scale = r * max|v| / 127, so the sum of squares and the
// maximum travel through the same shuffles and the same barrier.
//
// A thread works on pieces of 8 columns.  Where every row of every matrix starts on 16 bytes (VEC) a piece is 8
// neighbouring columns moved as 16-byte vectors; otherwise neighbouring threads take neighbouring columns, one element an
// access, so that a warp still touches whole sectors.  NV pieces a thread: a row of up to 8 * NV * threads columns stays in
// registers; longer rows (NV = 0) are walked twice.
#include <algorithm>

#include "dnns_internal.cuh"

namespace dnns {

namespace {

constexpr uint32_t kFullMask = 0xFFFFFFFFu;
constexpr uint32_t kInfBits = 0x7F800000u;
constexpr int kMaxRowThreads = 1024;
constexpr int kWarpRows = 8;       // rows per block where a warp has a row to itself
constexpr int kBackThreads = 512;  // threads a row of the norm's gradient at most

template <int DT>
struct Store;
template <>
struct Store<DNNS_F32> {
    typedef float type;
};
template <>
struct Store<DNNS_BF16> {
    typedef uint16_t type;
};

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
// two fp32 to two bf16, nearest even, in one word (lo in the low half)
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    uint32_t d;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
__device__ __forceinline__ void narrow(float x, float& d) { d = x; }
__device__ __forceinline__ void narrow(float x, uint16_t& d) { d = (uint16_t)bf16_pair(x, 0.0f); }

// Column of element e of piece j of thread t.
template <bool VEC>
__device__ __forceinline__ int64_t column(int64_t j, int e, int t, int threads) {
    return VEC ? (j * threads + t) * 8 + e : (j * 8 + e) * threads + t;
}

// Piece j of a row; columns past the end read as 0.
template <bool VEC, typename T>
__device__ __forceinline__ void load8(const T* row, int64_t j, int t, int threads, int64_t cols, float (&v)[8]) {
    const int64_t c0 = column<VEC>(j, 0, t, threads);
    if (VEC && c0 + 8 <= cols) {
        if constexpr (sizeof(T) == 4) {
            const float4 a = *reinterpret_cast<const float4*>(row + c0), b = *reinterpret_cast<const float4*>(row + c0 + 4);
            v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
        } else {
            const uint4 a = *reinterpret_cast<const uint4*>(row + c0);
            const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int64_t c = column<VEC>(j, e, t, threads);
        v[e] = c < cols ? widen(row[c]) : 0.0f;
    }
}

template <bool VEC, typename T>
__device__ __forceinline__ void store8(T* row, int64_t j, int t, int threads, int64_t cols, const float (&v)[8]) {
    const int64_t c0 = column<VEC>(j, 0, t, threads);
    if (VEC && c0 + 8 <= cols) {
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<float4*>(row + c0) = make_float4(v[0], v[1], v[2], v[3]);
            *reinterpret_cast<float4*>(row + c0 + 4) = make_float4(v[4], v[5], v[6], v[7]);
        } else {
            *reinterpret_cast<uint4*>(row + c0) = make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7]));
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int64_t c = column<VEC>(j, e, t, threads);
        if (c < cols) narrow(v[e], row[c]);
    }
}

template <bool VEC>
__device__ __forceinline__ void store8_int(int8_t* row, int64_t j, int t, int threads, int64_t cols, const int (&q)[8]) {
    const int64_t c0 = column<VEC>(j, 0, t, threads);
    if (VEC && c0 + 8 <= cols) {
        uint32_t w[2];
#pragma unroll
        for (int i = 0; i < 2; ++i)
            w[i] = __byte_perm(__byte_perm(q[4 * i], q[4 * i + 1], 0x0040), __byte_perm(q[4 * i + 2], q[4 * i + 3], 0x0040), 0x5410);
        *reinterpret_cast<uint2*>(row + c0) = make_uint2(w[0], w[1]);
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int64_t c = column<VEC>(j, e, t, threads);
        if (c < cols) row[c] = (int8_t)q[e];
    }
}

// Sum of `a`, sum of `b` and maximum of `m` over the threads of a row (a warp, or a block).  `scratch`: 3 * 33 words,
// free for the next row after one more barrier.
template <bool WARP, bool TWO>
__device__ __forceinline__ void row_reduce(float& a, float& b, uint32_t& m, uint32_t* scratch) {
#pragma unroll
    for (int d = 16; d; d >>= 1) {
        a += __shfl_xor_sync(kFullMask, a, d);
        if (TWO) b += __shfl_xor_sync(kFullMask, b, d);
    }
    m = __reduce_max_sync(kFullMask, m);
    if (WARP || blockDim.x == 32) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    if (lane == 0) scratch[warp] = __float_as_uint(a), scratch[33 + warp] = m, scratch[66 + warp] = __float_as_uint(b);
    __syncthreads();
    a = lane < warps ? __uint_as_float(scratch[lane]) : 0.0f;
    b = TWO && lane < warps ? __uint_as_float(scratch[66 + lane]) : 0.0f;
    m = lane < warps ? scratch[33 + lane] : 0u;
#pragma unroll
    for (int d = 16; d; d >>= 1) {
        a += __shfl_xor_sync(kFullMask, a, d);
        if (TWO) b += __shfl_xor_sync(kFullMask, b, d);
    }
    m = __reduce_max_sync(kFullMask, m);
}

enum RowOp { kPlain, kGate, kNorm };

struct QuantArgs {
    const void *x, *x2;   // the matrix; residual of the norm, `up` of the gate
    const float* weight;  // norm (nullable)
    void* h;              // norm (nullable)
    int8_t* q;
    float* scale;
    uint16_t* values;     // nullable
    int64_t ldx, ldx2, ldh, ldq, ldv, rows, cols;
    float eps;
};

__device__ __forceinline__ float sigmoid(float g) { return 1.0f / (1.0f + __expf(-g)); }

// What a row consists of: piece j of v (the values to be quantised up to a factor of the row), h on the way.
template <int OP, int DT, bool VEC>
__device__ __forceinline__ void row_piece(const QuantArgs& a, int64_t r, int64_t j, int t, int threads, float (&v)[8], float (&h)[8]) {
    typedef typename Store<DT>::type T;
    load8<VEC>(static_cast<const T*>(a.x) + r * a.ldx, j, t, threads, a.cols, h);
    if (OP == kPlain) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = h[e];
    } else if (OP == kGate) {
        float u[8];
        load8<VEC>(static_cast<const T*>(a.x2) + r * a.ldx2, j, t, threads, a.cols, u);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = h[e] * sigmoid(h[e]) * u[e];
    } else {
        if (a.x2) {
            float s[8];
            load8<VEC>(static_cast<const T*>(a.x2) + r * a.ldx2, j, t, threads, a.cols, s);
#pragma unroll
            for (int e = 0; e < 8; ++e) h[e] += s[e];
        }
        if (a.weight) {
            float w[8];
            load8<VEC>(a.weight, j, t, threads, a.cols, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = h[e] * w[e];
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = h[e];
        }
    }
}

// The factor that turns v into steps of the row, and the step itself.
struct RowScale {
    float pre, inv, scale;
};
__device__ __forceinline__ RowScale row_scale(uint32_t top_bits, float factor) {
    RowScale s{1.0f, 0.0f, 0.0f};
    const float top = __uint_as_float(top_bits);
    if (top_bits >= kInfBits || __float_as_uint(fabsf(factor)) >= kInfBits) {
        s.scale = __uint_as_float(0x7FC00000u);
    } else if (top_bits) {
        // 127 / top is out of range for a tiny top: the row is brought up by a power of two first (exact)
        if (top < 0x1p-100f) s.pre = 0x1p100f;
        s.inv = 127.0f / (top * s.pre);
        s.scale = top * factor / 127.0f;
        if (__float_as_uint(s.scale) >= kInfBits) s.scale = __uint_as_float(0x7FC00000u), s.inv = 0.0f;
    }
    return s;
}

template <bool VEC>
__device__ __forceinline__ void store_quantized(const QuantArgs& a, int64_t r, int64_t j, int t, int threads, const float (&v)[8], const RowScale& s) {
    int q[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) q[e] = s.inv == 0.0f ? 0 : __float2int_rn(v[e] * s.pre * s.inv);
    store8_int<VEC>(a.q + r * a.ldq, j, t, threads, a.cols, q);
    if (a.values) {
        float z[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = (float)q[e] * s.scale;
        store8<VEC>(a.values + r * a.ldv, j, t, threads, a.cols, z);
    }
}

// blockDim.x threads a row; WARP: 32 of them, blockDim.y rows a block.
template <int OP, int DT, bool VEC, bool WARP, int NV>
__global__ void __launch_bounds__(WARP ? 32 * kWarpRows : kMaxRowThreads) k_rows_quantize(const QuantArgs a) {
    typedef typename Store<DT>::type T;
    __shared__ uint32_t scratch[99];
    const int t = threadIdx.x, threads = WARP ? 32 : blockDim.x;
    const int64_t r = WARP ? (int64_t)blockIdx.x * blockDim.y + threadIdx.y : blockIdx.x;
    if (WARP && r >= a.rows) return;
    float sum = 0.0f, unused = 0.0f;
    uint32_t top = 0;
    constexpr int kHeld = NV ? NV : 1;
    float v[kHeld][8];
    const int64_t pieces = NV ? NV : (a.cols + 8 * threads - 1) / (8 * threads);
    auto take = [&](int64_t j, float (&p)[8]) {
        float h[8];
        row_piece<OP, DT, VEC>(a, r, j, t, threads, p, h);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (OP == kNorm) sum = fmaf(h[e], h[e], sum);
            top = max(top, __float_as_uint(fabsf(p[e])));
        }
        // (the first walk over a row that is read twice leaves h alone: it may be x or the residual itself)
        if (OP == kNorm && NV && a.h) store8<VEC>(static_cast<T*>(a.h) + r * a.ldh, j, t, threads, a.cols, h);
    };
    if (NV) {
#pragma unroll
        for (int j = 0; j < kHeld; ++j) take(j, v[j]);
    } else {
        for (int64_t j = 0; j < pieces; ++j) take(j, v[0]);
    }
    row_reduce<WARP, false>(sum, unused, top, scratch);
    const float factor = OP == kNorm ? 1.0f / sqrtf(sum / (float)a.cols + a.eps) : 1.0f;
    const bool lost = OP == kNorm && __float_as_uint(sum) >= kInfBits;
    const RowScale s = row_scale(lost ? kInfBits : top, factor);
    if (t == 0) a.scale[r] = s.scale;
    if (NV) {
#pragma unroll
        for (int j = 0; j < kHeld; ++j) store_quantized<VEC>(a, r, j, t, threads, v[j], s);
    } else {
        for (int64_t j = 0; j < pieces; ++j) {
            float h[8];
            row_piece<OP, DT, VEC>(a, r, j, t, threads, v[0], h);
            if (OP == kNorm && a.h) store8<VEC>(static_cast<T*>(a.h) + r * a.ldh, j, t, threads, a.cols, h);
            store_quantized<VEC>(a, r, j, t, threads, v[0], s);
        }
    }
}

template <int OP, int DT, bool VEC>
void launch_quantize(const QuantArgs& a, int n_sm, cudaStream_t st) {
    const int64_t cols = a.cols;
    if (cols <= 1024 && a.rows > n_sm) {
        const dim3 block(32, kWarpRows);
        const unsigned grid = (unsigned)((a.rows + kWarpRows - 1) / kWarpRows);
        if (cols <= 256) k_rows_quantize<OP, DT, VEC, true, 1><<<grid, block, 0, st>>>(a);
        else if (cols <= 512) k_rows_quantize<OP, DT, VEC, true, 2><<<grid, block, 0, st>>>(a);
        else k_rows_quantize<OP, DT, VEC, true, 4><<<grid, block, 0, st>>>(a);
        return;
    }
    const unsigned grid = (unsigned)a.rows;
    auto threads = [&](int nv) { return (int)std::max<int64_t>(1, (cols + 256 * nv - 1) / (256 * nv)) * 32; };
    // few rows: as many threads as the row feeds; many rows: more bytes in flight per thread, more rows per SM
    if (cols > 8 * 4 * kMaxRowThreads) k_rows_quantize<OP, DT, VEC, false, 0><<<grid, kMaxRowThreads, 0, st>>>(a);
    else if (a.rows <= n_sm && cols <= 8 * kMaxRowThreads) k_rows_quantize<OP, DT, VEC, false, 1><<<grid, threads(1), 0, st>>>(a);
    else if (a.rows <= n_sm && cols <= 16 * kMaxRowThreads) k_rows_quantize<OP, DT, VEC, false, 2><<<grid, threads(2), 0, st>>>(a);
    else k_rows_quantize<OP, DT, VEC, false, 4><<<grid, threads(4), 0, st>>>(a);
}

// ---- gradients -------------------------------------------------------------------------------------------------
struct NormBackArgs {
    const void *dy, *h, *dh;  // dh nullable
    const float* weight;      // nullable
    void* dx;
    float* part;              // [gridDim.x][cols] partial sums of dweight (nullable)
    int64_t lddy, ldh, lddh, lddx, rows, cols;
    float eps;
};

// A block takes rows blockIdx.x, + gridDim.x, ...; a thread keeps its columns, so the partial sums of dweight stay in
// registers (NV = 0: in the block's slice of the workspace) until the block is done.
template <int DT, bool VEC, int NV>
__global__ void __launch_bounds__(NV ? kBackThreads : kMaxRowThreads) k_norm_backward(const NormBackArgs a) {
    typedef typename Store<DT>::type T;
    __shared__ uint32_t scratch[2][99];
    const int t = threadIdx.x, threads = blockDim.x;
    constexpr int kHeld = NV ? NV : 1;
    float dw[kHeld][8];
#pragma unroll
    for (int j = 0; j < kHeld; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[j][e] = 0.0f;
    const int64_t pieces = NV ? NV : (a.cols + 8 * threads - 1) / (8 * threads);
    float* part = a.part ? a.part + (int64_t)blockIdx.x * a.cols : nullptr;
    int side = 0;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x, side ^= 1) {
        const T* dy = static_cast<const T*>(a.dy) + r * a.lddy;
        const T* h = static_cast<const T*>(a.h) + r * a.ldh;
        const T* dh = static_cast<const T*>(a.dh) + r * a.lddh;
        T* dx = static_cast<T*>(a.dx) + r * a.lddx;
        float hv[kHeld][8], gv[kHeld][8];
        float sq = 0.0f, along = 0.0f;
        uint32_t unused = 0;
        auto take = [&](int64_t j, float (&hp)[8], float (&gp)[8]) {
            load8<VEC>(h, j, t, threads, a.cols, hp);
            load8<VEC>(dy, j, t, threads, a.cols, gp);
        };
        auto weigh = [&](int64_t j, const float (&gp)[8], float (&g)[8]) {
            if (a.weight) {
                float w[8];
                load8<VEC>(a.weight, j, t, threads, a.cols, w);
#pragma unroll
                for (int e = 0; e < 8; ++e) g[e] = gp[e] * w[e];
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) g[e] = gp[e];
            }
        };
        auto sums = [&](int64_t j, const float (&hp)[8], const float (&gp)[8]) {
            float g[8];
            weigh(j, gp, g);
#pragma unroll
            for (int e = 0; e < 8; ++e) sq = fmaf(hp[e], hp[e], sq), along = fmaf(g[e], hp[e], along);
        };
        if (NV) {
#pragma unroll
            for (int j = 0; j < kHeld; ++j) take(j, hv[j], gv[j]);
#pragma unroll
            for (int j = 0; j < kHeld; ++j) sums(j, hv[j], gv[j]);
        } else {
            for (int64_t j = 0; j < pieces; ++j) take(j, hv[0], gv[0]), sums(j, hv[0], gv[0]);
        }
        row_reduce<false, true>(sq, along, unused, scratch[side]);  // (two buffers: a row's barrier frees the row before)
        const float inv_n = 1.0f / (float)a.cols;
        const float root = 1.0f / sqrtf(sq * inv_n + a.eps);
        const float coef = along * root * inv_n;
        auto give = [&](int64_t j, const float (&hp)[8], const float (&gp)[8], float (&w)[8]) {
            float g[8], o[8];
            weigh(j, gp, g);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float unit = hp[e] * root;
                o[e] = root * (g[e] - unit * coef);
                w[e] = fmaf(gp[e], unit, w[e]);
            }
            if (a.dh) {
                float p[8];
                load8<VEC>(dh, j, t, threads, a.cols, p);
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] += p[e];
            }
            store8<VEC>(dx, j, t, threads, a.cols, o);
        };
        if (NV) {
#pragma unroll
            for (int j = 0; j < kHeld; ++j) give(j, hv[j], gv[j], dw[j]);
        } else {
            for (int64_t j = 0; j < pieces; ++j) {
                float w[8] = {0, 0, 0, 0, 0, 0, 0, 0};
                take(j, hv[0], gv[0]);
                if (part && r != blockIdx.x) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int64_t c = column<VEC>(j, e, t, threads);
                        if (c < a.cols) w[e] = part[c];
                    }
                }
                give(j, hv[0], gv[0], w);
                if (part) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int64_t c = column<VEC>(j, e, t, threads);
                        if (c < a.cols) part[c] = w[e];
                    }
                }
            }
        }
    }
    if (NV && part) {
#pragma unroll
        for (int j = 0; j < kHeld; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int64_t c = column<VEC>(j, e, t, threads);
                if (c < a.cols) part[c] = dw[j][e];
            }
    }
}

// dweight[c] = sum of the row groups' partial sums, in order of the groups: 32 columns by 32 runs of groups a block.
__global__ void __launch_bounds__(1024) k_norm_weight_sum(const float* __restrict__ part, int64_t groups, int64_t cols, float* __restrict__ dweight) {
    __shared__ float s[32][33];
    const int64_t c = (int64_t)blockIdx.x * 32 + threadIdx.x;
    float sum = 0.0f;
    if (c < cols)
        for (int64_t g = threadIdx.y; g < groups; g += 32) sum += part[g * cols + c];
    s[threadIdx.y][threadIdx.x] = sum;
    __syncthreads();
    if (threadIdx.y == 0 && c < cols) {
        float all = 0.0f;
#pragma unroll
        for (int g = 0; g < 32; ++g) all += s[g][threadIdx.x];
        dweight[c] = all;
    }
}

struct GateBackArgs {
    const void *dy, *gate, *up;
    void *dgate, *dup;
    int64_t lddy, ldg, ldu, lddg, lddu, rows, cols;
};

template <int DT, bool VEC>
__global__ void __launch_bounds__(256) k_gate_backward(const GateBackArgs a, int64_t pieces) {
    typedef typename Store<DT>::type T;
    const int t = threadIdx.x;
    for (int64_t i = blockIdx.x; i < a.rows * pieces; i += gridDim.x) {
        const int64_t r = i / pieces, j = i - r * pieces;
        float d[8], g[8], u[8], dg[8], du[8];
        load8<VEC>(static_cast<const T*>(a.dy) + r * a.lddy, j, t, 256, a.cols, d);
        load8<VEC>(static_cast<const T*>(a.gate) + r * a.ldg, j, t, 256, a.cols, g);
        load8<VEC>(static_cast<const T*>(a.up) + r * a.ldu, j, t, 256, a.cols, u);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float s = sigmoid(g[e]);
            dg[e] = d[e] * u[e] * s * fmaf(g[e], 1.0f - s, 1.0f);
            du[e] = d[e] * g[e] * s;
        }
        store8<VEC>(static_cast<T*>(a.dgate) + r * a.lddg, j, t, 256, a.cols, dg);
        store8<VEC>(static_cast<T*>(a.dup) + r * a.lddu, j, t, 256, a.cols, du);
    }
}

// ---- host side ---------------------------------------------------------------------------------------------------
constexpr int64_t kMaxExtent = (int64_t)1 << 31;

bool extent_ok(int64_t rows, int64_t cols) { return rows < kMaxExtent && cols < kMaxExtent; }
bool span_ok(int64_t rows, int64_t ld) { return rows == 0 || ld <= ((int64_t)1 << 60) / rows; }
bool matrix_arg_ok(const void* p, int64_t ld, int64_t cols, size_t align) { return p && reinterpret_cast<uintptr_t>(p) % align == 0 && ld >= cols; }
bool on_16(const void* p, int64_t ld, int64_t rows, size_t elem) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (rows <= 1 || ld * (int64_t)elem % 16 == 0);
}
size_t elem_bytes(int32_t dtype) { return dtype == DNNS_F32 ? 4 : 2; }

int sm_count() {
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    return n;
}

// The checks that the three quantising calls share; on DNNS_OK *launch says whether there is anything to do.
dnns_status check_quantize(const QuantArgs& a, int32_t dtype, bool* launch) {
    *launch = false;
    if (a.rows < 0 || a.cols < 0) return DNNS_ERR_INVALID_ARG;
    if (dtype != DNNS_F32 && dtype != DNNS_BF16) return DNNS_ERR_UNSUPPORTED;
    if (!extent_ok(a.rows, a.cols)) return DNNS_ERR_UNSUPPORTED;
    const size_t e = elem_bytes(dtype);
    if (a.rows == 0) return DNNS_OK;
    if (!a.scale || reinterpret_cast<uintptr_t>(a.scale) % 4) return DNNS_ERR_INVALID_ARG;
    if (a.cols) {
        if (!matrix_arg_ok(a.x, a.ldx, a.cols, e) || !matrix_arg_ok(a.q, a.ldq, a.cols, 16) || a.ldq % 16) return DNNS_ERR_INVALID_ARG;
        if (a.x2 && !matrix_arg_ok(a.x2, a.ldx2, a.cols, e)) return DNNS_ERR_INVALID_ARG;
        if (a.h && !matrix_arg_ok(a.h, a.ldh, a.cols, e)) return DNNS_ERR_INVALID_ARG;
        if (a.values && !matrix_arg_ok(a.values, a.ldv, a.cols, 2)) return DNNS_ERR_INVALID_ARG;
        if (a.weight && reinterpret_cast<uintptr_t>(a.weight) % 4) return DNNS_ERR_INVALID_ARG;
        if (!span_ok(a.rows, a.ldx) || !span_ok(a.rows, a.ldq) || (a.x2 && !span_ok(a.rows, a.ldx2)) || (a.h && !span_ok(a.rows, a.ldh)) ||
            (a.values && !span_ok(a.rows, a.ldv)))
            return DNNS_ERR_UNSUPPORTED;
    }
    *launch = true;
    return DNNS_OK;
}

template <int OP>
dnns_status run_quantize(const QuantArgs& a, int32_t dtype, void* stream) {
    bool launch;
    const dnns_status s = check_quantize(a, dtype, &launch);
    if (s != DNNS_OK || !launch) return s;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (a.cols == 0) return cudaMemsetAsync(a.scale, 0, (size_t)a.rows * sizeof(float), st) == cudaSuccess ? DNNS_OK : DNNS_ERR_CUDA;
    const int n_sm = sm_count();
    if (n_sm == 0) return DNNS_ERR_CUDA;
    const size_t e = elem_bytes(dtype);
    const bool vec = on_16(a.x, a.ldx, a.rows, e) && (!a.x2 || on_16(a.x2, a.ldx2, a.rows, e)) && (!a.h || on_16(a.h, a.ldh, a.rows, e)) &&
                     (!a.values || on_16(a.values, a.ldv, a.rows, 2)) && (!a.weight || on_16(a.weight, 0, 1, 4));
    if (dtype == DNNS_F32) vec ? launch_quantize<OP, DNNS_F32, true>(a, n_sm, st) : launch_quantize<OP, DNNS_F32, false>(a, n_sm, st);
    else vec ? launch_quantize<OP, DNNS_BF16, true>(a, n_sm, st) : launch_quantize<OP, DNNS_BF16, false>(a, n_sm, st);
    return cudaGetLastError() == cudaSuccess ? DNNS_OK : DNNS_ERR_CUDA;
}

// Blocks of the norm's gradient: bounded by the rows, and by what a machine of up to 160 SMs holds at a time; the
// workspace is sized for it without asking the device.
int64_t norm_backward_groups(int64_t rows) { return std::min<int64_t>(rows, 320); }

template <int DT, bool VEC>
void launch_norm_backward(const NormBackArgs& a, cudaStream_t st) {
    const unsigned grid = (unsigned)norm_backward_groups(a.rows);
    auto threads = [&](int nv) { return (int)((a.cols + 256 * nv - 1) / (256 * nv)) * 32; };
    if (a.cols > 8 * 4 * kBackThreads) k_norm_backward<DT, VEC, 0><<<grid, kMaxRowThreads, 0, st>>>(a);
    else if (a.cols <= 8 * kBackThreads) k_norm_backward<DT, VEC, 1><<<grid, threads(1), 0, st>>>(a);
    else if (a.cols <= 16 * kBackThreads) k_norm_backward<DT, VEC, 2><<<grid, threads(2), 0, st>>>(a);
    else k_norm_backward<DT, VEC, 4><<<grid, threads(4), 0, st>>>(a);
}

bool eps_ok(float eps) { return eps >= 0x1p-126f && eps <= 3.402823466e38f; }

}  // namespace

}  // namespace dnns

extern "C" {

size_t dnns_quantized_row_bytes(size_t cols) { return (cols + 15) / 16 * 16; }

dnns_status dnns_quantize_rows(const void* x, int64_t ldx, int32_t dtype, int64_t rows, int64_t cols, int8_t* q, int64_t ldq,
                               float* scale, uint16_t* values, int64_t ldv, void* stream) {
    const dnns::QuantArgs a{x, nullptr, nullptr, nullptr, q, scale, values, ldx, 0, 0, ldq, ldv, rows, cols, 0.0f};
    return dnns::run_quantize<dnns::kPlain>(a, dtype, stream);
}

dnns_status dnns_rmsnorm_quantize(const void* x, int64_t ldx, const void* residual, int64_t ldr, const float* weight, float eps,
                                  int32_t dtype, int64_t rows, int64_t cols, void* h_out, int64_t ldh, int8_t* q, int64_t ldq,
                                  float* scale, uint16_t* values, int64_t ldv, void* stream) {
    if (!dnns::eps_ok(eps)) return DNNS_ERR_INVALID_ARG;
    const dnns::QuantArgs a{x, residual, weight, h_out, q, scale, values, ldx, ldr, ldh, ldq, ldv, rows, cols, eps};
    return dnns::run_quantize<dnns::kNorm>(a, dtype, stream);
}

dnns_status dnns_silu_gate_quantize(const void* gate, int64_t ldg, const void* up, int64_t ldu, int32_t dtype, int64_t rows,
                                    int64_t cols, int8_t* q, int64_t ldq, float* scale, uint16_t* values, int64_t ldv, void* stream) {
    if (rows > 0 && cols > 0 && !up) return DNNS_ERR_INVALID_ARG;
    const dnns::QuantArgs a{gate, up, nullptr, nullptr, q, scale, values, ldg, ldu, 0, ldq, ldv, rows, cols, 0.0f};
    return dnns::run_quantize<dnns::kGate>(a, dtype, stream);
}

size_t dnns_rmsnorm_backward_workspace_bytes(int64_t rows, int64_t cols) {
    if (rows <= 0 || cols <= 0 || !dnns::extent_ok(rows, cols)) return 0;
    return ((size_t)dnns::norm_backward_groups(rows) * (size_t)cols * sizeof(float) + 255) & ~(size_t)255;
}

dnns_status dnns_rmsnorm_backward(const void* dy, int64_t lddy, const void* h, int64_t ldh, const float* weight, float eps,
                                  const void* dh, int64_t lddh, int32_t dtype, int64_t rows, int64_t cols, void* dx, int64_t lddx,
                                  float* dweight, void* ws_dev, size_t ws_bytes, void* stream) {
    using namespace dnns;
    if (!eps_ok(eps) || rows < 0 || cols < 0) return DNNS_ERR_INVALID_ARG;
    if ((dtype != DNNS_F32 && dtype != DNNS_BF16) || !extent_ok(rows, cols)) return DNNS_ERR_UNSUPPORTED;
    const size_t e = elem_bytes(dtype);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (cols == 0) return DNNS_OK;
    if (reinterpret_cast<uintptr_t>(dweight) % 4 || reinterpret_cast<uintptr_t>(weight) % 4) return DNNS_ERR_INVALID_ARG;
    if (rows == 0) {
        if (dweight && cudaMemsetAsync(dweight, 0, (size_t)cols * sizeof(float), st) != cudaSuccess) return DNNS_ERR_CUDA;
        return DNNS_OK;
    }
    if (!matrix_arg_ok(dy, lddy, cols, e) || !matrix_arg_ok(h, ldh, cols, e) || !matrix_arg_ok(dx, lddx, cols, e) ||
        (dh && !matrix_arg_ok(dh, lddh, cols, e)))
        return DNNS_ERR_INVALID_ARG;
    if (!span_ok(rows, lddy) || !span_ok(rows, ldh) || !span_ok(rows, lddx) || (dh && !span_ok(rows, lddh))) return DNNS_ERR_UNSUPPORTED;
    if (dweight) {
        if (!ws_dev || reinterpret_cast<uintptr_t>(ws_dev) % 16) return DNNS_ERR_INVALID_ARG;
        if (ws_bytes < dnns_rmsnorm_backward_workspace_bytes(rows, cols)) return DNNS_ERR_WORKSPACE;
    }
    const NormBackArgs a{dy, h, dh, weight, dx, dweight ? static_cast<float*>(ws_dev) : nullptr, lddy, ldh, lddh, lddx, rows, cols, eps};
    const bool vec = on_16(dy, lddy, rows, e) && on_16(h, ldh, rows, e) && on_16(dx, lddx, rows, e) && (!dh || on_16(dh, lddh, rows, e)) &&
                     (!weight || on_16(weight, 0, 1, 4));
    if (dtype == DNNS_F32) vec ? launch_norm_backward<DNNS_F32, true>(a, st) : launch_norm_backward<DNNS_F32, false>(a, st);
    else vec ? launch_norm_backward<DNNS_BF16, true>(a, st) : launch_norm_backward<DNNS_BF16, false>(a, st);
    if (dweight) k_norm_weight_sum<<<(unsigned)((cols + 31) / 32), dim3(32, 32), 0, st>>>(a.part, norm_backward_groups(rows), cols, dweight);
    return cudaGetLastError() == cudaSuccess ? DNNS_OK : DNNS_ERR_CUDA;
}

dnns_status dnns_silu_gate_backward(const void* dy, int64_t lddy, const void* gate, int64_t ldg, const void* up, int64_t ldu,
                                    int32_t dtype, int64_t rows, int64_t cols, void* dgate, int64_t lddg, void* dup, int64_t lddu,
                                    void* stream) {
    using namespace dnns;
    if (rows < 0 || cols < 0) return DNNS_ERR_INVALID_ARG;
    if ((dtype != DNNS_F32 && dtype != DNNS_BF16) || !extent_ok(rows, cols)) return DNNS_ERR_UNSUPPORTED;
    if (rows == 0 || cols == 0) return DNNS_OK;
    const size_t e = elem_bytes(dtype);
    if (!matrix_arg_ok(dy, lddy, cols, e) || !matrix_arg_ok(gate, ldg, cols, e) || !matrix_arg_ok(up, ldu, cols, e) ||
        !matrix_arg_ok(dgate, lddg, cols, e) || !matrix_arg_ok(dup, lddu, cols, e))
        return DNNS_ERR_INVALID_ARG;
    if (!span_ok(rows, lddy) || !span_ok(rows, ldg) || !span_ok(rows, ldu) || !span_ok(rows, lddg) || !span_ok(rows, lddu))
        return DNNS_ERR_UNSUPPORTED;
    const int n_sm = sm_count();
    if (n_sm == 0) return DNNS_ERR_CUDA;
    const GateBackArgs a{dy, gate, up, dgate, dup, lddy, ldg, ldu, lddg, lddu, rows, cols};
    const bool vec = on_16(dy, lddy, rows, e) && on_16(gate, ldg, rows, e) && on_16(up, ldu, rows, e) && on_16(dgate, lddg, rows, e) &&
                     on_16(dup, lddu, rows, e);
    const int64_t pieces = (cols + 2047) / 2048;
    const unsigned grid = (unsigned)std::min<int64_t>(rows * pieces, (int64_t)n_sm * 64);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (dtype == DNNS_F32) vec ? k_gate_backward<DNNS_F32, true><<<grid, 256, 0, st>>>(a, pieces) : k_gate_backward<DNNS_F32, false><<<grid, 256, 0, st>>>(a, pieces);
    else vec ? k_gate_backward<DNNS_BF16, true><<<grid, 256, 0, st>>>(a, pieces) : k_gate_backward<DNNS_BF16, false><<<grid, 256, 0, st>>>(a, pieces);
    return cudaGetLastError() == cudaSuccess ? DNNS_OK : DNNS_ERR_CUDA;
}

}  // extern "C"
