// Rows in 8 bits: quantisation of a matrix's rows, fused with what produces them in a language model's block - the
// root-mean-square norm with the residual's addition, and the gated activation - and the gradients of those two.
//   Q(y): a = max |y|, scale = a / 127, q = rint(y * 127 / a).
//
// All five are bound by memory: a few operations an element against 3 to 10 bytes of traffic in bf16, 5 to 20 in fp32.  So each row is read
// once and kept in registers (fp32) between the reduction that its scale needs and the stores.  For the norm the
// reduction is a single one, because q does not depend on the row's root mean square: with v = h * weight and
// r = 1 / sqrt(mean(h^2) + eps), q = rint(v * 127 / max|v|) and scale = r * max|v| / 127, so the sum of squares and the
// maximum travel through the same shuffles and the same barrier.
//
// A team of warps has a row (a block; for short rows a warp, several a block), and a warp works on pieces of 256 columns.  Where
// every row of every matrix starts on 16 bytes (VEC) a lane takes 8 neighbouring columns of a piece and moves them as
// vectors.  Rows of a rebuilt layer have any width, so they start anywhere: then a lane takes every 32nd column, one element an
// access at fixed offsets from one address; a warp still touches whole sectors, and the accesses are fewer
// instructions than shifting misaligned vectors into place would be.  NV pieces a warp: a row of up to 256 * NV * warps columns
// stays in registers, and longer ones (NV = 0) are walked twice.  All loads of a row are issued before the first is used.
#include <algorithm>

#include "dnns_internal.cuh"

namespace dnns {

namespace {

constexpr uint32_t kFullMask = 0xFFFFFFFFu;
constexpr uint32_t kInfBits = 0x7F800000u;
constexpr uint32_t kNanBits = 0x7FC00000u;
constexpr int kBlockWarps = 8;  // warps of a block whose teams are single warps
// Warps of a team at most, by pieces a lane: what keeps a row in registers without spilling.
constexpr int quantize_warps(int nv) { return nv == 4 ? 16 : 32; }
constexpr int backward_warps(int nv) { return nv == 4 ? 16 : 8; }

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

// two fp32 to two bf16, nearest even, in one word (lo in the low half)
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    uint32_t d;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
__device__ __forceinline__ void narrow(float x, float& d) { d = x; }
__device__ __forceinline__ void narrow(float x, uint16_t& d) { d = (uint16_t)bf16_pair(x, 0.0f); }

// ---- pieces of 256 columns of a row, 8 of them a lane's -------------------------------------------------------------
// The first column of a lane in piece j of warp `warp` of a team of `warps`.
template <bool VEC>
__device__ __forceinline__ int first_column(int j, int warps, int warp) {
    const int lane = threadIdx.x & 31;
    return (j * warps + warp) * 256 + (VEC ? 8 * lane : lane);
}
template <bool VEC>
constexpr int kStep = VEC ? 1 : 32;  // from one of a lane's columns to the next
// All columns of the warp's piece are inside the row (the same for all lanes).
template <bool VEC>
__device__ __forceinline__ bool piece_inside(int c, int cols) { return c - (VEC ? 8 : 1) * (int)(threadIdx.x & 31) + 256 <= cols; }
// None is.
template <bool VEC>
__device__ __forceinline__ bool piece_outside(int c, int cols) { return c - (VEC ? 8 : 1) * (int)(threadIdx.x & 31) >= cols; }

// The 8 values as they are stored: vectors, or one element a word.  Loads are asm volatile, so that they are issued
// where they stand - all of a row's before the first of them is waited for.
template <bool VEC, typename T>
struct Raw {
    static constexpr int kWords = VEC ? 2 * sizeof(T) : 8;
    uint32_t w[kWords];
    __device__ __forceinline__ void fetch(const T* row, int c, int cols) {
        const T* p = row + c;
        if (piece_inside<VEC>(c, cols)) {
            if constexpr (VEC) {
#pragma unroll
                for (int i = 0; i < kWords / 4; ++i)
                    asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[4 * i]), "=r"(w[4 * i + 1]), "=r"(w[4 * i + 2]), "=r"(w[4 * i + 3]) : "l"(p + 16 / sizeof(T) * i) : "memory");
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) load_one(p + 32 * e, w[e]);
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = 0;
        if (piece_outside<VEC>(c, cols)) return;
        if constexpr (VEC) {
            const uint32_t whole = c + 8 <= cols;
#pragma unroll
            for (int i = 0; i < kWords / 4; ++i)
                asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %5, 0;\n\t@p ld.global.v4.u32 {%0, %1, %2, %3}, [%4];\n\t}"
                             : "+r"(w[4 * i]), "+r"(w[4 * i + 1]), "+r"(w[4 * i + 2]), "+r"(w[4 * i + 3])
                             : "l"(p + 16 / sizeof(T) * i), "r"(whole)
                             : "memory");
            if (!whole && c < cols) {  // the row's last columns
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (c + e < cols) {
                        if constexpr (sizeof(T) == 4) w[e] = __float_as_uint(p[e]);
                        else w[e / 2] |= (uint32_t)p[e] << (16 * (e & 1));
                    }
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (c + 32 * e < cols) load_one(p + 32 * e, w[e]);
        }
    }
    __device__ __forceinline__ float get(int e) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
        else if constexpr (VEC) return __uint_as_float(e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
        else return __uint_as_float(w[e] << 16);
    }
    static __device__ __forceinline__ void load_one(const T* p, uint32_t& x) {
        if constexpr (sizeof(T) == 4) asm volatile("ld.global.u32 %0, [%1];" : "=r"(x) : "l"(p) : "memory");
        else asm volatile("{\n\t.reg .u16 t;\n\tld.global.u16 t, [%1];\n\tcvt.u32.u16 %0, t;\n\t}" : "=r"(x) : "l"(p) : "memory");
    }
};
template <bool VEC>
__device__ __forceinline__ void load8(const float* row, int c, int cols, float (&v)[8]) {
    Raw<VEC, float> r;
    r.fetch(row, c, cols);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = r.get(e);
}

template <bool VEC, typename T>
__device__ __forceinline__ void store8(T* row, int c, int cols, const float (&v)[8]) {
    T* p = row + c;
    if (VEC ? c + 8 <= cols : piece_inside<VEC>(c, cols)) {
        if constexpr (!VEC) {
#pragma unroll
            for (int e = 0; e < 8; ++e) narrow(v[e], p[32 * e]);
        } else if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
            *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
        } else {
            *reinterpret_cast<uint4*>(p) = make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7]));
        }
        return;
    }
    if (piece_outside<VEC>(c, cols)) return;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (c + kStep<VEC> * e < cols) narrow(v[e], p[kStep<VEC> * e]);
}
// The low bytes of 8 words.
template <bool VEC>
__device__ __forceinline__ void store8_bytes(int8_t* row, int c, int cols, const uint32_t (&b)[8]) {
    int8_t* p = row + c;
    if (VEC ? c + 8 <= cols : piece_inside<VEC>(c, cols)) {
        if constexpr (VEC) {
            const uint32_t lo = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
            const uint32_t hi = __byte_perm(__byte_perm(b[4], b[5], 0x0040), __byte_perm(b[6], b[7], 0x0040), 0x5410);
            *reinterpret_cast<uint2*>(p) = make_uint2(lo, hi);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) p[32 * e] = (int8_t)b[e];
        }
        return;
    }
    if (piece_outside<VEC>(c, cols)) return;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (c + kStep<VEC> * e < cols) p[kStep<VEC> * e] = (int8_t)b[e];
}

// ---- reductions over a team: a warp (warps = 1), or the block ----------------------------------------------------
// Sum of `a` and maximum of `m`.  `scratch`: 64 words, free for another use after one more barrier.
template <bool SUM>
__device__ __forceinline__ void reduce_sum_max(int warps, float& a, uint32_t& m, uint32_t* scratch) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int round = 0; round < 2; ++round) {
        if (SUM) {
#pragma unroll
            for (int d = 16; d; d >>= 1) a += __shfl_xor_sync(kFullMask, a, d);
        }
        m = __reduce_max_sync(kFullMask, m);
        if (round || warps == 1) return;
        if (lane == 0) {
            if (SUM) scratch[warp] = __float_as_uint(a);
            scratch[32 + warp] = m;
        }
        __syncthreads();
        if (SUM) a = lane < warps ? __uint_as_float(scratch[lane]) : 0.0f;
        m = lane < warps ? scratch[32 + lane] : 0u;
    }
}

// Sums of `a` and `b` over up to 16 warps: the lower half of a warp adds up a, the upper half b, and after the barrier everybody
// adds up the warps' sums.
__device__ __forceinline__ void reduce_two_sums(int warps, float& a, float& b, float2 (&scratch)[16]) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const bool upper = lane >= 16;
    float x = upper ? b : a;
    x += __shfl_xor_sync(kFullMask, upper ? a : b, 16);
#pragma unroll
    for (int d = 8; d; d >>= 1) x += __shfl_xor_sync(kFullMask, x, d);
    if (warps == 1) {
        a = __shfl_sync(kFullMask, x, 0);
        b = __shfl_sync(kFullMask, x, 16);
        return;
    }
    if (lane == 0) scratch[warp].x = x;
    if (lane == 16) scratch[warp].y = x;
    if (warp == 0 && lane >= warps && lane < 16) scratch[lane] = make_float2(0.0f, 0.0f);
    __syncthreads();
    a = b = 0.0f;
    const float4* two = reinterpret_cast<const float4*>(scratch);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (2 * i >= warps) break;
        const float4 v = two[i];
        a += v.x + v.z, b += v.y + v.w;
    }
}

// ---- quantisation -------------------------------------------------------------------------------------------------
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

// 1 / (1 + exp(-g)), off by a relative (2 |g| + 12) * 2^-24 at most: -g log2(e) is rounded before its power of two is taken, which is
// a relative error of |g| * 2^-24, and the constant's rounding another; the rest are the approximations and the sum.  That is under 2^-16,
// far below what bf16 or 8 bits resolve.  Below g = -87.3, where 1 + exp(-g) passes 2^126, it is 0 (the sigmoid is under 2^-125 there).
__device__ __forceinline__ float sigmoid(float g) {
    float e, s;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(g * -1.4426950408889634f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s) : "f"(1.0f + e));
    return s;
}

// The factor that turns v into steps of the row, and the step itself.
struct RowScale {
    float pre, inv, scale;
};
__device__ __forceinline__ RowScale row_scale(uint32_t top_bits, float factor) {
    RowScale s{1.0f, 0.0f, 0.0f};
    const float top = __uint_as_float(top_bits);
    if (top_bits >= kInfBits) {
        s.scale = __uint_as_float(kNanBits);
    } else if (top_bits) {
        // 127 / top is out of range for a tiny top: the row is brought up by a power of two first (exact)
        if (top < 0x1p-100f) s.pre = 0x1p100f;
        s.inv = 127.0f / (top * s.pre);
        s.scale = top * factor / 127.0f;
        if (__float_as_uint(s.scale) >= kInfBits) s.scale = __uint_as_float(kNanBits), s.inv = 0.0f;
    }
    return s;
}

// v * inv is rounded to a whole number by adding 1.5 * 2^23 in one fused step: the sum's low byte is the number in two's
// complement (|v * inv| stays below 127.5).  A row without a finite non-zero step gets zeros.
template <bool VEC>
__device__ __forceinline__ void store_quantized(const QuantArgs& a, int64_t r, int c, float (&v)[8], const RowScale& s) {
    constexpr float kRound = 12582912.0f;
    uint32_t b[8];
    if (s.inv == 0.0f) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = 0.0f;
    }
    if (s.pre != 1.0f) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= s.pre;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) b[e] = __float_as_uint(fmaf(v[e], s.inv, kRound));
    store8_bytes<VEC>(a.q + r * a.ldq, c, (int)a.cols, b);
    if (a.values) {
        float z[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = (__uint_as_float(b[e]) - kRound) * s.scale;
        store8<VEC>(a.values + r * a.ldv, c, (int)a.cols, z);
    }
}

// Quantisation, of a matrix (OP rows), of h * weight behind the norm, or of silu(gate) * up.  Bound by memory where rows start on 16
// bytes: one pass, nothing but its inputs and outputs crosses HBM.  Measured (bf16, us; bandwidth of the bytes the call cannot do
// without): norm 16384 x 8192 with h written 180.5 (6.7 TB/s, as a plain copy); gate 8192 x 14336 124 (6.6 TB/s, gate and up read as
// the halves of one matrix; 130 and more after some tens of milliseconds under load); rows 14336 x 4096 45.  Other rows are bound by the
// load/store unit, which takes an element a lane: fp32 rows 2741 x 5003 19.2 (floor 14.7), bf16 rows 14336 x 4099 61 (45), gate 8192 x 5003
// 65 (44), norm 4096 x 4099 42 (23).  One token is bound by the latency of one block: norm 1 x 4096 2.4, gate 1 x 14336 3.6.
// blockDim: (32 * warps of a team, teams); more than one team only of one warp
template <int OP, int DT, bool VEC, int NV>
__global__ void __launch_bounds__(32 * quantize_warps(NV)) k_rows_quantize(const QuantArgs a) {
    chain_go();
    chain_wait();
    typedef typename Store<DT>::type T;
    __shared__ uint32_t s_scratch[64];
    const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5;
    const int64_t r = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    if (r >= a.rows) return;  // (a whole team)
    const int cols = (int)a.cols;
    auto column = [&](int j) { return first_column<VEC>(j, warps, warp); };
    const T* x = static_cast<const T*>(a.x) + r * a.ldx;
    const T* x2 = static_cast<const T*>(a.x2) + r * a.ldx2;
    T* h = static_cast<T*>(a.h) + r * a.ldh;
    constexpr int kHeld = NV ? NV : 1;
    float v[kHeld][8], sum = 0.0f;
    uint32_t top = 0;
    const bool two = OP == kGate || (OP == kNorm && a.x2);
    auto fetch = [&](int c, Raw<VEC, T>& p, Raw<VEC, T>& p2) {
        p.fetch(x, c, cols);
        if (two) p2.fetch(x2, c, cols);
    };
    // x + residual, or silu(gate) * up
    auto get = [&](const Raw<VEC, T>& p, const Raw<VEC, T>& p2, float (&o)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            o[e] = p.get(e);
            if (OP == kGate) o[e] = o[e] * sigmoid(o[e]) * p2.get(e);
            if (OP == kNorm && two) o[e] += p2.get(e);
            if (OP == kNorm) sum = fmaf(o[e], o[e], sum);
        }
    };
    auto weigh = [&](int c, float (&p)[8]) {
        if (OP == kNorm && a.weight) {
            float w[8];
            load8<VEC>(a.weight, c, cols, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) p[e] *= w[e];
        }
    };
    auto largest = [&](const float (&p)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(fabsf(p[e])));
    };
    if constexpr (NV != 0) {
        Raw<VEC, T> p[kHeld], p2[kHeld];
#pragma unroll
        for (int j = 0; j < kHeld; ++j) fetch(column(j), p[j], p2[j]);
#pragma unroll
        for (int j = 0; j < kHeld; ++j) get(p[j], p2[j], v[j]);
        if (OP == kNorm && a.h) {
#pragma unroll
            for (int j = 0; j < kHeld; ++j) store8<VEC>(h, column(j), cols, v[j]);
        }
#pragma unroll
        for (int j = 0; j < kHeld; ++j) weigh(column(j), v[j]), largest(v[j]);
    } else {
        for (int j = 0; column(j) < cols; ++j) {
            Raw<VEC, T> p, p2;
            fetch(column(j), p, p2);
            get(p, p2, v[0]);
            weigh(column(j), v[0]);
            largest(v[0]);
        }
        __syncwarp();
    }
    reduce_sum_max<OP == kNorm>(warps, sum, top, s_scratch);
    float factor = 1.0f;
    if (OP == kNorm) {
        factor = rsqrtf(sum / (float)cols + a.eps);
        if (__float_as_uint(sum) >= kInfBits) top = kInfBits;
    }
    const RowScale s = row_scale(top, factor);
    if (threadIdx.x == 0) a.scale[r] = s.scale;
    if constexpr (NV != 0) {
#pragma unroll
        for (int j = 0; j < kHeld; ++j) store_quantized<VEC>(a, r, column(j), v[j], s);
    } else {
        // the second walk; h is stored only now, since it may be x or the residual itself
        for (int j = 0; column(j) < cols; ++j) {
            Raw<VEC, T> p, p2;
            fetch(column(j), p, p2);
            get(p, p2, v[0]);
            if (OP == kNorm && a.h) store8<VEC>(h, column(j), cols, v[0]);
            weigh(column(j), v[0]);
            store_quantized<VEC>(a, r, column(j), v[0], s);
        }
    }
}

// How a row is laid over a team: NV pieces a warp, `warps` of them, `teams` a block.  nv = 0: longer than max_warps hold.
struct Shape {
    int nv, warps, teams;
};
Shape row_shape(int64_t cols, int nv, int max_warps) {
    Shape s{nv, (int)((cols + 256 * nv - 1) / (256 * nv)), 1};
    if (s.warps > max_warps) return Shape{0, max_warps, 1};
    if (s.warps == 1) s.teams = kBlockWarps;
    return s;
}

template <int OP, int DT, bool VEC>
bool launch_quantize(const QuantArgs& a, int n_sm, cudaStream_t st) {
    // few rows, or short ones: as many warps as a row feeds; else more bytes in flight a lane
    Shape s{0, 0, 0};
    for (int nv = a.rows <= n_sm || a.cols <= 256 ? 1 : a.cols <= 512 ? 2 : 4; nv <= 4 && s.nv == 0; nv *= 2) s = row_shape(a.cols, nv, quantize_warps(nv));
    if (s.nv == 0) s.warps = quantize_warps(0);
    const dim3 block(32 * s.warps, s.teams);
    const unsigned grid = (unsigned)((a.rows + s.teams - 1) / s.teams);
    const auto kernel = s.nv == 0   ? k_rows_quantize<OP, DT, VEC, 0>
                        : s.nv == 1 ? k_rows_quantize<OP, DT, VEC, 1>
                        : s.nv == 2 ? k_rows_quantize<OP, DT, VEC, 2>
                                    : k_rows_quantize<OP, DT, VEC, 4>;
    return launch_chained(kernel, grid, block, 0, st, 1, a);
}

// ---- gradients -------------------------------------------------------------------------------------------------
// fp32 values from one team's slice of partial sums to the next: slices start on 16 bytes
__host__ __device__ inline int64_t slice_stride(int64_t cols) { return (cols + 3) / 4 * 4; }

struct NormBackArgs {
    const void *dy, *h, *dh;  // dh nullable
    const float* weight;      // nullable
    void* dx;
    float* part;              // [blocks][slice_stride(cols)] partial sums of dweight (nullable)
    int64_t lddy, ldh, lddh, lddx, rows, cols;
    float eps;
};

// A row in a stage of shared memory.  Its bytes keep their place within 16, so that it can be copied in whole 16-byte pieces:
// the first may begin before the row (still in the row's allocation, which starts on 16 bytes), the last is cut at its end.
template <typename T>
__device__ __forceinline__ int row_shift(const T* row) { return (int)((reinterpret_cast<uintptr_t>(row) / sizeof(T)) & (16 / sizeof(T) - 1)); }

// Copies 16 bytes, or the `bytes` that are left of a row and zeros behind them; nothing where none is left.
__device__ __forceinline__ void copy16(uint32_t to, const void* from, int bytes) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.gt.s32 p, %2, 0;\n\t@p cp.async.cg.shared.global [%0], [%1], 16, %3;\n\t}" ::"r"(to), "l"(from), "r"(bytes),
                 "r"(min(16, bytes))
                 : "memory");
}
// One matrix on its way into the stages: this thread's pieces.  VEC: those of its own columns, so that no other thread waits for
// them; else every blockDim.x-th piece of the row's span, which is up to one longer than the team has places for.
template <bool VEC, int NV, typename T>
struct Copier {
    static constexpr int kEach = NV * (int)sizeof(T) / 2;
    const char* row;  // of the next copy; VEC: from this thread's first column on
    int64_t step;     // bytes from row to row
    __device__ __forceinline__ void init(const void* m, int64_t ld, int64_t r, int64_t teams, int lead) {
        row = static_cast<const char*>(m) + (r * ld + (VEC ? 8 * (int)threadIdx.x - lead : 0)) * (int64_t)sizeof(T);
        step = teams * ld * (int64_t)sizeof(T);
    }
    __device__ __forceinline__ void next(uint32_t stage, int cols) {
        const int t = threadIdx.x, threads = blockDim.x;
        if constexpr (VEC) {
            constexpr int kSpan = 8 * sizeof(T);
            const uint32_t to = stage + t * kSpan;
            const int left = (cols - 8 * t) * (int)sizeof(T);
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                const int at = j / (kSpan / 16) * threads * kSpan + j % (kSpan / 16) * 16;
                copy16(to + at, row + at, left - at);
            }
        } else {
            const int lead = (int)(reinterpret_cast<uintptr_t>(row) & 15), bytes = lead + cols * (int)sizeof(T);
            const char* from = row - lead + 16 * t;
            const uint32_t to = stage + 16 * t;
#pragma unroll
            for (int j = 0; j < kEach; ++j)
                copy16(to + 16 * j * threads, from + 16 * j * threads, bytes - 16 * (t + j * threads));
            const int more = kEach * threads * 16;
            if (t == 0) copy16(to + more, from + more, bytes - more);
        }
        row += step;
    }
};

// A lane's columns c, c + step, ... of a staged row; those past its end as 0.
template <bool VEC, typename T>
__device__ __forceinline__ void staged8(const T* row, const unsigned char* stage, int c, int cols, float (&v)[8]) {
    const T* p = reinterpret_cast<const T*>(stage) + (VEC ? 0 : row_shift(row)) + c;
    if constexpr (VEC && sizeof(T) == 2) {
        uint4 a = make_uint4(0, 0, 0, 0);
        if (c < cols) a = *reinterpret_cast<const uint4*>(p);  // (past the end the copy left zeros)
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
    } else if constexpr (VEC) {
        float4 a = make_float4(0, 0, 0, 0), b = a;
        if (c < cols) a = *reinterpret_cast<const float4*>(p);
        if (c + 4 < cols) b = *reinterpret_cast<const float4*>(p + 4);
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    } else {
        T x[8];
        if (piece_inside<false>(c, cols)) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = p[32 * e];
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = c + 32 * e < cols ? p[32 * e] : T(0);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if constexpr (sizeof(T) == 4) v[e] = x[e];
            else v[e] = __uint_as_float((uint32_t)x[e] << 16);
        }
    }
}

// Columns of the norm's gradient in VEC with LEAD: they count from the 16 bytes in which the team's rows begin, `lead` elements before them,
// the same in all of its rows and all matrices; so every access but a row's first and last is a vector wherever rows start.
// (Without LEAD the lead is 0 at compile time: as a variable it cost rows on 16 bytes a third, 8192 x 8192 99.6 -> 133 us.)
__device__ __forceinline__ void load8_from(const float* row, int lead, int c, int end, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = c + e >= lead && c + e < end ? row[c + e - lead] : 0.0f;
}
template <typename T>
__device__ __forceinline__ void store8_from(T* row, int lead, int c, int end, const float (&v)[8]) {
    if (c >= lead) return store8<true>(row - lead, c, end, v);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e >= lead && e < end) narrow(v[e], row[e - lead]);
}

// 1 / sqrt(mean(h^2) + eps) of a row whose squares add up to sq.  Past fp32's range it is NaN (sq - sq): the norm gives such a row
// up, like one with an Inf, and a root of 0 would pass for a gradient.  (As a selection behind the root this cost up to 3 %,
// 8192 x 4099 started differently 83.5 -> 86.3 us; in front of it nothing.)
__device__ __forceinline__ float inverse_root(float sq, float inv_n, float eps) {
    return rsqrtf(fmaf(sq, inv_n, eps + (sq - sq)));
}

// A team takes rows in steps of the number of teams.  Its rows pass through `stages` stages of shared memory that asynchronous
// copies fill ahead, so that what is in flight does not depend on where the team stands between its barriers.  A lane keeps its
// columns, so the weights and the partial sums of dweight stay in registers, NV pieces of 8.  blockDim: (32 * warps, teams), more
// than one team only of one warp.
//   With n = h r, r = 1 / sqrt(mean(h^2) + eps) and s = mean(dy weight n):  dx = r (dy weight - n s) + dh,  dweight = sum dy n.
// Both sums of a row go through one reduction, so a row costs one pass and one barrier.  Bound by memory where rows start on 16
// bytes: bf16 8192 x 4096 47.2 us (floor 41), 8192 x 8192 87.3 (82), 4096 x 14336 82.5 (72), fp32 8192 x 4096 94 (82); what is left is the partial sums' way
// and the last rows of the teams.  The same with LEAD, whose teams are fewer warps with more columns: 8192 x 4099 61.8.  Rows that
// start differently in different matrices are read from shared memory an element a lane, and stored so: bound by instructions and the
// load/store unit, 8192 x 4099 84.5.
template <int DT, bool VEC, bool LEAD, int NV>
__global__ void __launch_bounds__(NV == 4 ? 512 : NV == 2 ? 288 : 256, NV == 4 ? 1 : 2) k_norm_backward(const NormBackArgs a, int stages, uint32_t row_bytes) {
    chain_go();
    chain_wait();
    typedef typename Store<DT>::type T;
    extern __shared__ __align__(16) unsigned char s_rows[];  // [teams of the block][stages][3][row_bytes]
    __shared__ __align__(16) float2 s_scratch[2][16];
    const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5;
    const int cols = (int)a.cols;
    const int64_t me = (int64_t)blockIdx.x * blockDim.y + threadIdx.y, teams = (int64_t)gridDim.x * blockDim.y;
    const float inv_n = 1.0f / (float)cols;
    constexpr bool kHold = NV == 1;  // a row's values stay in registers over the reduction (NV > 1: they would spill)
    auto column = [&](int j) { return first_column<VEC>(j, warps, warp); };
    const uint32_t stage_bytes = 3 * row_bytes;
    unsigned char* const first = s_rows + threadIdx.y * stages * stage_bytes;
    unsigned char* const last = first + (stages - 1) * stage_bytes;
    const int lead = LEAD ? row_shift(static_cast<const T*>(a.h) + me * a.ldh) : 0, end = cols + lead;
    Copier<VEC, NV, T> copy_h, copy_dy, copy_dh;
    copy_h.init(a.h, a.ldh, me, teams, lead);
    copy_dy.init(a.dy, a.lddy, me, teams, lead);
    copy_dh.init(a.dh, a.lddh, me, teams, lead);
    auto copy = [&](unsigned char* stage, bool there) {
        const uint32_t to = (uint32_t)__cvta_generic_to_shared(stage);
        if (there) {
            copy_h.next(to, end);
            copy_dy.next(to + row_bytes, end);
            if (a.dh) copy_dh.next(to + 2 * row_bytes, end);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    for (int s = 0; s < stages - 1; ++s) copy(first + s * stage_bytes, me + s * teams < a.rows);
    float w[NV][8], sum[NV][8];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
#pragma unroll
        for (int e = 0; e < 8; ++e) w[j][e] = 1.0f, sum[j][e] = 0.0f;
        if (a.weight) {
            if constexpr (LEAD) load8_from(a.weight, lead, column(j), end, w[j]);
            else load8<VEC>(a.weight, column(j), cols, w[j]);
        }
    }
    // where rows start within 16 bytes (VEC: the lead)
    const T* h = static_cast<const T*>(a.h) + me * a.ldh;
    const T* dy = static_cast<const T*>(a.dy) + me * a.lddy;
    const T* dh = static_cast<const T*>(a.dh) + me * a.lddh;
    T* dx = static_cast<T*>(a.dx) + me * a.lddx;
    const int64_t step_h = teams * a.ldh, step_dy = teams * a.lddy, step_dh = teams * a.lddh, step_dx = teams * a.lddx;
    int side = 0;
    unsigned char* stage = first;
    for (int64_t r = me, ahead = me + (stages - 1) * teams; r < a.rows; r += teams, ahead += teams, side ^= 1) {
        // the row is there: this thread's copies and, past the barrier, everybody's; past it the stage before is free, too.  (VEC: a
        // thread reads what it copied itself, and needs neither.)
        if (stages == 2) asm volatile("cp.async.wait_group 0;" ::: "memory");
        else asm volatile("cp.async.wait_group 1;" ::: "memory");
        if constexpr (!VEC) {
            if (warps == 1) __syncwarp();
            else __syncthreads();
        }
        copy(stage == first ? last : stage - stage_bytes, ahead < a.rows);
        float hv[kHold ? NV : 1][8], gv[kHold ? NV : 1][8], sq = 0.0f, along = 0.0f;
        auto get = [&](int j) {
            const int i = kHold ? j : 0;
            staged8<VEC>(h, stage, column(j), end, hv[i]);
            staged8<VEC>(dy, stage + row_bytes, column(j), end, gv[i]);
            if (LEAD && j == 0 && column(0) < lead) {  // what stands before the row
#pragma unroll
                for (int e = 0; e < 7; ++e)
                    if (e < lead) hv[i][e] = 0.0f, gv[i][e] = 0.0f;
            }
        };
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            get(j);
            const int i = kHold ? j : 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) sq = fmaf(hv[i][e], hv[i][e], sq), along = fmaf(gv[i][e] * w[j][e], hv[i][e], along);
        }
        // (two buffers: the barrier of a row frees the buffer of the row before)
        reduce_two_sums(warps, sq, along, s_scratch[side]);
        const float root = inverse_root(sq, inv_n, a.eps);
        const float coef = along * root * inv_n * root;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int i = kHold ? j : 0;
            float o[8];
            if (!kHold) get(j);
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = 0.0f;
            if (a.dh) staged8<VEC>(dh, stage + 2 * row_bytes, column(j), end, o);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float g = gv[i][e] * root;
                o[e] = fmaf(g, w[j][e], fmaf(-coef * root, hv[i][e], o[e]));
                sum[j][e] = fmaf(g, hv[i][e], sum[j][e]);
            }
            if (LEAD && j == 0) store8_from(dx, lead, column(0), end, o);
            else store8<VEC>(dx - lead, column(j), end, o);
        }
        dx += step_dx;
        if constexpr (!VEC) h += step_h, dy += step_dy, dh += step_dh;
        stage = stage == last ? first : stage + stage_bytes;
    }
    if (!a.part) return;
    if constexpr (NV == 1) {
        // teams of one warp: the block's are added up here
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncthreads();
        float* all = reinterpret_cast<float*>(s_rows) + threadIdx.y * 256;
        const int lane = threadIdx.x;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int at = (VEC ? 8 * lane - lead : lane) + kStep<VEC> * e;
            if (at >= 0) all[at] = sum[0][e];
        }
        __syncthreads();
        const int c = threadIdx.y * 32 + lane;
        float total = 0.0f;
        for (int i = 0; i < (int)blockDim.y; ++i) total += reinterpret_cast<const float*>(s_rows)[i * 256 + c];
        if (c < cols) a.part[blockIdx.x * slice_stride(a.cols) + c] = total;
    } else {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float* part = a.part + me * slice_stride(a.cols);
            if constexpr (!LEAD) {
                store8<VEC>(part, column(j), cols, sum[j]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (column(j) + e >= lead && column(j) + e < end) part[column(j) + e - lead] = sum[j][e];
            }
        }
    }
}

// The same for rows of which two stages of three matrices do not fit in shared memory (fp32 from about 8530 columns on), or whose columns do
// not fit in a team's registers (16384): walked twice, the partial sums in the team's slice of the workspace.  Bound by that second
// walk and by the sums' way (a read and a write an element), and so 2.5 to 2.8 times the floor: fp32 4096 x 12288 310 us (floor 123),
// 4096 x 14336 389 (144), 1024 x 40000 280 (100).
template <int DT, bool VEC>
__global__ void __launch_bounds__(512) k_norm_backward_long(const NormBackArgs a) {
    chain_go();
    chain_wait();
    typedef typename Store<DT>::type T;
    __shared__ __align__(16) float2 s_scratch[2][16];
    const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5;
    const int cols = (int)a.cols;
    float* part = a.part ? a.part + blockIdx.x * slice_stride(a.cols) : nullptr;
    const float inv_n = 1.0f / (float)cols;
    auto column = [&](int j) { return first_column<VEC>(j, warps, warp); };
    int side = 0;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x, side ^= 1) {
        const T* hr = static_cast<const T*>(a.h) + r * a.ldh;
        const T* dyr = static_cast<const T*>(a.dy) + r * a.lddy;
        float sq = 0.0f, along = 0.0f, w[8];
        Raw<VEC, T> h, dy, dh;
        auto weights = [&](int c) {
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = 1.0f;
            if (a.weight) load8<VEC>(a.weight, c, cols, w);
        };
        for (int j = 0; column(j) < cols; ++j) {
            h.fetch(hr, column(j), cols);
            dy.fetch(dyr, column(j), cols);
            weights(column(j));
#pragma unroll
            for (int e = 0; e < 8; ++e) sq = fmaf(h.get(e), h.get(e), sq), along = fmaf(dy.get(e) * w[e], h.get(e), along);
        }
        __syncwarp();
        reduce_two_sums(warps, sq, along, s_scratch[side]);
        const float root = inverse_root(sq, inv_n, a.eps);
        const float coef = along * root * inv_n;
        for (int j = 0; column(j) < cols; ++j) {
            const int c = column(j);
            float o[8], sum[8];
            h.fetch(hr, c, cols);
            dy.fetch(dyr, c, cols);
            if (a.dh) dh.fetch(static_cast<const T*>(a.dh) + r * a.lddh, c, cols);
            weights(c);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] = 0.0f;
            if (part && r != blockIdx.x) load8<VEC>(part, c, cols, sum);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float unit = h.get(e) * root, g = dy.get(e);
                o[e] = fmaf(root, fmaf(g, w[e], -unit * coef), a.dh ? dh.get(e) : 0.0f);
                sum[e] = fmaf(g, unit, sum[e]);
            }
            store8<VEC>(static_cast<T*>(a.dx) + r * a.lddx, c, cols, o);
            if (part) store8<VEC>(part, c, cols, sum);
        }
    }
}

// dweight[c] = sum of the teams' partial sums in a fixed order: 8 columns (a sector) by 32 or 128 runs of teams a block.
// Bound by latency, so a thread has about ten loads, eight on their way together; narrow rows have many teams, hence the 128:
// 1328 slices of 1003 columns in 32 runs 19.7 us (cold), in 128 5.9 (gradient of 16384 rows 47.0 -> 36.4).
// With up to 320 slices 32 runs are the better: the gradient of 8192 x 4096, 296 slices, 46.9 us against 49.5 with 128.
constexpr int kSumRuns = 128;
__global__ void __launch_bounds__(8 * kSumRuns) k_norm_weight_sum(const float* part, int64_t teams, int64_t cols, float* dweight) {
    chain_go();
    chain_wait();
    __shared__ float s[kSumRuns][9];
    const int64_t c0 = (int64_t)blockIdx.x * 8;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = threadIdx.x & 7, run = threadIdx.x >> 3, runs = blockDim.x >> 3;
    float sum = 0.0f;
    if (c0 + col < cols) {
#pragma unroll 8
        for (int64_t g = run; g < teams; g += runs) sum += part[g * slice_stride(cols) + c0 + col];
    }
    s[run][col] = sum;
    __syncthreads();
    if (warp < 8 && c0 + warp < cols) {
        float all = s[lane][warp];
        for (int i = lane + 32; i < runs; i += 32) all += s[i][warp];
#pragma unroll
        for (int d = 16; d; d >>= 1) all += __shfl_xor_sync(kFullMask, all, d);
        if (lane == 0) dweight[c0 + warp] = all;
    }
}

struct GateBackArgs {
    const void *dy, *gate, *up;
    void *dgate, *dup;
    int64_t lddy, ldg, ldu, lddg, lddu, rows, cols;
};

// The gated activation's gradient, with g = gate, u = up and p = 1 / (1 + exp(-g)):
//   dup = dy g p,  dgate = dy u p (1 + g (1 - p)).
// Element by element, no reduction: bound by memory where rows start on 16 bytes (bf16 4096 x 11008 69.3 us, at its floor of 68.9),
// else by the load/store unit, about 4 clocks for each of the 64-byte accesses of a warp (4096 x 11003 96).
// blockIdx.x: rows, by teams of a block; blockIdx.y: pieces of a row, by warps of a team.
template <int DT, bool VEC>
__global__ void __launch_bounds__(32 * kBlockWarps) k_gate_backward(const GateBackArgs a) {
    chain_go();
    chain_wait();
    typedef typename Store<DT>::type T;
    const int cols = (int)a.cols, warps = blockDim.x >> 5, warp = threadIdx.x >> 5;
    for (int64_t r = (int64_t)blockIdx.x * blockDim.y + threadIdx.y; r < a.rows; r += (int64_t)gridDim.x * blockDim.y) {
        for (int j = blockIdx.y;; j += gridDim.y) {
            const int c = first_column<VEC>(j, warps, warp);
            if ((j * warps + warp) * 256 >= cols) break;
            Raw<VEC, T> d, g, u;
            d.fetch(static_cast<const T*>(a.dy) + r * a.lddy, c, cols);
            g.fetch(static_cast<const T*>(a.gate) + r * a.ldg, c, cols);
            u.fetch(static_cast<const T*>(a.up) + r * a.ldu, c, cols);
            float dg[8], du[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float x = g.get(e), s = sigmoid(x), ds = d.get(e) * s;
                dg[e] = ds * u.get(e) * fmaf(x, 1.0f - s, 1.0f);
                du[e] = ds * x;
            }
            store8<VEC>(static_cast<T*>(a.dgate) + r * a.lddg, c, cols, dg);
            store8<VEC>(static_cast<T*>(a.dup) + r * a.lddu, c, cols, du);
        }
    }
}

// ---- host side ---------------------------------------------------------------------------------------------------
constexpr int64_t kMaxRows = ((int64_t)1 << 31) - 1, kMaxCols = (int64_t)1 << 30;  // (columns, and those past the end, in 32 bits)

bool extent_ok(int64_t rows, int64_t cols) { return rows <= kMaxRows && cols <= kMaxCols; }
bool span_ok(int64_t rows, int64_t ld) { return rows == 0 || ld <= ((int64_t)1 << 60) / rows; }
bool matrix_arg_ok(const void* p, int64_t ld, int64_t cols, size_t align) { return p && reinterpret_cast<uintptr_t>(p) % align == 0 && ld >= cols; }
bool on_16(const void* p, int64_t ld, int64_t rows, size_t elem) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (rows <= 1 || ld * (int64_t)elem % 16 == 0);
}
size_t elem_bytes(int32_t dtype) { return dtype == DNNS_F32 ? 4 : 2; }

int sm_count() {
    int dev = 0, n = 0;
    if (!succeeded(cudaGetDevice(&dev)) || !succeeded(cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev))) return 0;
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
    if (a.cols == 0) return succeeded(cudaMemsetAsync(a.scale, 0, (size_t)a.rows * sizeof(float), st)) ? DNNS_OK : DNNS_ERR_CUDA;
    const int n_sm = sm_count();
    if (n_sm == 0) return DNNS_ERR_CUDA;
    const size_t e = elem_bytes(dtype);
    const bool vec = on_16(a.x, a.ldx, a.rows, e) && (!a.x2 || on_16(a.x2, a.ldx2, a.rows, e)) && (!a.h || on_16(a.h, a.ldh, a.rows, e)) &&
                     (!a.values || on_16(a.values, a.ldv, a.rows, 2)) && (!a.weight || on_16(a.weight, 0, 1, 4));
    const bool launched = dtype == DNNS_F32 ? (vec ? launch_quantize<OP, DNNS_F32, true>(a, n_sm, st) : launch_quantize<OP, DNNS_F32, false>(a, n_sm, st))
                                            : (vec ? launch_quantize<OP, DNNS_BF16, true>(a, n_sm, st) : launch_quantize<OP, DNNS_BF16, false>(a, n_sm, st));
    return launched ? DNNS_OK : DNNS_ERR_CUDA;
}

// Warps of a team of the norm's gradient: NV = 2 up to 4096 columns, 3 up to 6144, 4 above (fewer warps, but the weights and sums of 8
// more columns a lane in registers); 16 warps where 8 do not hold a row.
// (Widths that put rows off 16 bytes get room for what stands before a row.)
Shape norm_backward_shape(int64_t cols) {
    if (cols % 8) cols += 7;
    if (cols <= 256) return row_shape(cols, 1, 1);
    Shape s = row_shape(cols, cols <= 512 * backward_warps(2) ? 2 : cols <= 768 * backward_warps(3) ? 3 : 4, 16);
    s.teams = 1;
    return s;
}
// Blocks of an SM at most: 16 warps of 128 registers a thread.  NV = 2 is built for 96 and gets 18 warps (three teams of six, where 4096
// columns take two of eight); that spills 4 to 84 bytes a thread but for bf16 on 16 bytes.  The workspace is sized for that many, a slice a
// block; it is asked for without a device, so it and the grid count on a B200's SMs.
constexpr int kSms = 148;
int norm_backward_blocks(const Shape& s) { return std::max(1, (s.nv == 2 ? 18 : 16) / (s.warps * s.teams)); }
int64_t norm_backward_slices(int64_t rows, int64_t cols) {
    const Shape s = norm_backward_shape(cols);
    return std::min<int64_t>((rows + s.teams - 1) / s.teams, kSms * norm_backward_blocks(s));
}

template <int DT, bool VEC, bool LEAD>
auto norm_backward_kernel(int nv) {
    return nv == 1 ? k_norm_backward<DT, VEC, LEAD, 1> : nv == 2 ? k_norm_backward<DT, VEC, LEAD, 2> : nv == 3 ? k_norm_backward<DT, VEC, LEAD, 3> : k_norm_backward<DT, VEC, LEAD, 4>;
}

// Where rows start: all (and the weights) on 16 bytes; all matrices' the same way, row by row; anything else.
enum class Starts { kEven, kShared, kAny };
// Launches the gradient; how many slices of partial sums it writes, or -1.  Rows of a layer of any width, contiguous in all matrices,
// are the ordinary case of kShared: 8192 x 4099 takes 62 us with their vectors, 84.5 by elements at any place.
template <int DT>
int64_t launch_norm_backward(const NormBackArgs& a, Starts starts, cudaStream_t st) {
    static std::atomic<uint64_t> done[3][4];
    constexpr size_t kRoom = 200 * 1024;  // shared memory of an SM that the stages may take
    constexpr int kLead = DT == DNNS_F32 ? 3 : 7;
    const Shape s = norm_backward_shape(a.cols);
    const bool vec = starts == Starts::kEven || (starts == Starts::kShared && a.cols + kLead <= (int64_t)256 * s.nv * s.warps);
    const size_t row_bytes = ((size_t)a.cols * (DT == DNNS_F32 ? 4 : 2) + 15) / 16 * 16 + (starts == Starts::kEven ? 0 : 16), stage = 3 * row_bytes * s.teams;
    int blocks = norm_backward_blocks(s);
    // (two blocks of two stages rather than one of three: bf16 8192 x 8192 99.5 -> 87.4 us)
    while (blocks > 1 && kRoom / blocks < 2 * stage) --blocks;
    const int stages = (int)std::min<size_t>(3, kRoom / blocks / stage);
    if (s.nv == 0 || stages < 2) {
        const int64_t grid = std::min<int64_t>(a.rows, kSms);
        return launch_chained(starts == Starts::kEven ? k_norm_backward_long<DT, true> : k_norm_backward_long<DT, false>, (unsigned)grid, 512, 0, st, 1, a) ? grid : -1;
    }
    int64_t grid = std::min<int64_t>((a.rows + s.teams - 1) / s.teams, kSms * blocks);
    // a team's rows have one lead: it steps over a multiple of 8 rows
    if (vec && starts == Starts::kShared && grid * s.teams < a.rows) grid -= grid * s.teams % 8 / s.teams;
    const dim3 block(32 * s.warps, s.teams);
    const auto kernel = !vec ? norm_backward_kernel<DT, false, false>(s.nv) : starts == Starts::kEven ? norm_backward_kernel<DT, true, false>(s.nv) : norm_backward_kernel<DT, true, true>(s.nv);
    int dev = 0;
    if (!succeeded(cudaGetDevice(&dev)) || !allow_shared(kernel, kRoom, done[!vec ? 0 : starts == Starts::kEven ? 1 : 2][s.nv - 1], dev)) return -1;
    const size_t shared = std::max(stages * stage, s.nv == 1 ? (size_t)kBlockWarps * 256 * sizeof(float) : 0);
    return launch_chained(kernel, (unsigned)grid, block, shared, st, 1, a, stages, (uint32_t)row_bytes) ? grid : -1;
}

template <int DT, bool VEC>
bool launch_gate_backward(const GateBackArgs& a, cudaStream_t st) {
    Shape s = row_shape(a.cols, 1, kBlockWarps);
    const int rounds = (int)((a.cols + 256 * s.warps - 1) / (256 * s.warps));
    const dim3 grid((unsigned)std::min<int64_t>((a.rows + s.teams - 1) / s.teams, (int64_t)1 << 30), std::min(rounds, 65535));
    return launch_chained(k_gate_backward<DT, VEC>, grid, dim3(32 * s.warps, s.teams), 0, st, 1, a);
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
    return ((size_t)dnns::norm_backward_slices(rows, cols) * (size_t)dnns::slice_stride(cols) * sizeof(float) + 255) & ~(size_t)255;
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
        if (dweight && !succeeded(cudaMemsetAsync(dweight, 0, (size_t)cols * sizeof(float), st))) return DNNS_ERR_CUDA;
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
    auto like_h = [&](const void* p, int64_t ld) {
        return (reinterpret_cast<uintptr_t>(p) - reinterpret_cast<uintptr_t>(h)) % 16 == 0 && (rows <= 1 || (ld - ldh) * (int64_t)e % 16 == 0);
    };
    const Starts starts = !like_h(dy, lddy) || !like_h(dx, lddx) || (dh && !like_h(dh, lddh)) ? Starts::kAny : on_16(h, ldh, rows, e) && on_16(weight, 0, 1, 4) ? Starts::kEven : Starts::kShared;
    const int64_t slices = dtype == DNNS_F32 ? launch_norm_backward<DNNS_F32>(a, starts, st) : launch_norm_backward<DNNS_BF16>(a, starts, st);
    if (slices < 0) return DNNS_ERR_CUDA;
    if (dweight && !launch_chained(k_norm_weight_sum, (unsigned)((cols + 7) / 8), slices > 320 ? 8 * kSumRuns : 256, 0, st, 1, a.part, slices, cols, dweight)) return DNNS_ERR_CUDA;
    return DNNS_OK;
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
    const GateBackArgs a{dy, gate, up, dgate, dup, lddy, ldg, ldu, lddg, lddu, rows, cols};
    const bool vec = on_16(dy, lddy, rows, e) && on_16(gate, ldg, rows, e) && on_16(up, ldu, rows, e) && on_16(dgate, lddg, rows, e) &&
                     on_16(dup, lddu, rows, e);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool launched = dtype == DNNS_F32 ? (vec ? launch_gate_backward<DNNS_F32, true>(a, st) : launch_gate_backward<DNNS_F32, false>(a, st))
                                            : (vec ? launch_gate_backward<DNNS_BF16, true>(a, st) : launch_gate_backward<DNNS_BF16, false>(a, st));
    return launched ? DNNS_OK : DNNS_ERR_CUDA;
}

}  // extern "C"
