// Rows in 8 bits: quantisation of a matrix's rows, fused with what produces them in a language model's block - the
// root-mean-square norm with the residual's addition, and the gated activation - and the gradients of those two.
//   Q(y): a = max |y|, scale = a / 127, q = rint(y * 127 / a).
//
// All five are bound by memory: a few operations an element against 5 to 11 bytes of traffic.  So each row is read
// once and kept in registers (fp32) between the reduction that its scale needs and the stores.  For the norm the
// reduction is a single one, because q does not depend on the row's root mean square: with v = h * weight and
// r = 1 / sqrt(mean(h^2) + eps), q = rint(v * 127 / max|v|) and scale = r * max|v| / 127, so the sum of squares and the
// maximum travel through the same shuffles and the same barrier.
//
// A team of warps has a row (one warp for short rows, several teams a block).  A lane works on pieces of 8 neighbouring
// columns; NV pieces a lane, so a row of up to 8 * NV * lanes columns stays in registers, and longer ones (NV = 0) are walked
// twice.  Rows of a rebuilt layer have any width, so they start anywhere: SHIFT handles rows that do not start on 16 bytes
// with the same 16-byte accesses.  A lane then fetches the two aligned vectors around its piece and shifts its 8 columns
// out of them; it stores the aligned vector that ends inside its piece, whose front columns come from the lane before it
// by shuffles.  The first lane of a warp repeats the piece of the previous warp's last lane, so that every stored vector finds its
// front: 31 pieces a warp instead of 32.  Only the ends of a row go element by element.
#include <algorithm>

#include "dnns_internal.cuh"

namespace dnns {

namespace {

constexpr uint32_t kFullMask = 0xFFFFFFFFu;
constexpr uint32_t kInfBits = 0x7F800000u;
constexpr uint32_t kNanBits = 0x7FC00000u;
constexpr int kBlockWarps = 8;  // warps of a block whose teams are small
// Warps of a team at most, by pieces a lane: what keeps a row in registers without spilling.
constexpr int quantize_warps(int nv) { return nv == 4 ? 16 : 32; }
constexpr int backward_warps(int nv) { return nv == 2 ? 20 : 16; }

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

// ---- pieces of 8 columns -------------------------------------------------------------------------------------
// Where a lane's pieces are: team of `warps`, this one being number `warp`.
template <bool SHIFT>
struct Lanes {
    static constexpr int kPieces = SHIFT ? 31 : 32;  // of a warp
    int warps, warp, lane;
    __device__ __forceinline__ int column(int j) const { return 8 * ((j * warps + warp) * kPieces + lane - (SHIFT ? 1 : 0)); }
    // (SHIFT: lane 0's piece is the previous warp's; its values are counted there)
    __device__ __forceinline__ bool counted() const { return !SHIFT || lane != 0; }
};
// pieces of a row; SHIFT: one more, since the columns at the end may be stored by the lane after the last piece
template <bool SHIFT>
__host__ __device__ inline int row_pieces(int cols) { return (cols + 7) / 8 + (SHIFT ? 1 : 0); }

// Elements by which a row starts past a 16-byte boundary.
template <typename T>
__device__ __forceinline__ int row_shift(const T* row) { return (int)((reinterpret_cast<uintptr_t>(row) / sizeof(T)) & (16 / sizeof(T) - 1)); }

// Words s .. of a run of words: s in 16-bit steps below 8 (bf16), in words below 4 (fp32).
__device__ __forceinline__ void shift_out(const uint32_t (&w)[8], int s, uint32_t (&r)[4]) {
    uint32_t t[6], u[5];
#pragma unroll
    for (int i = 0; i < 6; ++i) t[i] = s & 4 ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i < 5; ++i) u[i] = s & 2 ? t[i + 1] : t[i];
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __funnelshift_r(u[i], u[i + 1], 16 * (s & 1));
}
__device__ __forceinline__ void shift_out(const uint32_t (&w)[12], int s, uint32_t (&r)[8]) {
    uint32_t t[9];
#pragma unroll
    for (int i = 0; i < 9; ++i) t[i] = s & 2 ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = s & 1 ? t[i + 1] : t[i];
}
__device__ __forceinline__ void widen8(const uint32_t (&w)[4], float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
}
__device__ __forceinline__ void widen8(const uint32_t (&w)[8], float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
}

// Columns c .. c + 7 of a row; those outside it read as 0.  In two steps, so that all of a lane's loads are on their way
// before the first of them is waited for: `fetch` issues the vector loads, predicated and without a branch, `get` shifts and
// widens what came, and reads element by element where a vector would have left the row.
template <bool SHIFT, typename T>
struct Piece {
    static constexpr int kPer = 16 / sizeof(T), kWords = 2 * sizeof(T);  // elements of a vector, words of a piece
    uint32_t w[kWords + (SHIFT ? 4 : 0)];
    static __device__ __forceinline__ bool whole(int c, int cols, int s) { return c >= s && c + 8 + (SHIFT && s ? kPer - s : 0) <= cols; }
    __device__ __forceinline__ void fetch(const T* row, int c, int cols) {
        const int s = SHIFT ? row_shift(row) : 0;
        const bool in = whole(c, cols, s);
        const T* p = row + (c - s);
#pragma unroll
        for (int i = 0; i < kWords / 4 + (SHIFT ? 1 : 0); ++i) {
            const bool need = in && (i < kWords / 4 || s);
            w[4 * i] = w[4 * i + 1] = w[4 * i + 2] = w[4 * i + 3] = 0;
            asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %5, 0;\n\t@p ld.global.v4.u32 {%0, %1, %2, %3}, [%4];\n\t}"
                         : "+r"(w[4 * i]), "+r"(w[4 * i + 1]), "+r"(w[4 * i + 2]), "+r"(w[4 * i + 3])
                         : "l"(p + i * kPer), "r"((uint32_t)need)
                         : "memory");
        }
    }
    __device__ __forceinline__ void get(const T* row, int c, int cols, float (&v)[8]) const {
        const int s = SHIFT ? row_shift(row) : 0;
        if constexpr (SHIFT) {
            uint32_t r[kWords];
            shift_out(w, s, r);
            widen8(r, v);
        } else {
            widen8(w, v);
        }
        if (!whole(c, cols, s) && c + 8 > 0 && c < cols) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (c + e >= 0 && c + e < cols) v[e] = widen(row[c + e]);
        }
    }
};
template <bool SHIFT, typename T>
__device__ __forceinline__ void load8(const T* row, int c, int cols, float (&v)[8]) {
    Piece<SHIFT, T> p;
    p.fetch(row, c, cols);
    p.get(row, c, cols, v);
}

// Stores columns c .. c + 7.  All lanes of the warp take part (SHIFT: a lane may store columns of the lane before it).
template <bool SHIFT, typename T>
__device__ __forceinline__ void store8(T* row, int c, int cols, const float (&v)[8]) {
    constexpr int kPer = 16 / sizeof(T), kWords = 2 * sizeof(T);
    uint32_t w[kWords + 4];  // behind the 4 words (SHIFT) of the lane before
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[4 + i] = __float_as_uint(v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[4 + i] = bf16_pair(v[2 * i], v[2 * i + 1]);
    }
    const int s = SHIFT ? row_shift(row) : 0;
    if (s == 0) {
        if (SHIFT && (threadIdx.x & 31) == 0) return;  // the previous warp's
        if (c >= 0 && c + 8 <= cols) {
#pragma unroll
            for (int i = 0; i < kWords / 4; ++i) *reinterpret_cast<uint4*>(row + c + i * kPer) = make_uint4(w[4 + 4 * i], w[5 + 4 * i], w[6 + 4 * i], w[7 + 4 * i]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (c + e >= 0 && c + e < cols) narrow(v[e], row[c + e]);
        }
        return;
    }
    if constexpr (SHIFT) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __shfl_up_sync(kFullMask, w[kWords + i], 1);
        if ((threadIdx.x & 31) == 0) return;
        uint32_t r[kWords];
        shift_out(w, kPer - s, r);  // columns c - s ..
        c -= s;
        if (c >= 0 && c + 8 <= cols) {
#pragma unroll
            for (int i = 0; i < kWords / 4; ++i) *reinterpret_cast<uint4*>(row + c + i * kPer) = make_uint4(r[4 * i], r[4 * i + 1], r[4 * i + 2], r[4 * i + 3]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (c + e >= 0 && c + e < cols) {
                    if constexpr (sizeof(T) == 4) row[c + e] = __uint_as_float(r[e]);
                    else row[c + e] = (uint16_t)(r[e / 2] >> (16 * (e & 1)));
                }
        }
    }
}

// Rows of q start on 16 bytes, so a piece is 8 bytes on a boundary of 8.
template <bool SHIFT>
__device__ __forceinline__ void store8_bytes(int8_t* row, int c, int cols, uint32_t lo, uint32_t hi) {
    if (SHIFT && (threadIdx.x & 31) == 0) return;
    if (c >= 0 && c + 8 <= cols) {
        *reinterpret_cast<uint2*>(row + c) = make_uint2(lo, hi);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (c + e >= 0 && c + e < cols) row[c + e] = (int8_t)((e < 4 ? lo : hi) >> (8 * (e & 3)));
    }
}

// ---- reductions over a team -------------------------------------------------------------------------------------
struct Team {
    int warps, warp, id;  // id: of the team in its block
    __device__ __forceinline__ void sync() const {
        if (warps > 1) asm volatile("bar.sync %0, %1;" ::"r"(id + 1), "r"(warps * 32) : "memory");
    }
};

// Sum of `a`, sum of `b` and maximum of `m` over a team.  `scratch`: 3 * 32 words of the team, free for another use
// after one more barrier.
template <bool A, bool B, bool M>
__device__ __forceinline__ void team_reduce(const Team& team, float& a, float& b, uint32_t& m, uint32_t* scratch) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int round = 0; round < 2; ++round) {
#pragma unroll
        for (int d = 16; d; d >>= 1) {
            if (A) a += __shfl_xor_sync(kFullMask, a, d);
            if (B) b += __shfl_xor_sync(kFullMask, b, d);
        }
        if (M) m = __reduce_max_sync(kFullMask, m);
        if (round || team.warps == 1) return;
        if (lane == 0) {
            if (A) scratch[team.warp] = __float_as_uint(a);
            if (B) scratch[32 + team.warp] = __float_as_uint(b);
            if (M) scratch[64 + team.warp] = m;
        }
        team.sync();
        const bool in = lane < team.warps;
        if (A) a = in ? __uint_as_float(scratch[lane]) : 0.0f;
        if (B) b = in ? __uint_as_float(scratch[32 + lane]) : 0.0f;
        if (M) m = in ? scratch[64 + lane] : 0u;
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

// 1 / (1 + exp(-g)) to a few units of the last place; the approximate quotient is 0 where 1 + exp(-g) passes 2^126, that is
// below g = -87.3, where the sigmoid is under 2^-125.
__device__ __forceinline__ float sigmoid(float g) { return __fdividef(1.0f, 1.0f + __expf(-g)); }

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
template <bool SHIFT>
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
    const uint32_t lo = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
    const uint32_t hi = __byte_perm(__byte_perm(b[4], b[5], 0x0040), __byte_perm(b[6], b[7], 0x0040), 0x5410);
    store8_bytes<SHIFT>(a.q + r * a.ldq, c, (int)a.cols, lo, hi);
    if (a.values) {
        float z[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = (__uint_as_float(b[e]) - kRound) * s.scale;
        store8<SHIFT>(a.values + r * a.ldv, c, (int)a.cols, z);
    }
}

// blockDim: (32 * warps of a team, teams)
template <int OP, int DT, bool SHIFT, int NV>
__global__ void __launch_bounds__(32 * quantize_warps(NV)) k_rows_quantize(const QuantArgs a) {
    typedef typename Store<DT>::type T;
    __shared__ uint32_t s_scratch[kBlockWarps][96];
    const Team team{(int)(blockDim.x >> 5), (int)(threadIdx.x >> 5), (int)threadIdx.y};
    const Lanes<SHIFT> at{team.warps, team.warp, (int)(threadIdx.x & 31)};
    const int64_t r = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    if (r >= a.rows) return;  // (a whole team)
    const int cols = (int)a.cols;
    const T* x = static_cast<const T*>(a.x) + r * a.ldx;
    const T* x2 = static_cast<const T*>(a.x2) + r * a.ldx2;
    T* h = static_cast<T*>(a.h) + r * a.ldh;
    constexpr int kHeld = NV ? NV : 1;
    const int rounds = (row_pieces<SHIFT>(cols) + team.warps * at.kPieces - 1) / (team.warps * at.kPieces);
    float v[kHeld][8], sum = 0.0f, unused = 0.0f;
    uint32_t top = 0;
    // a piece of x + residual, or of silu(gate) * up
    const bool two = OP == kGate || (OP == kNorm && a.x2);
    auto fetch = [&](int c, Piece<SHIFT, T>& p, Piece<SHIFT, T>& p2) {
        p.fetch(x, c, cols);
        if (two) p2.fetch(x2, c, cols);
    };
    auto get = [&](int c, const Piece<SHIFT, T>& p, const Piece<SHIFT, T>& p2, float (&o)[8]) {
        p.get(x, c, cols, o);
        if (two) {
            float u[8];
            p2.get(x2, c, cols, u);
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = OP == kGate ? o[e] * sigmoid(o[e]) * u[e] : o[e] + u[e];
        }
    };
    auto weigh = [&](int c, float (&p)[8]) {
        if (OP == kNorm && a.weight) {
            float w[8];
            load8<SHIFT>(a.weight, c, cols, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) p[e] *= w[e];
        }
    };
    auto squares = [&](const float (&p)[8]) {
        if (OP == kNorm && at.counted()) {
#pragma unroll
            for (int e = 0; e < 8; ++e) sum = fmaf(p[e], p[e], sum);
        }
    };
    auto largest = [&](const float (&p)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(fabsf(p[e])));
    };
    if constexpr (NV != 0) {
        Piece<SHIFT, T> p[kHeld], p2[kHeld];
#pragma unroll
        for (int j = 0; j < kHeld; ++j) fetch(at.column(j), p[j], p2[j]);
#pragma unroll
        for (int j = 0; j < kHeld; ++j) get(at.column(j), p[j], p2[j], v[j]), squares(v[j]);
        if (OP == kNorm && a.h) {
            // (SHIFT: a lane stores columns of the lane before it, which has fetched them first where h is x or the residual)
            if (SHIFT && (a.h == a.x || a.h == a.x2)) team.sync();
#pragma unroll
            for (int j = 0; j < kHeld; ++j) store8<SHIFT>(h, at.column(j), cols, v[j]);
        }
#pragma unroll
        for (int j = 0; j < kHeld; ++j) weigh(at.column(j), v[j]), largest(v[j]);
    } else {
        for (int j = 0; j < rounds; ++j) {
            Piece<SHIFT, T> p, p2;
            fetch(at.column(j), p, p2);
            get(at.column(j), p, p2, v[0]);
            squares(v[0]);
            weigh(at.column(j), v[0]);
            largest(v[0]);
        }
    }
    team_reduce<OP == kNorm, false, true>(team, sum, unused, top, s_scratch[team.id]);
    float factor = 1.0f;
    if (OP == kNorm) {
        factor = 1.0f / sqrtf(sum / (float)cols + a.eps);
        if (__float_as_uint(sum) >= kInfBits) top = kInfBits;
    }
    const RowScale s = row_scale(top, factor);
    if (threadIdx.x == 0) a.scale[r] = s.scale;
    if constexpr (NV != 0) {
#pragma unroll
        for (int j = 0; j < kHeld; ++j) store_quantized<SHIFT>(a, r, at.column(j), v[j], s);
    } else {
        // the second walk; h is stored only now, since it may be x or the residual itself.  (SHIFT: a lane stores columns of the lane
        // before it, so a round is stored when the whole team has fetched it and the next one.)
        Piece<SHIFT, T> p, p2;
        fetch(at.column(0), p, p2);
        get(at.column(0), p, p2, v[0]);
        for (int j = 0; j < rounds; ++j) {
            float next[8];
            if (j + 1 < rounds) {
                fetch(at.column(j + 1), p, p2);
                get(at.column(j + 1), p, p2, next);
            }
            if (OP == kNorm && a.h) {
                if (SHIFT) team.sync();
                store8<SHIFT>(h, at.column(j), cols, v[0]);
            }
            weigh(at.column(j), v[0]);
            store_quantized<SHIFT>(a, r, at.column(j), v[0], s);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[0][e] = next[e];
        }
    }
}

// How a row is laid over a team: NV pieces a lane, `warps` of them, `teams` a block.  nv = 0: longer than max_warps hold.
struct Shape {
    int nv, warps, teams;
};
Shape row_shape(int64_t cols, bool shift, int nv, int max_warps) {
    const int64_t lanes = shift ? 31 : 32, pieces = shift ? row_pieces<true>((int)cols) : row_pieces<false>((int)cols);
    Shape s{nv, (int)((pieces + lanes * nv - 1) / (lanes * nv)), 1};
    if (s.warps > max_warps) return Shape{0, 32, 1};
    if (s.warps <= kBlockWarps) s.teams = kBlockWarps / s.warps;
    return s;
}

template <int OP, int DT, bool SHIFT>
void launch_quantize(const QuantArgs& a, int n_sm, cudaStream_t st) {
    // few rows: as many lanes as a row feeds; many rows: more bytes in flight a lane
    Shape s{0, 0, 0};
    for (int nv = a.rows <= n_sm ? 1 : SHIFT ? 2 : 4; nv <= 4 && s.nv == 0; nv *= 2) s = row_shape(a.cols, SHIFT, nv, quantize_warps(nv));
    const dim3 block(32 * s.warps, s.teams);
    const unsigned grid = (unsigned)((a.rows + s.teams - 1) / s.teams);
    if (s.nv == 0) k_rows_quantize<OP, DT, SHIFT, 0><<<grid, block, 0, st>>>(a);
    else if (s.nv == 1) k_rows_quantize<OP, DT, SHIFT, 1><<<grid, block, 0, st>>>(a);
    else if (s.nv == 2) k_rows_quantize<OP, DT, SHIFT, 2><<<grid, block, 0, st>>>(a);
    else k_rows_quantize<OP, DT, SHIFT, 4><<<grid, block, 0, st>>>(a);
}

// ---- gradients -------------------------------------------------------------------------------------------------
struct NormBackArgs {
    const void *dy, *h, *dh;  // dh nullable
    const float* weight;      // nullable
    void* dx;
    float* part;              // [teams of the grid][cols] partial sums of dweight (nullable)
    int64_t lddy, ldh, lddh, lddx, rows, cols;
    float eps;
};

// A team takes rows in steps of the number of teams.  A lane keeps its columns, so the weights and the partial sums of
// dweight have a fixed place in shared memory (registers are what limits the rows in flight), NV pieces of two 16-byte
// vectors a lane; with NV = 0 the sums are in the team's slice of the workspace all along.
template <int DT, bool SHIFT, int NV>
__global__ void __launch_bounds__(32 * backward_warps(NV), NV == 1 ? 2 : 1) k_norm_backward(const NormBackArgs a) {
    typedef typename Store<DT>::type T;
    extern __shared__ float4 s_cols[];  // weights, then sums: [NV][2][threads of the block] each
    __shared__ uint32_t s_scratch[kBlockWarps][2][96];
    const Team team{(int)(blockDim.x >> 5), (int)(threadIdx.x >> 5), (int)threadIdx.y};
    const Lanes<SHIFT> at{team.warps, team.warp, (int)(threadIdx.x & 31)};
    const int cols = (int)a.cols;
    constexpr int kHeld = NV ? NV : 1;
    const int threads = blockDim.x * blockDim.y, self = threadIdx.y * blockDim.x + threadIdx.x;
    const int64_t me = (int64_t)blockIdx.x * blockDim.y + threadIdx.y, teams = (int64_t)gridDim.x * blockDim.y;
    if (me >= a.rows) return;  // (a whole team; it has no slice of the workspace)
    float* part = a.part ? a.part + me * a.cols : nullptr;
    const float inv_n = 1.0f / (float)cols;
    auto weights = [&](int c, float (&p)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = 1.0f;
        if (a.weight) load8<SHIFT>(a.weight, c, cols, p);
    };
    auto kept = [&](int which, int j, float (&p)[8]) {
        const float4 x = s_cols[((which * kHeld + j) * 2) * threads + self], y = s_cols[((which * kHeld + j) * 2 + 1) * threads + self];
        p[0] = x.x, p[1] = x.y, p[2] = x.z, p[3] = x.w, p[4] = y.x, p[5] = y.y, p[6] = y.z, p[7] = y.w;
    };
    auto keep = [&](int which, int j, const float (&p)[8]) {
        s_cols[((which * kHeld + j) * 2) * threads + self] = make_float4(p[0], p[1], p[2], p[3]);
        s_cols[((which * kHeld + j) * 2 + 1) * threads + self] = make_float4(p[4], p[5], p[6], p[7]);
    };
    auto give_part = [&](int c, const float (&p)[8]) {
        if (!at.counted()) return;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (c + e >= 0 && c + e < cols) part[c + e] = p[e];
    };
    if constexpr (NV != 0) {
#pragma unroll
        for (int j = 0; j < kHeld; ++j) {
            float p[8];
            weights(at.column(j), p);
            keep(0, j, p);
#pragma unroll
            for (int e = 0; e < 8; ++e) p[e] = 0.0f;
            keep(1, j, p);
        }
    }
    int side = 0;
    for (int64_t r = me; r < a.rows; r += teams, side ^= 1) {
        const T* dy = static_cast<const T*>(a.dy) + r * a.lddy;
        const T* h = static_cast<const T*>(a.h) + r * a.ldh;
        const T* dh = static_cast<const T*>(a.dh) + r * a.lddh;
        T* dx = static_cast<T*>(a.dx) + r * a.lddx;
        float hv[kHeld][8], gv[kHeld][8], pv[kHeld][8], w[8], sum[8];
        float sq = 0.0f, along = 0.0f;
        uint32_t unused = 0;
        auto fetch = [&](int c, Piece<SHIFT, T> (&p)[3]) {
            p[0].fetch(h, c, cols);
            p[1].fetch(dy, c, cols);
            if (a.dh) p[2].fetch(dh, c, cols);
        };
        auto get = [&](int c, const Piece<SHIFT, T> (&p)[3], float (&hp)[8], float (&gp)[8], float (&pp)[8]) {
            p[0].get(h, c, cols, hp);
            p[1].get(dy, c, cols, gp);
#pragma unroll
            for (int e = 0; e < 8; ++e) pp[e] = 0.0f;
            if (a.dh) p[2].get(dh, c, cols, pp);
        };
        auto sums = [&](const float (&hp)[8], const float (&gp)[8]) {
            if (!at.counted()) return;
#pragma unroll
            for (int e = 0; e < 8; ++e) sq = fmaf(hp[e], hp[e], sq), along = fmaf(gp[e] * w[e], hp[e], along);
        };
        if constexpr (NV != 0) {
            Piece<SHIFT, T> p[kHeld][3];
#pragma unroll
            for (int j = 0; j < kHeld; ++j) fetch(at.column(j), p[j]);
#pragma unroll
            for (int j = 0; j < kHeld; ++j) {
                get(at.column(j), p[j], hv[j], gv[j], pv[j]);
                kept(0, j, w);
                sums(hv[j], gv[j]);
            }
        } else {
            for (int j = 0; j * team.warps * at.kPieces < row_pieces<SHIFT>(cols); ++j) {
                load8<SHIFT>(h, at.column(j), cols, hv[0]);
                load8<SHIFT>(dy, at.column(j), cols, gv[0]);
                weights(at.column(j), w);
                sums(hv[0], gv[0]);
            }
        }
        // (two buffers: the barrier of a row frees the buffer of the row before.  It also orders every fetch of the row before
        // the first store to it, where dx is one of the inputs.)
        team_reduce<true, true, false>(team, sq, along, unused, s_scratch[team.id][side]);
        const float root = 1.0f / sqrtf(sq * inv_n + a.eps);
        const float coef = along * root * inv_n;
        auto give = [&](int c, const float (&hp)[8], const float (&gp)[8], const float (&pp)[8]) {
            float o[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float unit = hp[e] * root;
                o[e] = fmaf(root, fmaf(gp[e], w[e], -unit * coef), pp[e]);
                sum[e] = fmaf(gp[e], unit, sum[e]);
            }
            store8<SHIFT>(dx, c, cols, o);
        };
        if constexpr (NV != 0) {
#pragma unroll
            for (int j = 0; j < kHeld; ++j) {
                kept(0, j, w);
                kept(1, j, sum);
                give(at.column(j), hv[j], gv[j], pv[j]);
                keep(1, j, sum);
            }
        } else {
            float hn[8], gn[8], pn[8];
            Piece<SHIFT, T> p[3];
            fetch(at.column(0), p);
            get(at.column(0), p, hv[0], gv[0], pv[0]);
            for (int j = 0; j * team.warps * at.kPieces < row_pieces<SHIFT>(cols); ++j) {
                const int c = at.column(j);
                if ((j + 1) * team.warps * at.kPieces < row_pieces<SHIFT>(cols)) {
                    fetch(at.column(j + 1), p);
                    get(at.column(j + 1), p, hn, gn, pn);
                }
                if (SHIFT) team.sync();  // (as in the second walk of k_rows_quantize)
                weights(c, w);
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] = part && r != me && c + e >= 0 && c + e < cols ? part[c + e] : 0.0f;
                give(c, hv[0], gv[0], pv[0]);
                if (part) give_part(c, sum);
#pragma unroll
                for (int e = 0; e < 8; ++e) hv[0][e] = hn[e], gv[0][e] = gn[e], pv[0][e] = pn[e];
            }
        }
    }
    if constexpr (NV != 0) {
        if (part) {
#pragma unroll
            for (int j = 0; j < kHeld; ++j) {
                float p[8];
                kept(1, j, p);
                give_part(at.column(j), p);
            }
        }
    }
}

// dweight[c] = sum of the teams' partial sums in a fixed order: 32 columns by 32 runs of teams a block.
__global__ void __launch_bounds__(1024) k_norm_weight_sum(const float* __restrict__ part, int64_t teams, int64_t cols, float* __restrict__ dweight) {
    __shared__ float s[32][33];
    const int64_t c = (int64_t)blockIdx.x * 32 + threadIdx.x;
    float sum = 0.0f;
    if (c < cols) {
#pragma unroll 4
        for (int64_t g = threadIdx.y; g < teams; g += 32) sum += part[g * cols + c];
    }
    s[threadIdx.y][threadIdx.x] = sum;
    __syncthreads();
    // warp y adds up column y of the block's 32
    float all = s[threadIdx.x][threadIdx.y];
#pragma unroll
    for (int d = 16; d; d >>= 1) all += __shfl_xor_sync(kFullMask, all, d);
    const int64_t out = (int64_t)blockIdx.x * 32 + threadIdx.y;
    if (threadIdx.x == 0 && out < cols) dweight[out] = all;
}

struct GateBackArgs {
    const void *dy, *gate, *up;
    void *dgate, *dup;
    int64_t lddy, ldg, ldu, lddg, lddu, rows, cols;
};

// A team works on rounds of one piece a lane: all rounds of a row (ALIAS: an output is an input, and rows do not start on 16
// bytes, so the team fetches a round and the next before it stores the first), or those of its share of the grid.
template <int DT, bool SHIFT, bool ALIAS>
__global__ void __launch_bounds__(32 * kBlockWarps) k_gate_backward(const GateBackArgs a) {
    typedef typename Store<DT>::type T;
    const Team team{(int)(blockDim.x >> 5), (int)(threadIdx.x >> 5), (int)threadIdx.y};
    const Lanes<SHIFT> at{team.warps, team.warp, (int)(threadIdx.x & 31)};
    const int cols = (int)a.cols;
    const int rounds = (row_pieces<SHIFT>(cols) + team.warps * at.kPieces - 1) / (team.warps * at.kPieces);
    for (int64_t r = (int64_t)blockIdx.x * blockDim.y + threadIdx.y; r < a.rows; r += (int64_t)gridDim.x * blockDim.y) {
        const T* dy = static_cast<const T*>(a.dy) + r * a.lddy;
        const T* gate = static_cast<const T*>(a.gate) + r * a.ldg;
        const T* up = static_cast<const T*>(a.up) + r * a.ldu;
        T* dgate = static_cast<T*>(a.dgate) + r * a.lddg;
        T* dup = static_cast<T*>(a.dup) + r * a.lddu;
        float d[8], g[8], u[8], dn[8], gn[8], un[8];
        auto fetch = [&](int c, float (&dp)[8], float (&gp)[8], float (&up8)[8]) {
            Piece<SHIFT, T> p, q, o;
            p.fetch(dy, c, cols);
            q.fetch(gate, c, cols);
            o.fetch(up, c, cols);
            p.get(dy, c, cols, dp);
            q.get(gate, c, cols, gp);
            o.get(up, c, cols, up8);
        };
        if (ALIAS) fetch(at.column(0), d, g, u);
        for (int j = blockIdx.y; j < rounds; j += gridDim.y) {
            const int c = at.column(j);
            if (ALIAS) {
                if (j + 1 < rounds) fetch(at.column(j + 1), dn, gn, un);
                team.sync();
            } else {
                fetch(c, d, g, u);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float s = sigmoid(g[e]), ds = d[e] * s;
                u[e] = ds * u[e] * fmaf(g[e], 1.0f - s, 1.0f);
                d[e] = ds * g[e];
            }
            store8<SHIFT>(dgate, c, cols, u);
            store8<SHIFT>(dup, c, cols, d);
            if (ALIAS) {
#pragma unroll
                for (int e = 0; e < 8; ++e) d[e] = dn[e], g[e] = gn[e], u[e] = un[e];
            }
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
    if (dtype == DNNS_F32) vec ? launch_quantize<OP, DNNS_F32, false>(a, n_sm, st) : launch_quantize<OP, DNNS_F32, true>(a, n_sm, st);
    else vec ? launch_quantize<OP, DNNS_BF16, false>(a, n_sm, st) : launch_quantize<OP, DNNS_BF16, true>(a, n_sm, st);
    return cudaGetLastError() == cudaSuccess ? DNNS_OK : DNNS_ERR_CUDA;
}

// Teams of the norm's gradient: as many as stay busy on the 148 SMs with at least 16 rows each, so that the partial sums of
// dweight, one row of fp32 a team, stay small beside the matrices.
Shape norm_backward_shape(int64_t cols, bool shift) {
    Shape s{0, 0, 0};
    for (int nv = 1; nv <= 2 && s.nv == 0; nv *= 2) s = row_shape(cols, shift, nv, backward_warps(nv));
    if (s.nv == 0) s.warps = backward_warps(0);
    return s;
}
int64_t norm_backward_teams(int64_t rows, int64_t cols) {
    const Shape s = norm_backward_shape(cols, true);
    const int64_t room = 148 * std::max(1, (s.nv == 1 ? 32 : 20) / s.warps);  // (64 and 96 registers a thread)
    return std::min(rows, std::min(room, std::max<int64_t>(148, rows / 16)));
}

template <int DT, bool SHIFT>
bool launch_norm_backward(const NormBackArgs& a, cudaStream_t st) {
    static std::atomic<uint64_t> done{0};
    Shape s = norm_backward_shape(a.cols, SHIFT);
    const int64_t teams = norm_backward_teams(a.rows, a.cols);
    while (teams % s.teams) --s.teams;  // (every team of the grid has a slice of the workspace)
    const unsigned grid = (unsigned)(teams / s.teams);
    const dim3 block(32 * s.warps, s.teams);
    const size_t shared = (size_t)s.nv * 2 * 32 * block.x * block.y;
    if (s.nv == 0) k_norm_backward<DT, SHIFT, 0><<<grid, block, 0, st>>>(a);
    else if (s.nv == 1) k_norm_backward<DT, SHIFT, 1><<<grid, block, shared, st>>>(a);
    else {
        int dev = 0;
        if (cudaGetDevice(&dev) != cudaSuccess || !allow_shared(k_norm_backward<DT, SHIFT, 2>, 2 * 2 * 32 * 32 * backward_warps(2), done, dev)) return false;
        k_norm_backward<DT, SHIFT, 2><<<grid, block, shared, st>>>(a);
    }
    return true;
}

template <int DT, bool SHIFT, bool ALIAS>
void launch_gate_backward(const GateBackArgs& a, int n_sm, cudaStream_t st) {
    Shape s = row_shape(a.cols, SHIFT, 1, kBlockWarps);
    if (s.nv == 0) s = Shape{1, kBlockWarps, 1};
    const int lanes = SHIFT ? 31 : 32;
    const int rounds = (row_pieces<SHIFT>((int)a.cols) + lanes * s.warps - 1) / (lanes * s.warps);
    const dim3 grid((unsigned)std::min<int64_t>((a.rows + s.teams - 1) / s.teams, (int64_t)1 << 30), ALIAS ? 1 : std::min(rounds, 65535));
    k_gate_backward<DT, SHIFT, ALIAS><<<grid, dim3(32 * s.warps, s.teams), 0, st>>>(a);
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
    return ((size_t)dnns::norm_backward_teams(rows, cols) * (size_t)cols * sizeof(float) + 255) & ~(size_t)255;
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
    const bool launched = dtype == DNNS_F32 ? (vec ? launch_norm_backward<DNNS_F32, false>(a, st) : launch_norm_backward<DNNS_F32, true>(a, st))
                                            : (vec ? launch_norm_backward<DNNS_BF16, false>(a, st) : launch_norm_backward<DNNS_BF16, true>(a, st));
    if (!launched) return DNNS_ERR_CUDA;
    if (dweight) k_norm_weight_sum<<<(unsigned)((cols + 31) / 32), dim3(32, 32), 0, st>>>(a.part, norm_backward_teams(rows, cols), cols, dweight);
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
    bool alias = false;
    for (const void* out : {dgate, dup}) alias = alias || out == dy || out == gate || out == up;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (vec) dtype == DNNS_F32 ? launch_gate_backward<DNNS_F32, false, false>(a, n_sm, st) : launch_gate_backward<DNNS_BF16, false, false>(a, n_sm, st);
    else if (alias) dtype == DNNS_F32 ? launch_gate_backward<DNNS_F32, true, true>(a, n_sm, st) : launch_gate_backward<DNNS_BF16, true, true>(a, n_sm, st);
    else dtype == DNNS_F32 ? launch_gate_backward<DNNS_F32, true, false>(a, n_sm, st) : launch_gate_backward<DNNS_BF16, true, false>(a, n_sm, st);
    return cudaGetLastError() == cudaSuccess ? DNNS_OK : DNNS_ERR_CUDA;
}

}  // extern "C"
