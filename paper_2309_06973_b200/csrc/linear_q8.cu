// Product of rows in 8 bits:  y[t][n] = (sum_k xq[t][k] * wq[n][k]) * xscale[t] * wscale[n] + bias[n].
// The sum is exact in int32 (at most 2^17 - 1 products of at most 2^14 each), so any order of it gives the same bits.
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

// Bytes k0 .. k0 + 15 of a row of k bytes, those past the end as 0 (never read).
__device__ __forceinline__ int4 row16(const int8_t* row, int32_t k0, int32_t k) {
    if (k0 + 16 <= k) return *reinterpret_cast<const int4*>(row + k0);
    uint32_t w[4] = {0, 0, 0, 0};
    for (int i = 0; k0 + i < k; ++i) w[i >> 2] |= (uint32_t)(uint8_t)row[k0 + i] << (8 * (i & 3));
    return make_int4((int)w[0], (int)w[1], (int)w[2], (int)w[3]);
}

constexpr int kTokens = 8;  // tokens of a block
constexpr int kRowsWarp = 4;  // output channels of a warp

template <int DT>
__global__ void __launch_bounds__(256) k_linear_rows(const LinearArgs a) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t n0 = ((int64_t)blockIdx.x * 8 + warp) * kRowsWarp;
    const int32_t t0 = blockIdx.y * kTokens;
    int32_t acc[kRowsWarp][kTokens] = {};
    for (int32_t k0 = lane * 16; k0 < a.k; k0 += 512) {
        int4 x[kTokens];
#pragma unroll
        for (int t = 0; t < kTokens; ++t) x[t] = t0 + t < a.rows ? row16(a.xq + (int64_t)(t0 + t) * a.ldx, k0, a.k) : make_int4(0, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < kRowsWarp; ++i) {
            if (n0 + i >= a.n) break;
            const int4 w = row16(a.wq + (n0 + i) * a.ldw, k0, a.k);
#pragma unroll
            for (int t = 0; t < kTokens; ++t)
                acc[i][t] = __dp4a(w.x, x[t].x, __dp4a(w.y, x[t].y, __dp4a(w.z, x[t].z, __dp4a(w.w, x[t].w, acc[i][t]))));
        }
    }
#pragma unroll
    for (int i = 0; i < kRowsWarp; ++i)
#pragma unroll
        for (int t = 0; t < kTokens; ++t) {
            const int32_t s = __reduce_add_sync(0xFFFFFFFFu, acc[i][t]);
            if (lane == 0 && n0 + i < a.n && t0 + t < a.rows)
                store_out<DT>(a.y, (int64_t)(t0 + t) * a.ldy + n0 + i, scaled(s, a.xscale[t0 + t], a.wscale[n0 + i], a.bias ? a.bias[n0 + i] : 0.0f));
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
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int64_t step = 8 * kRowsWarp;
    for (int64_t t0 = 0; t0 < rows; t0 += 65535 * (int64_t)kTokens) {  // (the grid's second extent)
        LinearArgs part = a;
        part.rows = (int32_t)std::min<int64_t>(rows - t0, 65535 * (int64_t)kTokens);
        part.xq += t0 * ldx, part.xscale += t0;
        part.y = static_cast<char*>(y) + t0 * ldy * (dtype == DNNS_F32 ? 4 : 2);
        const dim3 grid((unsigned)((out_cols + step - 1) / step), (unsigned)((part.rows + kTokens - 1) / kTokens));
        if (dtype == DNNS_F32) k_linear_rows<DNNS_F32><<<grid, 256, 0, st>>>(part);
        else k_linear_rows<DNNS_BF16><<<grid, 256, 0, st>>>(part);
    }
    return cudaGetLastError() == cudaSuccess ? DNNS_OK : DNNS_ERR_CUDA;
}
