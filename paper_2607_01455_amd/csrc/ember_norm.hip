// Root-mean-square norm with the residual's addition, its 8-bit output, and
// its gradient (gfx950).
//
// A row of D columns: s = x + r, rstd = 1 / sqrt(mean_j s_j^2 + eps),
// y_j = s_j rstd gain_j; in 8 bits q_j = rint(y_j 127 / a) with a = max_j |y_j|
// and scale a / 127.  The sum stays in fp32 from the addition to y: the rounded
// s that is stored is an output, not what y is made of.
//
// Gradient, with u = dy gain and k = mean_j u_j s_j:
//   dx_j = rstd u_j - rstd^3 k s_j + ds_j,   dgain_j = sum_t dy_tj s_tj rstd_t.
//
// One pass over the data each: TPR threads hold a row in registers, 16-byte
// chunks dealt round robin, between the loads, the row's one or two reductions
// and the stores.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "ember_device.h"
#include "ember_launch.h"

namespace ember {
namespace {

constexpr int kCodeMax = 127;
// Rows whose largest value is below this are held as zeros: 127 / a would
// leave the fp32 range.
constexpr float kTinyRow = 1e-36f;

struct FwdParams {
    const void* X;
    int64_t ldx;
    const void* R;        // or null
    int64_t ldr;
    const void* gain;     // null: rows are only rounded to 8 bits (no norm)
    bool gain_bf16;
    float eps;
    int64_t T;
    int D;
    void* S;              // or null
    int64_t lds;
    void* Y;              // or null
    bool y_bf16;
    int64_t ldy;
    int8_t* Q;            // or null
    int64_t ldq;
    float* qscale;
    float* rstd;          // or null
};

template <typename XT>
__device__ __forceinline__ void load_gain(const void* gain, bool bf16, int col, int D, float (&g)[kChunkElems<XT>]) {
    constexpr int N = kChunkElems<XT>;
    if (col + N <= D) {
        if (bf16) {
            const uint32_t* p = reinterpret_cast<const uint32_t*>(static_cast<const uint16_t*>(gain) + col);
#pragma unroll
            for (int e = 0; e < N; e += 2) {
                const uint32_t w = p[e >> 1];
                g[e] = __uint_as_float(w << 16);
                g[e + 1] = __uint_as_float(w & 0xFFFF0000u);
            }
        } else {
            const u32x4_t* p = reinterpret_cast<const u32x4_t*>(static_cast<const float*>(gain) + col);
#pragma unroll
            for (int e = 0; e < N; e += 4) {
                const u32x4_t w = p[e >> 2];
#pragma unroll
                for (int q = 0; q < 4; ++q) g[e + q] = __uint_as_float(w[q]);
            }
        }
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) g[e] = col + e < D ? load_elem(gain, col + e, bf16) : 0.0f;
    }
}

// N codes into columns [col, col + N) of a row of Q.
template <int N>
__device__ __forceinline__ void store_codes(int8_t* row, int col, int D, const float (&y)[N], float inv) {
    uint32_t w[N / 4];
#pragma unroll
    for (int q = 0; q < N / 4; ++q) {
        w[q] = 0;
#pragma unroll
        for (int b = 0; b < 4; ++b) w[q] |= ((uint32_t)(int)rintf(y[4 * q + b] * inv) & 0xFFu) << (8 * b);
    }
    if (col + N <= D) {
        if constexpr (N == 8) *reinterpret_cast<u32x2_t*>(row + col) = u32x2_t{w[0], w[1]};
        else *reinterpret_cast<uint32_t*>(row + col) = w[0];
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (col + e < D) row[col + e] = (int8_t)(w[e >> 2] >> (8 * (e & 3)));
    }
}

// kNorm: with the norm; otherwise the row itself goes to 8 bits.
template <typename XT, int TPR, int NC, bool kNorm>
__global__ __launch_bounds__(TPR < kBlock ? kBlock : TPR) void ember_rmsnorm_fwd(FwdParams a) {
    constexpr int kThreads = TPR < kBlock ? kBlock : TPR;
    constexpr int kRows = kThreads / TPR;
    constexpr int N = kChunkElems<XT>;
    __shared__ float red_sum[kThreads / kWave];
    __shared__ uint32_t red_max[kThreads / kWave];
    const int lane = threadIdx.x % TPR;
    // the loop's bounds are the same for all threads of a row, and where a
    // row's threads meet at barriers it is the block's only one
    for (int64_t t = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR; t < a.T; t += (int64_t)gridDim.x * kRows) {
        const XT* x = static_cast<const XT*>(a.X) + t * a.ldx;
        const XT* r = static_cast<const XT*>(a.R) + (a.R ? t * a.ldr : 0);
        float v[NC][N];
        float sq = 0.0f;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int col = (lane + c * TPR) * N;
            const u32x4_t w = load_chunk<XT>(x, col, a.D);
#pragma unroll
            for (int e = 0; e < N; ++e) v[c][e] = elem<XT>(w, e);
            if (a.R) {
                const u32x4_t z = load_chunk<XT>(r, col, a.D);
#pragma unroll
                for (int e = 0; e < N; ++e) v[c][e] += elem<XT>(z, e);
            }
        }
        if constexpr (kNorm) {
#pragma unroll
            for (int c = 0; c < NC; ++c) {
#pragma unroll
                for (int e = 0; e < N; ++e) sq += v[c][e] * v[c][e];
                if (a.S) store_values<XT, N>(static_cast<XT*>(a.S) + t * a.lds, (lane + c * TPR) * N, a.D, v[c]);
            }
            sq = row_all<TPR>(sq, [](float p, float q) { return p + q; }, red_sum);
            const float rstd = 1.0f / sqrtf(sq / (float)a.D + a.eps);
            if (a.rstd && lane == 0) a.rstd[t] = rstd;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int col = (lane + c * TPR) * N;
                float g[N];
                load_gain<XT>(a.gain, a.gain_bf16, col, a.D, g);
#pragma unroll
                for (int e = 0; e < N; ++e) v[c][e] = v[c][e] * rstd * g[e];
                if (a.Y) {
                    if (a.y_bf16) store_values<uint16_t, N>(static_cast<uint16_t*>(a.Y) + t * a.ldy, col, a.D, v[c]);
                    else store_values<float, N>(static_cast<float*>(a.Y) + t * a.ldy, col, a.D, v[c]);
                }
            }
        }
        if (a.Q) {
            // the largest magnitude as an integer: NaN is above infinity is above every number
            uint32_t m = 0;
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int e = 0; e < N; ++e) m = max(m, __float_as_uint(v[c][e]) & 0x7FFFFFFFu);
            m = row_all<TPR>(m, [](uint32_t p, uint32_t q) { return max(p, q); }, red_max);
            const float top = __uint_as_float(m);
            const bool finite = m < 0x7F800000u, some = finite && top >= kTinyRow;
            const float inv = some ? (float)kCodeMax / top : 0.0f;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                if (!finite) {
#pragma unroll
                    for (int e = 0; e < N; ++e) v[c][e] = 0.0f;
                }
                store_codes<N>(a.Q + t * a.ldq, (lane + c * TPR) * N, a.D, v[c], inv);
            }
            if (lane == 0) a.qscale[t] = some ? top / (float)kCodeMax : finite ? 0.0f : __uint_as_float(0x7FC00000u);
        }
        if constexpr (TPR > kWave) __syncthreads();   // the reductions' slots are used again
    }
}

struct GradParams {
    const void* dY;
    int64_t lddy;
    const void* S;
    int64_t lds;
    const void* gain;
    bool gain_bf16;
    const float* rstd;
    const void* dS;       // or null
    int64_t ldds;
    int64_t T;
    int D;
    void* dX;
    int64_t lddx;
    float* part;          // [gridDim.x * rows per block][D]: sums of dgain
};

template <typename XT, int TPR, int NC>
__global__ __launch_bounds__(TPR < kBlock ? kBlock : TPR) void ember_rmsnorm_bwd(GradParams a) {
    constexpr int kThreads = TPR < kBlock ? kBlock : TPR;
    constexpr int kRows = kThreads / TPR;
    constexpr int N = kChunkElems<XT>;
    __shared__ float red[kThreads / kWave];
    const int lane = threadIdx.x % TPR;
    const int64_t group = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR;
    float acc[NC][N];
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int e = 0; e < N; ++e) acc[c][e] = 0.0f;
    for (int64_t t = group; t < a.T; t += (int64_t)gridDim.x * kRows) {
        const XT* dy = static_cast<const XT*>(a.dY) + t * a.lddy;
        const XT* s = static_cast<const XT*>(a.S) + t * a.lds;
        const float rstd = a.rstd[t];
        u32x4_t wy[NC], ws[NC];
        float k = 0.0f;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int col = (lane + c * TPR) * N;
            wy[c] = load_chunk<XT>(dy, col, a.D);
            ws[c] = load_chunk<XT>(s, col, a.D);
        }
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            float g[N];
            load_gain<XT>(a.gain, a.gain_bf16, (lane + c * TPR) * N, a.D, g);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float p = elem<XT>(wy[c], e) * elem<XT>(ws[c], e);
                k += p * g[e];
                acc[c][e] += p * rstd;
            }
        }
        k = row_all<TPR>(k, [](float p, float q) { return p + q; }, red);
        const float ks = k / (float)a.D * rstd * rstd * rstd;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int col = (lane + c * TPR) * N;
            float g[N], d[N];
            load_gain<XT>(a.gain, a.gain_bf16, col, a.D, g);
#pragma unroll
            for (int e = 0; e < N; ++e) d[e] = elem<XT>(wy[c], e) * g[e] * rstd - ks * elem<XT>(ws[c], e);
            if (a.dS) {
                const u32x4_t w = load_chunk<XT>(static_cast<const XT*>(a.dS) + t * a.ldds, col, a.D);
#pragma unroll
                for (int e = 0; e < N; ++e) d[e] += elem<XT>(w, e);
            }
            store_values<XT, N>(static_cast<XT*>(a.dX) + t * a.lddx, col, a.D, d);
        }
        if constexpr (TPR > kWave) __syncthreads();   // the reduction's slots are used again
    }
    float* part = a.part + group * a.D;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const int col = (lane + c * TPR) * N + e;
            if (col < a.D) part[col] = acc[c][e];
        }
    }
}

constexpr int kSumCols = 64;      // columns per block of the partials' sum
constexpr int kSumGroups = kBlock / kSumCols;

// dgain_j = the sum of the partial rows in a fixed order: kSumGroups
// interleaved sums a column, then those in order.
__global__ __launch_bounds__(kBlock) void ember_rmsnorm_dgain(const float* part, int n, int D, float* dgain) {
    __shared__ float sums[kSumGroups][kSumCols];
    const int x = threadIdx.x % kSumCols, g = threadIdx.x / kSumCols;
    const int col = blockIdx.x * kSumCols + x;
    float s = 0.0f;
    if (col < D)
        for (int i = g; i < n; i += kSumGroups) s += part[(int64_t)i * D + col];
    sums[g][x] = s;
    __syncthreads();
    if (g == 0 && col < D) {
#pragma unroll
        for (int q = 1; q < kSumGroups; ++q) s += sums[q][x];
        dgain[col] = s;
    }
}

// Threads per row and chunks per thread for a row of `chunks` 16-byte chunks.
struct RowPlan {
    int tpr, nc;
};
RowPlan row_plan(int64_t T, int D, int dtype) {
    const int epc = dtype == EMBER_F32 ? 4 : 8;
    const int chunks = (D + epc - 1) / epc;
    int tpr = chunks <= 64 ? 64 : chunks <= 2048 ? 256 : 1024;
    int nc = 1;
    while (tpr * nc < chunks) nc *= 2;
    (void)T;
    return RowPlan{tpr, nc};
}

template <typename XT, bool kNorm>
hipError_t launch_fwd(const FwdParams& p, const RowPlan& pl, hipStream_t s) {
    const int rows = pl.tpr < kBlock ? kBlock / pl.tpr : 1;
    const dim3 grid((unsigned)capped_blocks((p.T + rows - 1) / rows));
#define EMBER_FWD(TPR, NC) \
    if (pl.tpr == TPR && pl.nc == NC) ember_rmsnorm_fwd<XT, TPR, NC, kNorm><<<grid, TPR < kBlock ? kBlock : TPR, 0, s>>>(p)
    EMBER_FWD(64, 1);
    else EMBER_FWD(256, 1);
    else EMBER_FWD(256, 2);
    else EMBER_FWD(256, 4);
    else EMBER_FWD(256, 8);
    else EMBER_FWD(1024, 4);
    else EMBER_FWD(1024, 8);
    else return hipErrorInvalidValue;
#undef EMBER_FWD
    return hipGetLastError();
}

template <typename XT>
hipError_t launch_bwd(const GradParams& p, const RowPlan& pl, int blocks, hipStream_t s) {
    const dim3 grid((unsigned)blocks);
#define EMBER_BWD(TPR, NC) \
    if (pl.tpr == TPR && pl.nc == NC) ember_rmsnorm_bwd<XT, TPR, NC><<<grid, TPR < kBlock ? kBlock : TPR, 0, s>>>(p)
    EMBER_BWD(64, 1);
    else EMBER_BWD(256, 1);
    else EMBER_BWD(256, 2);
    else EMBER_BWD(256, 4);
    else EMBER_BWD(256, 8);
    else EMBER_BWD(1024, 4);
    else EMBER_BWD(1024, 8);
    else return hipErrorInvalidValue;
#undef EMBER_BWD
    return hipGetLastError();
}

constexpr int kGradBlocks = 1024;   // blocks of the gradient's pass at most

int grad_blocks(int64_t T, const RowPlan& pl) {
    const int rows = pl.tpr < kBlock ? kBlock / pl.tpr : 1;
    return (int)std::min<int64_t>((T + rows - 1) / rows, kGradBlocks);
}

} // namespace

hipError_t launch_rmsnorm(const NormArgs& x, hipStream_t s) {
    FwdParams p{x.X, x.ldx, x.R, x.ldr, x.gain, x.gain_dtype == EMBER_BF16, x.eps, x.T, (int)x.D, x.S, x.lds,
                x.Y, x.y_dtype == EMBER_BF16, x.ldy, x.Q, x.ldq, x.qscale, x.rstd};
    const RowPlan pl = row_plan(x.T, (int)x.D, x.x_dtype);
    if (x.x_dtype == EMBER_F32) return x.gain ? launch_fwd<float, true>(p, pl, s) : launch_fwd<float, false>(p, pl, s);
    return x.gain ? launch_fwd<uint16_t, true>(p, pl, s) : launch_fwd<uint16_t, false>(p, pl, s);
}

size_t norm_grad_ws_bytes(int64_t T, int64_t D) {
    size_t n = 1;
    for (int dtype : {(int)EMBER_F32, (int)EMBER_BF16}) {
        const RowPlan pl = row_plan(T, (int)D, dtype);
        const size_t rows = pl.tpr < kBlock ? kBlock / pl.tpr : 1;
        n = std::max(n, (size_t)grad_blocks(T, pl) * rows);
    }
    return (n * (size_t)D * sizeof(float) + 255) / 256 * 256;
}

hipError_t launch_rmsnorm_grad(const NormGradArgs& x, hipStream_t s) {
    GradParams p{x.dY, x.lddy, x.S, x.lds, x.gain, x.gain_dtype == EMBER_BF16, x.rstd, x.dS, x.ldds, x.T, (int)x.D,
                 x.dX, x.lddx, reinterpret_cast<float*>(x.ws)};
    const RowPlan pl = row_plan(x.T, (int)x.D, x.x_dtype);
    const int blocks = grad_blocks(x.T, pl);
    const int n = blocks * (pl.tpr < kBlock ? kBlock / pl.tpr : 1);
    if (blocks > 0) {
        const hipError_t e = x.x_dtype == EMBER_F32 ? launch_bwd<float>(p, pl, blocks, s)
                                                    : launch_bwd<uint16_t>(p, pl, blocks, s);
        if (e != hipSuccess) return e;
    }
    ember_rmsnorm_dgain<<<dim3((unsigned)((x.D + kSumCols - 1) / kSumCols)), kBlock, 0, s>>>(p.part, n, (int)x.D,
                                                                                            x.dgain);
    return hipGetLastError();
}

} // namespace ember
