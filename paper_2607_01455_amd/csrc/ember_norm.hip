// Root-mean-square norm with the residual's addition, its 8-bit output, and
// its gradient (gfx950).
//
// A row of D columns: s = x + r, rstd = 1 / sqrt(mean_j s_j^2 + eps),
// y_j = s_j rstd gain_j; in 8 bits q_j = rint(y_j 127 / a) with a = max_j |y_j|
// and scale a / 127.  The sum stays in fp32 from the addition to y: the rounded
// s that is stored is an output, not what y is made of.
//
// Gradient, with u = dy gain, h = s rstd and k = mean_j u_j h_j:
//   dx_j = rstd (u_j - k h_j) + ds_j,   dgain_j = sum_t dy_tj h_tj.
// h is formed first, so that no product leaves the fp32 range where s is far from 1.
//
// One pass over the data each (but the gradient of few tokens, see kSumAtOnceT).  TPR
// threads hold a row between its loads, its one or two reductions and its stores,
// 16-byte chunks dealt round robin.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "ember_device.h"
#include "ember_interface_launch.h"

namespace ember {
namespace {

constexpr int kCodeMax = 127;
// Rows whose largest value is below this are held as zeros: 127 / a would
// leave the fp32 range.
constexpr float kTinyRow = 1e-36f;
// A mean square (eps included) between this and infinity is right as summed in fp32:
// squares below 2^-126 are then off by less than 2^-24 of it.  Other rows, finite ones
// whose squares leave the range among them, are summed again scaled by 2^100 or 2^-100:
// the one's values are below 2^-42, the other's largest is above 2^56.
constexpr float kLeastMean = 0x1p-100f;

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

// The chunk at column col: a full row (D a multiple of the chunk) has whole ones only.
template <typename XT, bool kFull>
__device__ __forceinline__ u32x4_t chunk_at(const XT* row, int col, int D, bool follows) {
    if constexpr (kFull) {
        u32x4_t w = {0, 0, 0, 0};
        if (col < D) w = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(row + col));
        return w;
    } else {
        return load_chunk<XT>(row, col, D, follows);
    }
}
// Element e of it; keep: what counts of it (kept_words), applied where the chunk is
// used, so that the loads of a row are in flight together (the gradient of 16384 x
// 2047 bf16: 101 us with element loads at the end of every row, 53 like this).
template <typename XT, bool kFull>
__device__ __forceinline__ float elem_at(const u32x4_t& w, int e, const u32x4_t& keep) {
    if constexpr (kFull) return elem<XT>(w, e);
    else return elem<XT>(w & keep, e);
}
template <typename T, int N, bool kFull>
__device__ __forceinline__ void store_at(T* row, int col, int D, const float (&v)[N], bool stream) {
    if (kFull && col >= D) return;
    const int end = kFull ? col + N : D;
    if (stream) {
        // the empty statements keep the compiler from making one ordinary store of the two
        asm volatile("");
        store_values<T, N, true>(row, col, end, v);
        asm volatile("");
    } else {
        store_values<T, N, false>(row, col, end, v);
    }
}
template <int N, bool kFull>
__device__ __forceinline__ void codes_at(int8_t* row, int col, int D, const float (&y)[N], float inv) {
    if constexpr (kFull) {
        if (col < D) store_codes<N>(row, col, col + N, y, inv);
    } else {
        store_codes<N>(row, col, D, y, inv);
    }
}

constexpr int threads_of(int tpr) { return tpr < kBlock ? kBlock : tpr; }

// kNorm: with the norm; otherwise the row itself goes to 8 bits.  The threads of a
// row that spans several waves are the block's, so all of them meet at its
// barriers; a block's rows have LDS slots by turns, which the barrier between
// two rows' reductions keeps apart.
// bf16 rows of two chunks a thread: six waves a SIMD, two registers less than the compiler
// would take (16384 x 1024 22.9 us, 24.2 with five waves).
template <typename XT, int TPR, int NC, bool kNorm, bool kFull>
__global__ __launch_bounds__(threads_of(TPR), kNorm && kFull && sizeof(XT) == 2 && TPR == 64 && NC == 2 ? 6 : 1) void ember_rmsnorm_fwd(FwdParams a) {
    constexpr int kRows = threads_of(TPR) / TPR;
    constexpr int N = kChunkElems<XT>;
    __shared__ float red_sum[2][threads_of(TPR) / kWave];
    __shared__ uint32_t red_max[2][threads_of(TPR) / kWave];
    __shared__ float red_again[threads_of(TPR) / kWave];
    const int lane = threadIdx.x % TPR, D = a.D;
    const int64_t step = (int64_t)gridDim.x * kRows;
    int64_t t = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR;
    float g[NC][N];
    constexpr bool kHoldGain = TPR < 1024 || NC <= 2;   // else there are no registers for it
    if constexpr (kNorm && kHoldGain) {
#pragma unroll
        for (int c = 0; c < NC; ++c) load_gain<XT>(a.gain, a.gain_bf16, (lane + c * TPR) * N, D, g[c]);
    }
    for (int turn = 0; t < a.T; t += step, turn ^= 1) {
        const bool follows = t + 1 < a.T;
        u32x4_t wx[NC], wr[NC];
#pragma unroll
        for (int c = 0; c < NC; ++c)
            wx[c] = chunk_at<XT, kFull>(static_cast<const XT*>(a.X) + t * a.ldx, (lane + c * TPR) * N, D, follows);
        if (kNorm && a.R) {
#pragma unroll
            for (int c = 0; c < NC; ++c)
                wr[c] = chunk_at<XT, kFull>(static_cast<const XT*>(a.R) + t * a.ldr, (lane + c * TPR) * N, D, follows);
        }
        float v[NC][N];
        int kl = lane;
        // what counts (and a gain that is not held) is formed anew for each row, not kept in registers
        if constexpr (!kFull || !kHoldGain) asm volatile("" : "+v"(kl));
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const u32x4_t keep = kept_words<XT>((kl + c * TPR) * N, D);
#pragma unroll
            for (int e = 0; e < N; ++e) v[c][e] = elem_at<XT, kFull>(wx[c], e, keep);
        }
        if (kNorm && a.R) {
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const u32x4_t keep = kept_words<XT>((kl + c * TPR) * N, D);
#pragma unroll
                for (int e = 0; e < N; ++e) v[c][e] += elem_at<XT, kFull>(wr[c], e, keep);
            }
        }
        if constexpr (kNorm) {
            float sq = 0.0f;
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int e = 0; e < N; ++e) sq += v[c][e] * v[c][e];
            sq = row_all<TPR>(sq, [](float p, float q) { return p + q; }, red_sum[turn]);
            const float mean = sq / (float)D + a.eps;
            float rstd = 1.0f / sqrtf(mean);
            if (!(mean >= kLeastMean && mean < __builtin_inff())) {
                // the same in all threads of the row, so they meet here too; the next row's first
                // sum keeps the uses of red_again apart
                const float by = mean < 1.0f ? 0x1p100f : 0x1p-100f, root = sqrtf(a.eps) * by;
                float part = 0.0f;
#pragma unroll
                for (int c = 0; c < NC; ++c)
#pragma unroll
                    for (int e = 0; e < N; ++e) part += (v[c][e] * by) * (v[c][e] * by);
                part = row_all<TPR>(part, [](float p, float q) { return p + q; }, red_again);
                rstd = by / sqrtf(part / (float)D + root * root);
            }
            if (a.rstd && lane == 0) a.rstd[t] = rstd;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int col = (lane + c * TPR) * N;
                if (a.S) store_at<XT, N, kFull>(static_cast<XT*>(a.S) + t * a.lds, col, D, v[c], true);
                if constexpr (!kHoldGain) load_gain<XT>(a.gain, a.gain_bf16, (kl + c * TPR) * N, D, g[c]);
#pragma unroll
                for (int e = 0; e < N; ++e) v[c][e] = v[c][e] * rstd * g[c][e];
                if (a.Y) {
                    if (a.y_bf16)
                        store_at<uint16_t, N, kFull>(static_cast<uint16_t*>(a.Y) + t * a.ldy, col, D, v[c], false);
                    else
                        store_at<float, N, kFull>(static_cast<float*>(a.Y) + t * a.ldy, col, D, v[c], false);
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
            m = row_all<TPR>(m, [](uint32_t p, uint32_t q) { return max(p, q); }, red_max[turn]);
            const float top = __uint_as_float(m);
            const bool finite = m < 0x7F800000u, some = finite && top >= kTinyRow;
            const float inv = some ? (float)kCodeMax / top : 0.0f;
            if (!finite) {
#pragma unroll
                for (int c = 0; c < NC; ++c)
#pragma unroll
                    for (int e = 0; e < N; ++e) v[c][e] = 0.0f;
            }
#pragma unroll
            for (int c = 0; c < NC; ++c)
                codes_at<N, kFull>(a.Q + t * a.ldq, (lane + c * TPR) * N, D, v[c], inv);
            if (lane == 0) a.qscale[t] = some ? top / (float)kCodeMax : finite ? 0.0f : __uint_as_float(0x7FC00000u);
        }
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
    int blocks;           // blocks of rows; the others sum dgain themselves
    float* part;          // [blocks][D]: sums of dgain, or null
    float* dgain;
    bool stream;          // dX is stored non-temporally
};

constexpr int kSumGroups = 16;    // interleaved sums of the partial rows

// dgain of 8 chunks of columns, from dY and S themselves, in the order in which the
// partial rows of `blocks` blocks of kGroups rows would give it: what block b's group g
// has over its rounds, those over the groups, those of every 16th block, and
// those sixteen.  Wave w takes the blocks b = w (mod 16), eight at a time, a lane
// the rows of one of them.
template <typename XT, int kGroups, bool kFull>
__device__ __forceinline__ void sum_dgain(const GradParams& a, int first_chunk, float* lds) {
    constexpr int N = kChunkElems<XT>, kAtOnce = kGroups >= 4 ? 4 : 2;   // rows in flight
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, x = lane % 8;
    const int col = (first_chunk + x) * N, step = a.blocks * kGroups;
    const int rounds = (int)((a.T + step - 1) / step);
    float sum[N];
#pragma unroll
    for (int e = 0; e < N; ++e) sum[e] = 0.0f;
    for (int b0 = wave; b0 < a.blocks; b0 += kSumGroups * 8) {
        const int b = b0 + kSumGroups * (lane / 8);
        float acc[N], p[N];
#pragma unroll
        for (int e = 0; e < N; ++e) acc[e] = p[e] = 0.0f;
        int g = 0, i = 0;     // group and round of the next row to load,
        int ug = 0, ui = 0;   // and to add
        for (int j = 0; j < kGroups * rounds; j += kAtOnce) {
            u32x4_t wy[kAtOnce], ws[kAtOnce];
            float r[kAtOnce];
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                const int64_t t = min((int64_t)b * kGroups + g + (int64_t)i * step, a.T - 1);
                wy[u] = chunk_at<XT, kFull>(static_cast<const XT*>(a.dY) + t * a.lddy, col, a.D, t + 1 < a.T);
                ws[u] = chunk_at<XT, kFull>(static_cast<const XT*>(a.S) + t * a.lds, col, a.D, t + 1 < a.T);
                r[u] = a.rstd[t];
                if (++i == rounds) { i = 0; ++g; }
            }
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                if (ug < kGroups) {
                    const bool there = (int64_t)b * kGroups + ug + (int64_t)ui * step < a.T;
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        const float term = __builtin_fmaf(elem<XT>(wy[u], e), elem<XT>(ws[u], e) * r[u], acc[e]);
                        acc[e] = there ? term : acc[e];
                    }
                    if (++ui == rounds) {
                        ui = 0;
#pragma unroll
                        for (int e = 0; e < N; ++e) {
                            p[e] = ug == 0 ? acc[e] : p[e] + acc[e];
                            acc[e] = 0.0f;
                        }
                        ++ug;
                    }
                }
            }
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if (b0 + kSumGroups * k < a.blocks) {
#pragma unroll
                for (int e = 0; e < N; ++e) sum[e] += __shfl(p[e], k * 8 + x);
            }
        }
    }
    if (lane < 8) {
#pragma unroll
        for (int e = 0; e < N; ++e) lds[wave * 8 * N + lane * N + e] = sum[e];
    }
    __syncthreads();
    const int y = threadIdx.x, to = first_chunk * N + y;
    if (y < 8 * N && to < a.D) {
        float total = lds[y];
#pragma unroll
        for (int q = 1; q < kSumGroups; ++q) total += lds[q * 8 * N + y];
        a.dgain[to] = total;
    }
}

// kGroups rows at a time per block, TPR threads each; every thread keeps the
// sums of dgain for its columns over all its rows, and the block adds up its
// groups' at the end, in order.
template <typename XT, int TPR, int NC, int kGroups, bool kFull>
__global__ __launch_bounds__(TPR * kGroups) void ember_rmsnorm_bwd(GradParams a) {
    constexpr int N = kChunkElems<XT>;
    constexpr int kRowWaves = TPR / kWave;
    __shared__ float red[2][kGroups][kRowWaves];
    __shared__ float sums[kGroups > 1 ? kGroups - 1 : 1][TPR * N];
    static_assert(TPR * kGroups == kSumGroups * kWave, "a wave for each of the interleaved sums");
    if ((int)blockIdx.x >= a.blocks) {
        sum_dgain<XT, kGroups, kFull>(a, ((int)blockIdx.x - a.blocks) * 8, &sums[0][0]);
        return;
    }
    const int lane = threadIdx.x % TPR, group = threadIdx.x / TPR, D = a.D;
    const int64_t step = (int64_t)a.blocks * kGroups;
    const int64_t rounds = (a.T - (int64_t)blockIdx.x * kGroups + step - 1) / step;   // of the block: all its threads take part
    int64_t t = (int64_t)blockIdx.x * kGroups + group;
    // else there are no registers for it (1500 x 9001 bf16 held 48.6 us, so 40.2)
    constexpr bool kHoldGain = NC * N <= 8;
    float g[NC][N], acc[NC][N];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        if constexpr (kHoldGain) load_gain<XT>(a.gain, a.gain_bf16, (lane + c * TPR) * N, D, g[c]);
#pragma unroll
        for (int e = 0; e < N; ++e) acc[c][e] = 0.0f;
    }
    u32x4_t ny[NC], ns[NC], nd[NC];
    float nrstd;
    auto load = [&](int64_t row) {
        row = min(row, a.T - 1);
        const bool follows = row + 1 < a.T;
        nrstd = a.rstd[row];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int col = (lane + c * TPR) * N;
            ny[c] = chunk_at<XT, kFull>(static_cast<const XT*>(a.dY) + row * a.lddy, col, D, follows);
            ns[c] = chunk_at<XT, kFull>(static_cast<const XT*>(a.S) + row * a.lds, col, D, follows);
            if (a.dS) nd[c] = chunk_at<XT, kFull>(static_cast<const XT*>(a.dS) + row * a.ldds, col, D, follows);
        }
    };
    // the next row's loads are in flight behind this one's reduction, where the
    // registers hold both
    constexpr bool kAhead = NC == 1;
    if (kAhead) load(t);
    for (int64_t i = 0; i < rounds; ++i, t += step) {
        if (!kAhead) load(t);
        u32x4_t wy[NC], ws[NC], wd[NC];
        const float rstd = nrstd;
        const bool there = t < a.T;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            wy[c] = ny[c];
            ws[c] = ns[c];
            if (a.dS) wd[c] = nd[c];
            if constexpr (!kFull) {   // dS past the row only reaches dX past it, which is not stored
                const u32x4_t keep = kept_words<XT>((lane + c * TPR) * N, D);
                wy[c] &= keep;
                ws[c] &= keep;
            }
        }
        if (kAhead && i + 1 < rounds) load(t + step);
        float k = 0.0f;
        int kl = lane;
        if constexpr (!kHoldGain) asm volatile("" : "+v"(kl));
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            if constexpr (!kHoldGain) load_gain<XT>(a.gain, a.gain_bf16, (kl + c * TPR) * N, D, g[c]);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float dy = elem<XT>(wy[c], e), h = elem<XT>(ws[c], e) * rstd;
                k += dy * g[c][e] * h;
                if (there) acc[c][e] = __builtin_fmaf(dy, h, acc[c][e]);
            }
        }
        // by hand over the row's waves: the block's other rows have slots of their own
        k = wave_all(k, [](float p, float q) { return p + q; });
        if constexpr (TPR > kWave) {
            float* slot = red[i & 1][group];
            if ((threadIdx.x & (kWave - 1)) == 0) slot[lane / kWave] = k;
            __syncthreads();
            k = slot[0];
#pragma unroll
            for (int w = 1; w < kRowWaves; ++w) k += slot[w];
        }
        k /= (float)D;
        if (there) {
            if constexpr (!kHoldGain) asm volatile("" : "+v"(kl));
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                if constexpr (!kHoldGain) load_gain<XT>(a.gain, a.gain_bf16, (kl + c * TPR) * N, D, g[c]);
                float d[N];
#pragma unroll
                for (int e = 0; e < N; ++e) d[e] = (elem<XT>(wy[c], e) * g[c][e] - k * (elem<XT>(ws[c], e) * rstd)) * rstd;
                if (a.dS) {
#pragma unroll
                    for (int e = 0; e < N; ++e) d[e] += elem<XT>(wd[c], e);
                }
                store_at<XT, N, kFull>(static_cast<XT*>(a.dX) + t * a.lddx, (lane + c * TPR) * N, D, d, a.stream);
            }
        }
    }
    if (a.part == nullptr) return;
    float* part = a.part + (int64_t)blockIdx.x * D;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        if constexpr (kGroups > 1) {
            __syncthreads();
            if (group > 0) {
#pragma unroll
                for (int e = 0; e < N; ++e) sums[group - 1][lane + e * TPR] = acc[c][e];
            }
            __syncthreads();
            if (group == 0) {
#pragma unroll
                for (int q = 1; q < kGroups; ++q)
#pragma unroll
                    for (int e = 0; e < N; ++e) acc[c][e] += sums[q - 1][lane + e * TPR];
            }
        }
        if (group == 0) {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const int col = (lane + c * TPR) * N + e;
                if (col < D) part[col] = acc[c][e];
            }
        }
    }
}

constexpr int kSumCols = 64;      // columns per block of the partials' sum
constexpr int kSumThreads = kSumGroups * kSumCols;

// dgain_j = the sum of the partial rows in a fixed order: kSumGroups
// interleaved sums a column, then those in order.
__global__ __launch_bounds__(kSumThreads) void ember_rmsnorm_dgain(const float* part, int n, int D, float* dgain) {
    __shared__ float sums[kSumGroups][kSumCols];
    const int x = threadIdx.x % kSumCols, g = threadIdx.x / kSumCols;
    const int col = blockIdx.x * kSumCols + x;
    float s = 0.0f;
    if (col < D) {
#pragma unroll 8
        for (int i = g; i < n; i += kSumGroups) s += part[(int64_t)i * D + col];
    }
    sums[g][x] = s;
    __syncthreads();
    if (g == 0 && col < D) {
#pragma unroll
        for (int q = 1; q < kSumGroups; ++q) s += sums[q][x];
        dgain[col] = s;
    }
}

// Threads per row and chunks per thread.  The norm has a row in one wave up to 256
// chunks (us, y / 8 bits: 16384 x 2048 bf16 47.3 / 43.5, in four waves 49.0 / 44.5) and in
// four up to 1024 (2000 x 5000 bf16 19.2 / 16.8, in eight 20.2 / 19.4; 8192 x 4096 fp32
// 92.3 / 75.5 and 94.2 / 76.9; 10000 x 8192 bf16 118 / 102 and 115 / 106).  Its
// gradient, whose registers hold one chunk a thread best, in as few waves as have
// one for each (16384 x 1024 bf16 in two waves 28.9, in four 34.4, in one with two
// chunks a thread 31.7).
struct RowPlan {
    int tpr, nc;
    bool full;     // D a multiple of the chunk
};
RowPlan row_plan(int D, int dtype, bool grad) {
    const int epc = dtype == EMBER_F32 ? 4 : 8, chunks = (D + epc - 1) / epc;
    RowPlan p;
    if (grad) p.tpr = chunks <= 64 ? 64 : chunks <= 128 ? 128 : chunks <= 256 ? 256 : chunks <= 512 ? 512 : 1024;
    else p.tpr = chunks <= 256 ? 64 : chunks <= 1024 ? 256 : 1024;
    const int n = (chunks + p.tpr - 1) / p.tpr;
    p.nc = n <= 1 ? 1 : n <= 2 ? 2 : n <= 4 ? 4 : 8;
    p.full = D % epc == 0;
    return p;
}

// The caches are left to what is read next.  The inputs are read once, with
// non-temporal loads, and S, which waits for the gradient, is stored so; Y ordinarily,
// dX too while the caches can keep it.  us, alone and with a kernel that reads Y next, 16384 x
// 4096 bf16: all ordinary 94.8 and 132, S non-temporal 93.5 and 128, the loads too 93.6
// and 116, Y too 91.0 and 126; 8192 x 4096 48.0 and 66.6, 48.3 and 65.3, 43.1 and 60.3,
// 46.3 and 65.5.  dX ordinary / non-temporal, x 4096 bf16, alone, with a kernel that reads it
// next and with one that adds it to another tensor: 14000 85 / 79, 103 / 109, 138 / 140;
// 16384 (128 MiB) 97 / 91, 123 / 125, 154 / 160; 18000 106 / 99, 136 / 136, 180 / 176; 24576 137 / 131,
// 181 / 182, 252 / 237; 49152 278 / 264, 369 / 363, 494 / 467.
constexpr int64_t kKeptDX = (int64_t)128 << 20;
int64_t bytes_of(int64_t T, int64_t D, int dtype) { return T * D * (dtype == EMBER_F32 ? 4 : 2); }

template <typename XT, bool kNorm, bool kFull>
hipError_t launch_fwd(const FwdParams& p, const RowPlan& pl, hipStream_t s) {
    const int threads = threads_of(pl.tpr), rows = threads / pl.tpr;
    // one row a block (or four): fewer blocks that go through more rows each took
    // 99 to 103 us instead of 94 at 16384 x 4096 bf16
    const dim3 grid((unsigned)capped_blocks((p.T + rows - 1) / rows));
#define EMBER_FWD(TPR, NC) \
    if (pl.tpr == TPR && pl.nc == NC) ember_rmsnorm_fwd<XT, TPR, NC, kNorm, kFull><<<grid, threads, 0, s>>>(p)
    EMBER_FWD(64, 1);
    else EMBER_FWD(64, 2);
    else EMBER_FWD(64, 4);
    else EMBER_FWD(256, 2);
    else EMBER_FWD(256, 4);
    else EMBER_FWD(1024, 2);
    else EMBER_FWD(1024, 4);
    else if constexpr (sizeof(XT) == 4) {
        EMBER_FWD(1024, 8);
        else return hipErrorInvalidValue;
    } else return hipErrorInvalidValue;
#undef EMBER_FWD
    return hipGetLastError();
}

// Rows a block of the gradient takes at a time, and its blocks: one of 16 waves a
// compute unit, so that few partial rows are left to add up (512 blocks: 106 us
// instead of 102 at 16384 x 4096 bf16, 40 instead of 33 at 2048 x 8192).
constexpr int kGradBlocks = 256;
int grad_groups(const RowPlan& pl) { return 1024 / pl.tpr; }
int grad_blocks(int64_t T, const RowPlan& pl) {
    return (int)std::min<int64_t>((T + grad_groups(pl) - 1) / grad_groups(pl), kGradBlocks);
}

// Up to this many tokens dgain is summed in the same launch, from dY and S read
// again, unless dX takes the place of one of them (us, so / in a second launch: 128 x
// 4096 bf16 7.3 / 10.4, 500 x 2048 7.4 / 10.8, 500 x 4096 11.2 / 12.8, 1000 x 4096 14.4 /
// 13.3, 2000 x 2048 17.1 / 11.3).
constexpr int64_t kSumAtOnceT = 512;

template <typename XT, bool kFull>
hipError_t launch_bwd(const GradParams& p, const RowPlan& pl, int sum_blocks, hipStream_t s) {
    const dim3 grid((unsigned)(p.blocks + sum_blocks));
#define EMBER_BWD(TPR, NC, G) \
    if (pl.tpr == TPR && pl.nc == NC) ember_rmsnorm_bwd<XT, TPR, NC, G, kFull><<<grid, TPR * G, 0, s>>>(p)
    EMBER_BWD(64, 1, 16);
    else EMBER_BWD(128, 1, 8);
    else EMBER_BWD(256, 1, 4);
    else EMBER_BWD(512, 1, 2);
    else EMBER_BWD(1024, 1, 1);
    else EMBER_BWD(1024, 2, 1);
    else EMBER_BWD(1024, 4, 1);
    else if constexpr (sizeof(XT) == 4) {
        EMBER_BWD(1024, 8, 1);
        else return hipErrorInvalidValue;
    } else return hipErrorInvalidValue;
#undef EMBER_BWD
    return hipGetLastError();
}

template <typename XT>
hipError_t launch_bwd_of(const GradParams& p, const RowPlan& pl, int sum_blocks, hipStream_t s) {
    return pl.full ? launch_bwd<XT, true>(p, pl, sum_blocks, s) : launch_bwd<XT, false>(p, pl, sum_blocks, s);
}

template <typename XT>
hipError_t launch_fwd_of(const FwdParams& p, bool norm, const RowPlan& pl, hipStream_t s) {
    if (norm) return pl.full ? launch_fwd<XT, true, true>(p, pl, s) : launch_fwd<XT, true, false>(p, pl, s);
    return pl.full ? launch_fwd<XT, false, true>(p, pl, s) : launch_fwd<XT, false, false>(p, pl, s);
}

} // namespace

hipError_t launch_rmsnorm(const NormArgs& x, hipStream_t s) {
    FwdParams p{x.X, x.ldx, x.R, x.ldr, x.gain, x.gain_dtype == EMBER_BF16, x.eps, x.T, (int)x.D, x.S, x.lds,
                x.Y, x.y_dtype == EMBER_BF16, x.ldy, x.Q, x.ldq, x.qscale, x.rstd};
    const RowPlan pl = row_plan((int)x.D, x.x_dtype, false);
    return x.x_dtype == EMBER_F32 ? launch_fwd_of<float>(p, x.gain != nullptr, pl, s)
                                  : launch_fwd_of<uint16_t>(p, x.gain != nullptr, pl, s);
}

size_t norm_grad_ws_bytes(int64_t T, int64_t D) {
    int n = 1;
    for (int dtype : {(int)EMBER_F32, (int)EMBER_BF16}) n = std::max(n, grad_blocks(T, row_plan((int)D, dtype, true)));
    return ((size_t)n * (size_t)D * sizeof(float) + 255) / 256 * 256;
}

hipError_t launch_rmsnorm_grad(const NormGradArgs& x, hipStream_t s) {
    GradParams p{x.dY, x.lddy, x.S, x.lds, x.gain, x.gain_dtype == EMBER_BF16, x.rstd, x.dS, x.ldds, x.T, (int)x.D,
                 x.dX, x.lddx, 0, reinterpret_cast<float*>(x.ws), x.dgain, bytes_of(x.T, x.D, x.x_dtype) > kKeptDX};
    const RowPlan pl = row_plan((int)x.D, x.x_dtype, true);
    p.blocks = grad_blocks(x.T, pl);
    if (p.blocks > 0) {
        int sum_blocks = 0;
        if (p.blocks == 1) {
            p.part = x.dgain;   // a single block's sums are the result
        } else if (x.T <= kSumAtOnceT && x.dX != x.dY && x.dX != x.S) {
            p.part = nullptr;   // dY and S stay as they are: other blocks sum dgain meanwhile
            const int chunk = x.x_dtype == EMBER_F32 ? 4 : 8;
            sum_blocks = ((int)x.D + 8 * chunk - 1) / (8 * chunk);
        }
        hipError_t e;
        if (x.x_dtype == EMBER_F32) e = launch_bwd_of<float>(p, pl, sum_blocks, s);
        else e = launch_bwd_of<uint16_t>(p, pl, sum_blocks, s);
        if (e != hipSuccess || p.blocks == 1 || sum_blocks > 0) return e;
    }
    ember_rmsnorm_dgain<<<dim3((unsigned)((x.D + kSumCols - 1) / kSumCols)), kSumThreads, 0, s>>>(p.part, p.blocks,
                                                                                                 (int)x.D, x.dgain);
    return hipGetLastError();
}

} // namespace ember
