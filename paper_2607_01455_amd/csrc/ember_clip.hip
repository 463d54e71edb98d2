// Global gradient norm over many tensors, and clipping (gfx950).
//
//   n = sqrt(sum over all tensors of sum g^2),  f = max_norm / n if n > max_norm,
//   else 1 (also for a norm that is not a number or infinite),  g <- f g.
//
// Two passes over the gradients and no host read between them.  The first
// leaves one float64 sum a block; the second starts by adding those up, in every
// block in the same order, so all of them have the same factor, and scales.  In
// place with f = 1 it ends there and writes nothing.  Squares are formed and
// added in float64: fp32 squares leave the range at gradients of 2e19 and would
// have to be scaled, and beside the memory the float64 arithmetic is free.
//
// The work is cut into runs: at most kRun elements of one row, or of a tensor
// whose rows are contiguous and which is taken as one row.  A wave takes
// consecutive runs.  Tensors are described in the kernel's arguments, a few
// dozen a launch, so nothing is uploaded.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "ember_device.h"
#include "ember_launch.h"

namespace ember {
namespace {

constexpr int kRun = 4096;            // elements a run at most
constexpr int kMaxClipBlocks = 1024;  // blocks (and float64 sums) a launch

struct ClipTensor {
    const void* src;
    void* dst;
    const int64_t* rows_dev;   // or null
    int64_t rows;
    int64_t cols;
    int64_t lds;
    int64_t ldd;
    int64_t run0;              // runs of this launch before this tensor's
    int32_t segs;              // runs a row
    int16_t src_bf16;
    int16_t dst_bf16;
};
static_assert(sizeof(ClipTensor) == 72, "packed into the kernel's arguments");

struct ClipBatch {
    ClipTensor t[kClipPerLaunch];
    int n;
    bool moved;       // some tensor's result goes elsewhere
    int64_t runs;
};

template <typename T>
__device__ __forceinline__ double square_run(const T* p, int n, int lane) {
    double s = 0.0;
    // elements before the first 16-byte boundary, whole chunks, the rest
    const int head = min(n, (int)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / (int)sizeof(T));
    const int chunks = (n - head) / kChunkElems<T>;
    const int tail = head + chunks * kChunkElems<T>;
    const u32x4_t* q = reinterpret_cast<const u32x4_t*>(p + head);
#pragma unroll 4
    for (int c = lane; c < chunks; c += kWave) {
        const u32x4_t w = q[c];
#pragma unroll
        for (int e = 0; e < kChunkElems<T>; ++e) {
            const double x = (double)elem<T>(w, e);
            s += x * x;
        }
    }
    if (lane < head) {
        const double x = (double)load_elem(p, lane, sizeof(T) == 2);
        s += x * x;
    }
    if (lane < n - tail) {
        const double x = (double)load_elem(p, tail + lane, sizeof(T) == 2);
        s += x * x;
    }
    return s;
}

template <typename T, typename U>
__device__ __forceinline__ void scale_run(const T* p, U* out, int n, int lane, float f) {
    const int head = min(n, (int)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / (int)sizeof(T));
    const int chunks = (n - head) / kChunkElems<T>;
    const int tail = head + chunks * kChunkElems<T>;
    const u32x4_t* q = reinterpret_cast<const u32x4_t*>(p + head);
    constexpr int N = kChunkElems<T>;
    // whole chunks are stored as vectors where the destination's are aligned too
    constexpr int kOut = N * (int)sizeof(U) < 16 ? N * (int)sizeof(U) : 16;
    const bool vec = (reinterpret_cast<uintptr_t>(out + head) & (kOut - 1)) == 0;
    auto put = [&](int i, float v) {
        if constexpr (sizeof(U) == 4) out[i] = v;
        else out[i] = (U)pack_bf16(v, 0.0f);
    };
#pragma unroll 4
    for (int c = lane; c < chunks; c += kWave) {
        const u32x4_t w = q[c];
        float v[N];
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = elem<T>(w, e) * f;
        if (vec) {
            store_values<U, N>(out + head + c * N, 0, N, v);
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) put(head + c * N + e, v[e]);
        }
    }
    if (lane < head) put(lane, load_elem(p, lane, sizeof(T) == 2) * f);
    if (lane < n - tail) put(tail + lane, load_elem(p, tail + lane, sizeof(T) == 2) * f);
}

// Calls f(tensor, row, first column, columns) for this wave's runs of the launch.
template <typename F>
__device__ __forceinline__ void each_run(const ClipBatch& b, F f) {
    const int64_t waves = (int64_t)gridDim.x * kWaves;
    const int64_t wave = (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int64_t r0 = b.runs / waves * wave + min(wave, b.runs % waves);
    const int64_t r1 = r0 + b.runs / waves + (wave < b.runs % waves ? 1 : 0);
    int i = 0;
    int64_t held = -1;
    for (int64_t r = r0; r < r1; ++r) {
        while (i + 1 < b.n && r >= b.t[i + 1].run0) {
            ++i;
            held = -1;
        }
        const ClipTensor& t = b.t[i];
        if (held < 0) {
            // a count outside [0, rows] is taken as the nearer end
            held = t.rows;
            if (t.rows_dev) held = max((int64_t)0, min(held, *t.rows_dev));
        }
        const int64_t k = r - t.run0, row = k / t.segs;
        if (row >= held) continue;
        const int64_t col = (k - row * t.segs) * kRun;
        f(t, row, col, (int)min((int64_t)kRun, t.cols - col));
    }
}

__global__ __launch_bounds__(kBlock) void ember_grad_squares(ClipBatch b, double* sums) {
    __shared__ double red[kWaves];
    const int lane = threadIdx.x & (kWave - 1);
    double s = 0.0;
    each_run(b, [&](const ClipTensor& t, int64_t row, int64_t col, int n) {
        const int64_t at = row * t.lds + col;
        if (t.src_bf16) s += square_run(static_cast<const uint16_t*>(t.src) + at, n, lane);
        else s += square_run(static_cast<const float*>(t.src) + at, n, lane);
    });
    s = row_all<kBlock>(s, [](double p, double q) { return p + q; }, red);
    if (threadIdx.x == 0) sums[blockIdx.x] = s;
}

// The factor from the n sums: the same in every block.
__device__ __forceinline__ float clip_factor(const double* sums, int n, float max_norm, double* red, double& norm) {
    double s = 0.0;
    for (int i = threadIdx.x; i < n; i += kBlock) s += sums[i];
    s = row_all<kBlock>(s, [](double p, double q) { return p + q; }, red);
    norm = sqrt(s);
    const bool clip = norm > (double)max_norm && norm < __builtin_inf();
    return clip ? (float)((double)max_norm / norm) : 1.0f;
}

__global__ __launch_bounds__(kBlock) void ember_grad_scale(ClipBatch b, const double* sums, int n, float max_norm,
                                                           float* out) {
    __shared__ double red[kWaves];
    double norm;
    const float f = clip_factor(sums, n, max_norm, red, norm);
    if (blockIdx.x == 0 && threadIdx.x == 0 && out) {
        out[0] = (float)norm;
        out[1] = f;
    }
    if (f == 1.0f && !b.moved) return;
    const int lane = threadIdx.x & (kWave - 1);
    each_run(b, [&](const ClipTensor& t, int64_t row, int64_t col, int n) {
        if (t.src == t.dst && f == 1.0f) return;   // in place: it is what it would be
        const int64_t i = row * t.lds + col, o = row * t.ldd + col;
        if (t.src_bf16) {
            const uint16_t* p = static_cast<const uint16_t*>(t.src) + i;
            if (t.dst_bf16) scale_run(p, static_cast<uint16_t*>(t.dst) + o, n, lane, f);
            else scale_run(p, static_cast<float*>(t.dst) + o, n, lane, f);
        } else {
            const float* p = static_cast<const float*>(t.src) + i;
            if (t.dst_bf16) scale_run(p, static_cast<uint16_t*>(t.dst) + o, n, lane, f);
            else scale_run(p, static_cast<float*>(t.dst) + o, n, lane, f);
        }
    });
}

int clip_blocks(const ClipBatch& b) {
    return (int)std::max<int64_t>(1, std::min<int64_t>((b.runs + kWaves - 1) / kWaves, kMaxClipBlocks));
}

} // namespace

size_t clip_ws_bytes(int64_t n) {
    const int64_t launches = std::max<int64_t>(1, (n + kClipPerLaunch - 1) / kClipPerLaunch);
    return (size_t)launches * kMaxClipBlocks * sizeof(double);
}

hipError_t launch_clip(const ember_grad* g, int64_t n, float max_norm, float* out, char* ws, hipStream_t s) {
    double* const sums = reinterpret_cast<double*>(ws);
    auto batch = [&](int64_t i0, ClipBatch& b) {
        b.n = 0;
        b.runs = 0;
        b.moved = false;
        for (int64_t i = i0; i < std::min(n, i0 + kClipPerLaunch); ++i) {
            const ember_grad& x = g[i];
            if (x.rows == 0 || x.cols == 0) continue;
            ClipTensor& t = b.t[b.n];
            const bool flat = x.rows_dev == nullptr && (x.rows == 1 || (x.lds == x.cols && x.ldd == x.cols));
            t.src = x.src;
            t.dst = x.dst;
            t.rows_dev = x.rows_dev;
            t.rows = flat ? 1 : x.rows;
            t.cols = flat ? x.rows * x.cols : x.cols;
            t.lds = x.lds;
            t.ldd = x.ldd;
            t.run0 = b.runs;
            t.segs = (int32_t)((t.cols + kRun - 1) / kRun);
            t.src_bf16 = x.src_dtype == EMBER_BF16;
            t.dst_bf16 = x.dst_dtype == EMBER_BF16;
            b.moved = b.moved || t.src != t.dst;
            b.runs += t.rows * t.segs;
            ++b.n;
        }
    };
    ClipBatch b;
    int total = 0;
    for (int64_t i = 0; i == 0 || i < n; i += kClipPerLaunch) {
        batch(i, b);
        const int nb = clip_blocks(b);
        ember_grad_squares<<<dim3((unsigned)nb), kBlock, 0, s>>>(b, sums + total);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        total += nb;
    }
    for (int64_t i = 0; i == 0 || i < n; i += kClipPerLaunch) {
        batch(i, b);
        // a limit of infinity never clips: the first block writes the norm
        const bool scale = b.moved || !std::isinf(max_norm);
        if (!scale) b.runs = b.n = 0;
        if (!scale && i > 0) continue;
        ember_grad_scale<<<dim3((unsigned)clip_blocks(b)), kBlock, 0, s>>>(b, sums, total, max_norm,
                                                                           i == 0 ? out : nullptr);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

} // namespace ember
