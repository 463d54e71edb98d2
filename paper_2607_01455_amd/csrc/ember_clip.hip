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
// whose rows are contiguous and which is taken as one row.  A block takes
// consecutive runs, one a wave at a time; the second pass takes them in the
// opposite order, so that it begins with what the first one left in the
// last-level cache.  Tensors are described in the kernel's arguments (nothing is
// uploaded, and a captured launch holds its own copy), contiguous ones in
// 24 bytes each, 152 a launch.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "ember_device.h"
#include "ember_launch.h"

namespace ember {
namespace {

constexpr int kRun = 4096;            // elements a run at most
constexpr int kMaxClipBlocks = 1024;  // blocks (and float64 sums) a launch at most
constexpr int kMinClipBlocks = 64;    // and at least, where there is work for them
constexpr int kMaxSums = 8192;        // sums of all launches, as far as kMinClipBlocks allows
constexpr int kLoadsInFlight = 8;     // 16-byte loads a lane

// A contiguous tensor of fewer than 2^30 elements.
struct FlatTensor {
    const void* src;
    void* dst;
    uint32_t n;       // elements; bit 31: src is bf16, bit 30: dst is
    uint32_t run0;    // runs of this launch before this tensor's
};
// Any other: rows at a stride, a device row count, or more elements.
struct RowsTensor {
    const void* src;
    void* dst;
    const int64_t* rows_dev;   // or null
    int64_t rows;
    int64_t cols;
    int64_t lds;
    int64_t ldd;
    int64_t run0;
    int32_t segs;              // runs a row
    int16_t src_bf16;
    int16_t dst_bf16;
};
constexpr int kFlatPerLaunch = 152, kRowsPerLaunch = 48;

template <typename T> constexpr int kPerLaunch = 0;
template <> constexpr int kPerLaunch<FlatTensor> = kFlatPerLaunch;
template <> constexpr int kPerLaunch<RowsTensor> = kRowsPerLaunch;

template <typename T>
struct Batch {
    T t[kPerLaunch<T>];
    int64_t runs;
    int n;
    bool always;      // the second pass has work at f = 1 too
};
static_assert(sizeof(Batch<FlatTensor>) <= 3840 && sizeof(Batch<RowsTensor>) <= 3840, "kernel arguments");

template <typename T>
__device__ __forceinline__ void add_squares(const u32x4_t& w, double (&s)[2]) {
#pragma unroll
    for (int e = 0; e < kChunkElems<T>; ++e) {
        const double x = (double)elem<T>(w, e);
        s[e & 1] += x * x;
    }
}

template <typename T>
__device__ __forceinline__ void square_run(const T* p, int n, int lane, double (&s)[2]) {
    // elements before the first 16-byte boundary, whole chunks, the rest
    const int head = min(n, (int)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / (int)sizeof(T));
    const int chunks = (n - head) / kChunkElems<T>;
    const int tail = head + chunks * kChunkElems<T>;
    const u32x4_t* q = reinterpret_cast<const u32x4_t*>(p + head);
    int c = lane;
    for (; c + (kLoadsInFlight - 1) * kWave < chunks; c += kLoadsInFlight * kWave) {
        u32x4_t w[kLoadsInFlight];
#pragma unroll
        for (int u = 0; u < kLoadsInFlight; ++u) w[u] = q[c + u * kWave];
#pragma unroll
        for (int u = 0; u < kLoadsInFlight; ++u) add_squares<T>(w[u], s);
    }
    for (; c < chunks; c += kWave) add_squares<T>(q[c], s);
    if (lane < head) {
        const double x = (double)load_elem(p, lane, sizeof(T) == 2);
        s[0] += x * x;
    }
    if (lane < n - tail) {
        const double x = (double)load_elem(p, tail + lane, sizeof(T) == 2);
        s[1] += x * x;
    }
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
    auto chunk = [&](int c, const u32x4_t& w) {
        float v[N];
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = elem<T>(w, e) * f;
        if (vec) {
            store_values<U, N>(out + head + c * N, 0, N, v);
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) put(head + c * N + e, v[e]);
        }
    };
    int c = lane;
    for (; c + (kLoadsInFlight - 1) * kWave < chunks; c += kLoadsInFlight * kWave) {
        u32x4_t w[kLoadsInFlight];
#pragma unroll
        for (int u = 0; u < kLoadsInFlight; ++u) w[u] = q[c + u * kWave];
#pragma unroll
        for (int u = 0; u < kLoadsInFlight; ++u) chunk(c + u * kWave, w[u]);
    }
    for (; c < chunks; c += kWave) chunk(c, q[c]);
    if (lane < head) put(lane, load_elem(p, lane, sizeof(T) == 2) * f);
    if (lane < n - tail) put(tail + lane, load_elem(p, tail + lane, sizeof(T) == 2) * f);
}

// A run of a batch: n elements at src and dst; absent: its row holds no gradient.
struct Run {
    const char* src;
    char* dst;
    int n;
    bool src_bf16, dst_bf16, absent, in_place;
};

// The tensor of run r: its runs begin at or before r, the next one's after it.
template <typename T>
__device__ __forceinline__ int tensor_of(const Batch<T>& b, int64_t r) {
    int lo = 0, hi = b.n;   // in [lo, hi)
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if ((int64_t)b.t[mid].run0 <= r) lo = mid;
        else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ Run run_of(const FlatTensor& t, int64_t r) {
    Run x;
    const uint32_t n = t.n & 0x3FFFFFFFu;
    const uint32_t at = (uint32_t)(r - t.run0) * kRun;
    x.src_bf16 = t.n >> 31;
    x.dst_bf16 = (t.n >> 30) & 1;
    x.src = static_cast<const char*>(t.src) + (size_t)at * (x.src_bf16 ? 2 : 4);
    x.dst = static_cast<char*>(t.dst) + (size_t)at * (x.dst_bf16 ? 2 : 4);
    x.n = (int)min(n - at, (uint32_t)kRun);
    x.absent = false;
    x.in_place = t.src == t.dst;
    return x;
}

__device__ __forceinline__ Run run_of(const RowsTensor& t, int64_t r) {
    Run x;
    const int64_t k = r - t.run0, row = t.segs == 1 ? k : k / t.segs, col = (k - row * t.segs) * kRun;
    x.src_bf16 = t.src_bf16;
    x.dst_bf16 = t.dst_bf16;
    x.src = static_cast<const char*>(t.src) + (row * t.lds + col) * (x.src_bf16 ? 2 : 4);
    x.dst = static_cast<char*>(t.dst) + (row * t.ldd + col) * (x.dst_bf16 ? 2 : 4);
    x.n = (int)min(t.cols - col, (int64_t)kRun);
    x.absent = t.rows_dev && row >= *t.rows_dev;   // a count of less than 0: no row
    x.in_place = t.src == t.dst;
    return x;
}

// Calls f(run) for this wave's runs of the launch.  Block i has the i-th of
// gridDim.x even shares; its waves take the runs of its share in turn.
template <bool kBackwards, typename T, typename F>
__device__ __forceinline__ void each_run(const Batch<T>& b, F f) {
    const int64_t share = b.runs / gridDim.x, over = b.runs % gridDim.x, i = blockIdx.x;
    const int64_t r0 = share * i + min(i, over), r1 = r0 + share + (i < over ? 1 : 0);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    for (int64_t k = wave; k < r1 - r0; k += kWaves) {
        const int64_t r = kBackwards ? r1 - 1 - k : r0 + k;
        f(run_of(b.t[tensor_of(b, r)], r));
    }
}

template <typename T>
__global__ __launch_bounds__(kBlock) void ember_grad_squares(Batch<T> b, double* sums) {
    __shared__ double red[kWaves];
    const int lane = threadIdx.x & (kWave - 1);
    double s[2] = {0.0, 0.0};
    each_run<false>(b, [&](const Run& x) {
        if (x.absent) return;
        if (x.src_bf16) square_run(reinterpret_cast<const uint16_t*>(x.src), x.n, lane, s);
        else square_run(reinterpret_cast<const float*>(x.src), x.n, lane, s);
    });
    const double total = row_all<kBlock>(s[0] + s[1], [](double p, double q) { return p + q; }, red);
    if (threadIdx.x == 0) sums[blockIdx.x] = total;
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

template <typename T>
__global__ __launch_bounds__(kBlock) void ember_grad_scale(Batch<T> b, const double* sums, int n, float max_norm,
                                                           float* out) {
    __shared__ double red[kWaves];
    double norm;
    const float f = clip_factor(sums, n, max_norm, red, norm);
    if (blockIdx.x == 0 && threadIdx.x == 0 && out) {
        out[0] = (float)norm;
        out[1] = f;
    }
    if (f == 1.0f && !b.always) return;
    const int lane = threadIdx.x & (kWave - 1);
    each_run<true>(b, [&](const Run& x) {
        if (x.absent) {
            if (x.dst_bf16) {
                for (int i = lane; i < x.n; i += kWave) reinterpret_cast<uint16_t*>(x.dst)[i] = 0;
            } else {
                for (int i = lane; i < x.n; i += kWave) reinterpret_cast<float*>(x.dst)[i] = 0.0f;
            }
            return;
        }
        if (x.in_place && f == 1.0f) return;   // it is what it would be
        if (x.src_bf16) {
            const uint16_t* p = reinterpret_cast<const uint16_t*>(x.src);
            if (x.dst_bf16) scale_run(p, reinterpret_cast<uint16_t*>(x.dst), x.n, lane, f);
            else scale_run(p, reinterpret_cast<float*>(x.dst), x.n, lane, f);
        } else {
            const float* p = reinterpret_cast<const float*>(x.src);
            if (x.dst_bf16) scale_run(p, reinterpret_cast<uint16_t*>(x.dst), x.n, lane, f);
            else scale_run(p, reinterpret_cast<float*>(x.dst), x.n, lane, f);
        }
    });
}

bool empty(const ember_grad& x) { return x.rows == 0 || x.cols == 0; }
bool contiguous(const ember_grad& x) {
    return x.rows_dev == nullptr && (x.rows == 1 || (x.lds == x.cols && x.ldd == x.cols));
}
bool is_flat(const ember_grad& x) { return contiguous(x) && x.rows * x.cols < ((int64_t)1 << 30); }

int64_t fill(FlatTensor& t, const ember_grad& x, int64_t run0) {
    const int64_t n = x.rows * x.cols;
    t.src = x.src;
    t.dst = x.dst;
    t.n = (uint32_t)n | (x.src_dtype == EMBER_BF16 ? 1u << 31 : 0) | (x.dst_dtype == EMBER_BF16 ? 1u << 30 : 0);
    t.run0 = (uint32_t)run0;   // below 152 * 2^18
    return (n + kRun - 1) / kRun;
}
int64_t fill(RowsTensor& t, const ember_grad& x, int64_t run0) {
    const bool one = contiguous(x);
    t.src = x.src;
    t.dst = x.dst;
    t.rows_dev = x.rows_dev;
    t.rows = one ? 1 : x.rows;
    t.cols = one ? x.rows * x.cols : x.cols;
    t.lds = x.lds;
    t.ldd = x.ldd;
    t.run0 = run0;
    t.segs = (int32_t)((t.cols + kRun - 1) / kRun);   // at most 2^30
    t.src_bf16 = x.src_dtype == EMBER_BF16;
    t.dst_bf16 = x.dst_dtype == EMBER_BF16;
    return t.rows * t.segs;
}

// The k-th launch's tensors of one kind.
template <typename T>
void batch_of(const ember_grad* g, int64_t n, int64_t k, Batch<T>& b) {
    constexpr bool kFlat = sizeof(T) == sizeof(FlatTensor);
    b.n = 0;
    b.runs = 0;
    b.always = false;
    int64_t seen = 0;
    for (int64_t i = 0; i < n && b.n < kPerLaunch<T>; ++i) {
        if (empty(g[i]) || is_flat(g[i]) != kFlat) continue;
        if (seen++ < k * kPerLaunch<T>) continue;
        b.always = b.always || g[i].src != g[i].dst || g[i].rows_dev != nullptr;
        b.runs += fill(b.t[b.n++], g[i], b.runs);
    }
}

struct ClipCall {
    const ember_grad* g;
    int64_t n;
    float max_norm;
    float* out;
    double* sums;
    int most;        // blocks a launch
    hipStream_t s;
};
template <typename T>
int blocks_of(const Batch<T>& b, const ClipCall& c) {
    return (int)std::max<int64_t>(1, std::min<int64_t>((b.runs + kWaves - 1) / kWaves, c.most));
}

// The first pass over the launches of one kind; total: sums so far.
template <typename T>
hipError_t squares(const ClipCall& c, int64_t launches, int& total) {
    Batch<T> b;
    for (int64_t k = 0; k < launches; ++k) {
        batch_of(c.g, c.n, k, b);
        const int nb = blocks_of(b, c);
        ember_grad_squares<T><<<dim3((unsigned)nb), kBlock, 0, c.s>>>(b, c.sums + total);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        total += nb;
    }
    return hipSuccess;
}

// The second pass, last launch first; the norm and the factor are written by
// the first one made.
template <typename T>
hipError_t scales(const ClipCall& c, int64_t launches, int total, float*& out) {
    Batch<T> b;
    for (int64_t k = launches - 1; k >= 0; --k) {
        batch_of(c.g, c.n, k, b);
        const bool work = b.always || !std::isinf(c.max_norm);
        if (!work && out == nullptr) continue;
        const int nb = work ? blocks_of(b, c) : 1;
        ember_grad_scale<T><<<dim3((unsigned)nb), kBlock, 0, c.s>>>(b, c.sums, total, c.max_norm, out);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        out = nullptr;
    }
    return hipSuccess;
}

} // namespace

size_t clip_ws_bytes(int64_t n) {
    // the most sums that n tensors can have: launches of either kind, each at
    // its most blocks
    const int64_t launches = (n + kRowsPerLaunch - 1) / kRowsPerLaunch + 1;
    const int64_t sums = std::max<int64_t>(launches * kMinClipBlocks, std::min<int64_t>(launches * kMaxClipBlocks,
                                                                                      kMaxSums));
    return ((size_t)sums * sizeof(double) + 255) / 256 * 256;
}

hipError_t launch_clip(const ember_grad* g, int64_t n, float max_norm, float* out, char* ws, hipStream_t s) {
    int64_t flats = 0, others = 0;
    for (int64_t i = 0; i < n; ++i)
        if (!empty(g[i])) ++(is_flat(g[i]) ? flats : others);
    int64_t lf = (flats + kFlatPerLaunch - 1) / kFlatPerLaunch;
    const int64_t lr = (others + kRowsPerLaunch - 1) / kRowsPerLaunch;
    if (lf + lr == 0) lf = 1;   // no element at all: an empty launch writes the norm
    ClipCall c{g, n, max_norm, out, reinterpret_cast<double*>(ws), 0, s};
    c.most = (int)std::max<int64_t>(kMinClipBlocks, std::min<int64_t>(kMaxClipBlocks, kMaxSums / (lf + lr)));
    int total = 0;
    hipError_t e = squares<RowsTensor>(c, lr, total);
    if (e == hipSuccess) e = squares<FlatTensor>(c, lf, total);
    if (e == hipSuccess) e = scales<FlatTensor>(c, lf, total, out);
    if (e == hipSuccess) e = scales<RowsTensor>(c, lr, total, out);
    return e;
}

} // namespace ember
