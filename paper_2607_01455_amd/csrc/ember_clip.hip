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
// The work is cut into runs: at most 8 KB of one row, or of a tensor whose rows
// are contiguous and which is taken as one row.  A wave takes one run at a
// time, eight 16-byte loads a lane; the waves of the launch go through the runs
// side by side.  (With a share of consecutive runs for each block, the blocks
// read a power of two apart, which few of the memory's channels serve.)  The
// second pass goes backwards, so that it begins with what the first one left in
// the last-level cache, and its own loads and stores are non-temporal, which
// leaves more of that there (128256 x 4096 and 16384 x 4096 bf16 written elsewhere:
// 649 us with ordinary ones, 588 like this).  Tensors are described in the kernel's arguments (nothing is
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

constexpr int kLoads = 8;             // 16-byte loads a lane of a whole run
constexpr int kRunBytes = kLoads * kWave * 16;
constexpr int kMaxClipBlocks = 1024;  // blocks (and float64 sums) a launch at most
constexpr int kMinClipBlocks = 64;    // and at least, where there is work for them
constexpr int kMaxSums = 8192;        // sums of all launches, as far as kMinClipBlocks allows

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

template <typename T> constexpr int kRun = kRunBytes / (int)sizeof(T);   // elements of a whole run of T

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

// A whole run that begins on a 16-byte boundary: its loads, all at once.
template <typename T>
__device__ __forceinline__ bool whole(const void* p, int n) {
    return n == kRun<T> && (reinterpret_cast<uintptr_t>(p) & 15) == 0;
}
template <bool kNT>
__device__ __forceinline__ void load_whole(const void* p, int lane, u32x4_t (&w)[kLoads]) {
    const u32x4_t* q = static_cast<const u32x4_t*>(p);
#pragma unroll
    for (int u = 0; u < kLoads; ++u) w[u] = kNT ? __builtin_nontemporal_load(q + lane + u * kWave) : q[lane + u * kWave];
}

// Any other run: the elements before its first 16-byte boundary, whole chunks, the rest.
struct Parts {
    int head, chunks, tail;
};
template <typename T>
__device__ __forceinline__ Parts parts_of(const T* p, int n) {
    Parts x;
    x.head = min(n, (int)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / (int)sizeof(T));
    x.chunks = (n - x.head) / kChunkElems<T>;
    x.tail = x.head + x.chunks * kChunkElems<T>;
    return x;
}

template <typename T>
__device__ __forceinline__ void square_run(const T* p, int n, int lane, double (&s)[2]) {
    const Parts x = parts_of(p, n);
    const u32x4_t* q = reinterpret_cast<const u32x4_t*>(p + x.head);
#pragma unroll 4
    for (int c = lane; c < x.chunks; c += kWave) add_squares<T>(q[c], s);
    if (lane < x.head) {
        const double v = (double)load_elem(p, lane, sizeof(T) == 2);
        s[0] += v * v;
    }
    if (lane < n - x.tail) {
        const double v = (double)load_elem(p, x.tail + lane, sizeof(T) == 2);
        s[1] += v * v;
    }
}

// A chunk of T, scaled, to N elements of U; vec: they are aligned for vector stores.
template <typename T, typename U>
__device__ __forceinline__ void scale_chunk(const u32x4_t& w, U* out, bool vec, float f) {
    constexpr int N = kChunkElems<T>;
    float v[N];
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = elem<T>(w, e) * f;
    if (vec) {
        store_values<U, N, true>(out, 0, N, v);
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            if constexpr (sizeof(U) == 4) out[e] = v[e];
            else out[e] = (U)pack_bf16(v[e], 0.0f);
        }
    }
}
template <typename T, typename U>
__device__ __forceinline__ bool stores_vectors(const U* out) {
    constexpr int kOut = kChunkElems<T> * (int)sizeof(U) < 16 ? kChunkElems<T> * (int)sizeof(U) : 16;
    return (reinterpret_cast<uintptr_t>(out) & (kOut - 1)) == 0;
}

template <typename T, typename U>
__device__ __forceinline__ void scale_run(const T* p, U* out, int n, int lane, float f) {
    if (whole<T>(p, n)) {
        u32x4_t w[kLoads];
        load_whole<true>(p, lane, w);
        const bool vec = stores_vectors<T>(out);
#pragma unroll
        for (int u = 0; u < kLoads; ++u) scale_chunk<T>(w[u], out + (lane + u * kWave) * kChunkElems<T>, vec, f);
        return;
    }
    const Parts x = parts_of(p, n);
    const u32x4_t* q = reinterpret_cast<const u32x4_t*>(p + x.head);
    const bool vec = stores_vectors<T>(out + x.head);
#pragma unroll 4
    for (int c = lane; c < x.chunks; c += kWave) scale_chunk<T>(q[c], out + x.head + c * kChunkElems<T>, vec, f);
    auto one = [&](int i) {
        const float v = load_elem(p, i, sizeof(T) == 2) * f;
        if constexpr (sizeof(U) == 4) out[i] = v;
        else out[i] = (U)pack_bf16(v, 0.0f);
    };
    if (lane < x.head) one(lane);
    if (lane < n - x.tail) one(x.tail + lane);
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

// Run k of a row of n elements at p: whole runs begin on 16-byte boundaries of
// the source, so the first one is short by the elements between the boundary
// before p and p.
struct Piece {
    int64_t at;
    int n;
};
__device__ __forceinline__ Piece piece_of(const void* p, bool bf16, int64_t n, int64_t k) {
    const int64_t run = bf16 ? kRun<uint16_t> : kRun<float>;
    const int64_t before = (int64_t)(reinterpret_cast<uintptr_t>(p) & 15) >> (bf16 ? 1 : 2);
    const int64_t begin = max(k * run - before, (int64_t)0), end = min((k + 1) * run - before, n);
    return Piece{begin, (int)(end - begin)};
}

__device__ __forceinline__ Run run_of(const FlatTensor& t, int64_t r) {
    Run x;
    x.src_bf16 = t.n >> 31;
    x.dst_bf16 = (t.n >> 30) & 1;
    const Piece q = piece_of(t.src, x.src_bf16, t.n & 0x3FFFFFFFu, r - t.run0);
    x.src = static_cast<const char*>(t.src) + q.at * (x.src_bf16 ? 2 : 4);
    x.dst = static_cast<char*>(t.dst) + q.at * (x.dst_bf16 ? 2 : 4);
    x.n = q.n;
    x.absent = false;
    x.in_place = t.src == t.dst;
    return x;
}

__device__ __forceinline__ Run run_of(const RowsTensor& t, int64_t r) {
    Run x;
    x.src_bf16 = t.src_bf16;
    x.dst_bf16 = t.dst_bf16;
    const int64_t k = r - t.run0, row = t.segs == 1 ? k : k / t.segs;
    const char* src = static_cast<const char*>(t.src) + row * t.lds * (x.src_bf16 ? 2 : 4);
    const Piece q = piece_of(src, x.src_bf16, t.cols, k - row * t.segs);   // a row's last one may be empty
    x.src = src + q.at * (x.src_bf16 ? 2 : 4);
    x.dst = static_cast<char*>(t.dst) + (row * t.ldd + q.at) * (x.dst_bf16 ? 2 : 4);
    x.n = max(q.n, 0);
    x.absent = t.rows_dev && row >= *t.rows_dev;   // a count of less than 0: no row
    x.in_place = t.src == t.dst;
    return x;
}

// This wave's first run of the launch, and how far apart its runs are.
__device__ __forceinline__ int64_t first_run() {
    return (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
}
__device__ __forceinline__ int64_t run_step() { return (int64_t)gridDim.x * kWaves; }

template <typename T>
__global__ __launch_bounds__(kBlock) void ember_grad_squares(Batch<T> b, double* sums) {
    __shared__ double red[kWaves];
    const int lane = threadIdx.x & (kWave - 1);
    double s[2] = {0.0, 0.0};
    int64_t r = first_run();
    Run x{};
    if (r < b.runs) x = run_of(b.t[tensor_of(b, r)], r);
    while (r < b.runs) {
        const Run c = x;
        u32x4_t w[kLoads];
        const bool all = !c.absent && (c.src_bf16 ? whole<uint16_t>(c.src, c.n) : whole<float>(c.src, c.n));
        if (all) load_whole<false>(c.src, lane, w);
        // the next run is looked up while the loads are on their way
        r += run_step();
        if (r < b.runs) x = run_of(b.t[tensor_of(b, r)], r);
        if (all) {
            if (c.src_bf16) {
#pragma unroll
                for (int u = 0; u < kLoads; ++u) add_squares<uint16_t>(w[u], s);
            } else {
#pragma unroll
                for (int u = 0; u < kLoads; ++u) add_squares<float>(w[u], s);
            }
        } else if (!c.absent) {
            if (c.src_bf16) square_run(reinterpret_cast<const uint16_t*>(c.src), c.n, lane, s);
            else square_run(reinterpret_cast<const float*>(c.src), c.n, lane, s);
        }
    }
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
    for (int64_t r = first_run(); r < b.runs; r += run_step()) {
        const int64_t back = b.runs - 1 - r;
        const Run x = run_of(b.t[tensor_of(b, back)], back);
        if (x.absent) {
            if (x.dst_bf16) {
                for (int i = lane; i < x.n; i += kWave) reinterpret_cast<uint16_t*>(x.dst)[i] = 0;
            } else {
                for (int i = lane; i < x.n; i += kWave) reinterpret_cast<float*>(x.dst)[i] = 0.0f;
            }
            continue;
        }
        if (x.in_place && f == 1.0f) continue;   // it is what it would be
        if (x.src_bf16) {
            const uint16_t* p = reinterpret_cast<const uint16_t*>(x.src);
            if (x.dst_bf16) scale_run(p, reinterpret_cast<uint16_t*>(x.dst), x.n, lane, f);
            else scale_run(p, reinterpret_cast<float*>(x.dst), x.n, lane, f);
        } else {
            const float* p = reinterpret_cast<const float*>(x.src);
            if (x.dst_bf16) scale_run(p, reinterpret_cast<uint16_t*>(x.dst), x.n, lane, f);
            else scale_run(p, reinterpret_cast<float*>(x.dst), x.n, lane, f);
        }
    }
}

bool empty(const ember_grad& x) { return x.rows == 0 || x.cols == 0; }
bool contiguous(const ember_grad& x) {
    return x.rows_dev == nullptr && (x.rows == 1 || (x.lds == x.cols && x.ldd == x.cols));
}
bool is_flat(const ember_grad& x) { return contiguous(x) && x.rows * x.cols < ((int64_t)1 << 30); }

// Runs of n elements that begin `at` bytes behind a 16-byte boundary (2^40 elements
// at most: below 2^29).
int64_t runs_of(const ember_grad& x, int64_t n, int64_t at) {
    const int64_t es = x.src_dtype == EMBER_BF16 ? 2 : 4;
    return (n * es + at + kRunBytes - 1) / kRunBytes;
}

int64_t fill(FlatTensor& t, const ember_grad& x, int64_t run0) {
    const int64_t n = x.rows * x.cols;
    t.src = x.src;
    t.dst = x.dst;
    t.n = (uint32_t)n | (x.src_dtype == EMBER_BF16 ? 1u << 31 : 0) | (x.dst_dtype == EMBER_BF16 ? 1u << 30 : 0);
    t.run0 = (uint32_t)run0;   // below 152 * 2^19
    return runs_of(x, n, reinterpret_cast<uintptr_t>(x.src) & 15);
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
    // rows that begin on different boundaries: as many runs as the worst of them
    const int64_t es = x.src_dtype == EMBER_BF16 ? 2 : 4;
    const uintptr_t at = reinterpret_cast<uintptr_t>(x.src) & 15;
    t.segs = (int32_t)runs_of(x, t.cols, t.rows == 1 || x.lds * es % 16 == 0 ? at : 16 - es);
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
