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
// 649 us with ordinary ones, 588 like this).
//
// Narrow rows at a stride share runs: a run is then 512 pieces of 16 bytes, or of
// one element where rows do not begin on 16-byte boundaries, and a lane has eight
// loads in flight there too (copied and clipped, bf16, us: 156294 rows of 108 a wave
// each 100, sharing runs 32; 100000 of 130 at a stride of 131 96 and 40).  Rows of
// more than 256 pieces have waves of their own.
//
// Tensors are described in the kernel's arguments (nothing is uploaded, and a
// captured launch holds its own copy), contiguous ones in 12 bytes each, others in
// 80, as many a launch as fit: 304 and 45.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "ember_device.h"
#include "ember_interface_launch.h"

namespace ember {
namespace {

constexpr int kLoads = 8;             // 16-byte loads a lane of a whole run
constexpr int kRunBytes = kLoads * kWave * 16;
constexpr int kMaxClipBlocks = 1024;  // blocks (and float64 sums) a launch at most
constexpr int kMinClipBlocks = 64;    // and at least, where there is work for them
constexpr int kMaxSums = 8192;        // sums of all launches, as far as kMinClipBlocks allows

// A contiguous tensor of fewer than 2^29 elements.
struct FlatTensor {
    int32_t src, dst;   // in 2 bytes, from the launch's bases
    uint32_t n;         // elements; bit 31: src is bf16, bit 30: dst is
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
    int32_t segs;              // runs a row; 0: rows share runs
    int32_t pieces;            // if they do: whole pieces a row,
    uint32_t inverse;          // 2^20 / pieces, rounded up,
    int8_t vec;                // pieces of 16 bytes, else of an element
    int8_t vec_dst;            // and their results can be stored as vectors
    int8_t src_bf16;
    int8_t dst_bf16;
};
constexpr int kPerRun = 512;          // pieces of a shared run
constexpr int kMaxPieces = 256;       // of a row that shares runs: below 256 + 512 pieces, x / pieces = (x inverse) >> 20

template <typename T> constexpr int kRun = kRunBytes / (int)sizeof(T);   // elements of a whole run of T

// The tensors of a launch: contiguous ones from the front of the space, others from its back.
constexpr int kSpace = 3648;
constexpr int kGroup = 8;              // contiguous tensors whose first run is found by adding up
constexpr int kGroups = kSpace / (kGroup * (int)sizeof(FlatTensor));
constexpr int kLeastPerLaunch = kSpace / (int)sizeof(RowsTensor);
constexpr int kMaxLaunches = (EMBER_MAX_GRADS + kLeastPerLaunch - 1) / kLeastPerLaunch;
struct Batch {
    alignas(8) char space[kSpace];
    uint32_t group_run0[kGroups];      // runs before each group
    const char* src;                   // bases of the contiguous ones
    char* dst;
    int64_t flat_runs, runs;           // of the contiguous tensors, and in all
    int16_t flats, others;
    bool always;                       // the second pass has work at f = 1 too
    __host__ __device__ const FlatTensor& flat(int i) const { return reinterpret_cast<const FlatTensor*>(space)[i]; }
    __host__ __device__ const RowsTensor& other(int i) const {
        return reinterpret_cast<const RowsTensor*>(space + kSpace)[-1 - i];
    }
};
static_assert(sizeof(Batch) <= 3840 && kSpace % 16 == 0 && kSpace % (kGroup * sizeof(FlatTensor)) == 0 &&
                  sizeof(RowsTensor) == 80, "kernel arguments");

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
__device__ __forceinline__ void scale_whole(const u32x4_t (&w)[kLoads], U* out, int lane, float f) {
    const bool vec = stores_vectors<T>(out);
#pragma unroll
    for (int u = 0; u < kLoads; ++u) scale_chunk<T>(w[u], out + (lane + u * kWave) * kChunkElems<T>, vec, f);
}

// Any other run.
template <typename T, typename U>
__device__ __forceinline__ void scale_run(const T* p, U* out, int n, int lane, float f) {
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

// A run of rows that share runs, from its first piece on.
template <typename T, bool kVec>
struct Shared {
    static constexpr int N = kVec ? kChunkElems<T> : 1;   // elements a piece
    int64_t row;       // the run's first row
    int x0;            // pieces of it that belong to earlier runs
    int64_t there;     // rows from it on, and
    int64_t held;      // those that hold gradients (may be negative)
    int tail;          // elements of a row behind its whole pieces
    int tails;         // rows whose last whole piece is in this run
    __device__ __forceinline__ Shared(const RowsTensor& t, int64_t k) {
        const int64_t base = k * kPerRun;
        row = base / t.pieces;
        x0 = (int)(base - row * t.pieces);
        there = t.rows - row;
        // the count before the difference: it may be any int64
        held = t.rows_dev ? min(max(*t.rows_dev, (int64_t)0) - row, there) : there;
        tail = (int)t.cols - t.pieces * N;
        tails = (int)min((int64_t)(((uint32_t)(x0 + kPerRun) * t.inverse) >> 20), there);
    }
    // piece x0 + i: its row behind the first and its first element there
    __device__ __forceinline__ void at(const RowsTensor& t, int i, int& q, int& e) const {
        const uint32_t x = (uint32_t)(x0 + i);
        q = (int)((x * t.inverse) >> 20);
        e = ((int)x - q * t.pieces) * N;
    }
    // element i of the rows' tails, i < tails * tail
    __device__ __forceinline__ void at_tail(const RowsTensor& t, int i, int& q, int& e) const {
        q = i / tail;
        e = t.pieces * N + i - q * tail;
    }
};

// The pieces of a run, all of their loads at once; those of rows without a gradient are zeros.
template <typename T, bool kVec, bool kNT>
__device__ __forceinline__ void load_shared(const RowsTensor& t, const Shared<T, kVec>& h, int lane,
                                            u32x4_t (&w)[kLoads]) {
    const T* p = static_cast<const T*>(t.src) + h.row * t.lds;
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
        int q, e;
        h.at(t, lane + u * kWave, q, e);
        // the others load the run's first row, which has one
        const T* from = q < h.held ? p + (int64_t)q * t.lds + e : p;
        if constexpr (kVec) {
            const u32x4_t* v = reinterpret_cast<const u32x4_t*>(from);
            w[u] = kNT ? __builtin_nontemporal_load(v) : *v;
        } else {
            using Bits = std::conditional_t<sizeof(T) == 2, uint16_t, uint32_t>;
            const Bits* v = reinterpret_cast<const Bits*>(from);
            w[u][0] = kNT ? __builtin_nontemporal_load(v) : *v;
        }
    }
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
        int q, e;
        h.at(t, lane + u * kWave, q, e);
        if (q >= h.held) w[u] = u32x4_t{0, 0, 0, 0};
    }
}

template <typename T, bool kVec>
__device__ __forceinline__ void square_shared(const RowsTensor& t, int64_t k, int lane, double (&s)[2]) {
    const Shared<T, kVec> h(t, k);
    if (h.held <= 0) return;
    u32x4_t w[kLoads];
    load_shared<T, kVec, false>(t, h, lane, w);
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
        if constexpr (kVec) {
            add_squares<T>(w[u], s);
        } else {
            const double x = (double)elem<T>(w[u], 0);
            s[u & 1] += x * x;
        }
    }
    if (!kVec || h.tail == 0) return;
    const T* p = static_cast<const T*>(t.src) + h.row * t.lds;
    const int n = (int)min((int64_t)h.tails, h.held) * h.tail;
    for (int i = lane; i < n; i += kWave) {
        int q, e;
        h.at_tail(t, i, q, e);
        const double x = (double)load_elem(p + (int64_t)q * t.lds, e, sizeof(T) == 2);
        s[0] += x * x;
    }
}

template <typename U>
__device__ __forceinline__ void store_elem(U* out, float v) {
    if constexpr (sizeof(U) == 4) *out = v;
    else *out = (U)pack_bf16(v, 0.0f);
}

template <typename T, typename U, bool kVec>
__device__ __forceinline__ void scale_shared(const RowsTensor& t, int64_t k, int lane, float f) {
    const Shared<T, kVec> h(t, k);
    // in place and unscaled, the rows with a gradient are what they would be
    const int64_t from = t.src == t.dst && f == 1.0f ? h.held : 0;
    if (from >= h.there) return;
    u32x4_t w[kLoads];
    if (h.held > 0) {
        load_shared<T, kVec, true>(t, h, lane, w);
    } else {
#pragma unroll
        for (int u = 0; u < kLoads; ++u) w[u] = u32x4_t{0, 0, 0, 0};
    }
    U* out = static_cast<U*>(t.dst) + h.row * t.ldd;
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
        int q, e;
        h.at(t, lane + u * kWave, q, e);
        if (q >= h.there || q < from) continue;
        U* to = out + (int64_t)q * t.ldd + e;
        if constexpr (kVec) scale_chunk<T>(w[u], to, t.vec_dst, f);
        else store_elem(to, elem<T>(w[u], 0) * f);
    }
    if (!kVec || h.tail == 0) return;
    const T* p = static_cast<const T*>(t.src) + h.row * t.lds;
    const int n = h.tails * h.tail;
    for (int i = lane; i < n; i += kWave) {
        int q, e;
        h.at_tail(t, i, q, e);
        if (q < from) continue;
        const float v = q < h.held ? load_elem(p + (int64_t)q * t.lds, e, sizeof(T) == 2) * f : 0.0f;
        store_elem(out + (int64_t)q * t.ldd + e, v);
    }
}

// A run of a batch: n elements at src and dst; absent: its row holds no gradient.
// Or run k of tensor `shared`, whose rows share runs.
struct Run {
    const char* src;
    char* dst;
    int n;
    int shared;        // or -1
    int64_t k;
    bool src_bf16, dst_bf16, absent, in_place;
};

// The last of n whose first run, run0(i), is not behind run r.
template <typename F>
__device__ __forceinline__ int last_before(int n, int64_t r, F run0) {
    int lo = 0, hi = n;   // in [lo, hi)
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if ((int64_t)run0(mid) <= r) lo = mid;
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

// Runs of n < 2^29 contiguous elements at p.
__host__ __device__ __forceinline__ uint32_t flat_runs_of(const void* p, uint32_t n, bool bf16) {
    return ((n << (bf16 ? 1 : 2)) + (uint32_t)(reinterpret_cast<uintptr_t>(p) & 15) + kRunBytes - 1) / kRunBytes;
}
__device__ __forceinline__ Run flat_run_of(const Batch& b, int64_t r) {
    const int group = last_before((b.flats + kGroup - 1) / kGroup, r, [&](int i) { return b.group_run0[i]; });
    uint32_t k = (uint32_t)r - b.group_run0[group];
    int i = 0;
#pragma unroll
    for (int j = 0; j < kGroup - 1; ++j) {   // the tensor with run r is not behind the last one
        const FlatTensor& t = b.flat(group * kGroup + j);
        const uint32_t runs = flat_runs_of(b.src + (int64_t)t.src * 2, t.n & 0x1FFFFFFFu, t.n >> 31);
        if (i == j && k >= runs) {
            k -= runs;
            ++i;
        }
    }
    const FlatTensor& t = b.flat(group * kGroup + i);
    const char* const src = b.src + (int64_t)t.src * 2;
    char* const dst = b.dst + (int64_t)t.dst * 2;
    Run x;
    x.src_bf16 = t.n >> 31;
    x.dst_bf16 = (t.n >> 30) & 1;
    const Piece q = piece_of(src, x.src_bf16, t.n & 0x1FFFFFFFu, k);
    x.src = src + q.at * (x.src_bf16 ? 2 : 4);
    x.dst = dst + q.at * (x.dst_bf16 ? 2 : 4);
    x.n = q.n;
    x.in_place = src == dst;
    x.absent = false;
    x.shared = -1;
    return x;
}

__device__ __forceinline__ Run run_of(const RowsTensor& t, int i, int64_t r) {
    Run x;
    x.src_bf16 = t.src_bf16;
    x.dst_bf16 = t.dst_bf16;
    x.shared = t.segs == 0 ? i : -1;
    x.k = r - t.run0;
    if (t.segs == 0) return x;
    const int64_t k = x.k, row = t.segs == 1 ? k : k / t.segs;
    const char* src = static_cast<const char*>(t.src) + row * t.lds * (x.src_bf16 ? 2 : 4);
    const Piece q = piece_of(src, x.src_bf16, t.cols, k - row * t.segs);   // a row's last one may be empty
    x.src = src + q.at * (x.src_bf16 ? 2 : 4);
    x.dst = static_cast<char*>(t.dst) + (row * t.ldd + q.at) * (x.dst_bf16 ? 2 : 4);
    x.n = max(q.n, 0);
    x.absent = t.rows_dev && row >= *t.rows_dev;   // a count of less than 0: no row
    x.in_place = t.src == t.dst;
    return x;
}

__device__ __forceinline__ Run run_of(const Batch& b, int64_t r) {
    if (r < b.flat_runs) return flat_run_of(b, r);
    const int i = last_before(b.others, r, [&](int j) { return b.other(j).run0; });
    return run_of(b.other(i), i, r);
}

// This wave's first run of the launch, and how far apart its runs are.
__device__ __forceinline__ int64_t first_run() {
    return (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
}
__device__ __forceinline__ int64_t run_step() { return (int64_t)gridDim.x * kWaves; }

__global__ __launch_bounds__(kBlock) void ember_grad_squares(Batch b, double* sums) {
    __shared__ double red[kWaves];
    const int lane = threadIdx.x & (kWave - 1);
    double s[2] = {0.0, 0.0};
    int64_t r = first_run();
    Run x{};
    if (r < b.runs) x = run_of(b, r);
    while (r < b.runs) {
        const Run c = x;
        u32x4_t w[kLoads];
        const bool all = c.shared < 0 && !c.absent &&
                         (c.src_bf16 ? whole<uint16_t>(c.src, c.n) : whole<float>(c.src, c.n));
        if (all) load_whole<false>(c.src, lane, w);
        // the next run is looked up while the loads are on their way
        r += run_step();
        if (r < b.runs) x = run_of(b, r);
        if (all) {
            if (c.src_bf16) {
#pragma unroll
                for (int u = 0; u < kLoads; ++u) add_squares<uint16_t>(w[u], s);
            } else {
#pragma unroll
                for (int u = 0; u < kLoads; ++u) add_squares<float>(w[u], s);
            }
        } else if (c.shared >= 0) {
            const RowsTensor& t = b.other(c.shared);
            if (c.src_bf16) {
                if (t.vec) square_shared<uint16_t, true>(t, c.k, lane, s);
                else square_shared<uint16_t, false>(t, c.k, lane, s);
            } else {
                if (t.vec) square_shared<float, true>(t, c.k, lane, s);
                else square_shared<float, false>(t, c.k, lane, s);
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

template <typename T, typename U>
__device__ __forceinline__ void scale_shared(const RowsTensor& t, int64_t k, int lane, float f) {
    if (t.vec) scale_shared<T, U, true>(t, k, lane, f);
    else scale_shared<T, U, false>(t, k, lane, f);
}

__global__ __launch_bounds__(kBlock) void ember_grad_scale(Batch b, const double* sums, int n, float max_norm,
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
    int64_t r = first_run();
    Run next{};
    if (r < b.runs) next = run_of(b, b.runs - 1 - r);
    while (r < b.runs) {
        const Run x = next;
        const bool work = x.shared < 0 && !x.absent && !(x.in_place && f == 1.0f);   // else it is what it would be
        const bool all = work && (x.src_bf16 ? whole<uint16_t>(x.src, x.n) : whole<float>(x.src, x.n));
        u32x4_t w[kLoads];
        if (all) load_whole<true>(x.src, lane, w);
        r += run_step();
        if (r < b.runs) next = run_of(b, b.runs - 1 - r);
        if (all) {
            if (x.src_bf16) {
                if (x.dst_bf16) scale_whole<uint16_t>(w, reinterpret_cast<uint16_t*>(x.dst), lane, f);
                else scale_whole<uint16_t>(w, reinterpret_cast<float*>(x.dst), lane, f);
            } else {
                if (x.dst_bf16) scale_whole<float>(w, reinterpret_cast<uint16_t*>(x.dst), lane, f);
                else scale_whole<float>(w, reinterpret_cast<float*>(x.dst), lane, f);
            }
        } else if (work) {
            if (x.src_bf16) {
                const uint16_t* p = reinterpret_cast<const uint16_t*>(x.src);
                if (x.dst_bf16) scale_run(p, reinterpret_cast<uint16_t*>(x.dst), x.n, lane, f);
                else scale_run(p, reinterpret_cast<float*>(x.dst), x.n, lane, f);
            } else {
                const float* p = reinterpret_cast<const float*>(x.src);
                if (x.dst_bf16) scale_run(p, reinterpret_cast<uint16_t*>(x.dst), x.n, lane, f);
                else scale_run(p, reinterpret_cast<float*>(x.dst), x.n, lane, f);
            }
        } else if (x.shared >= 0) {
            const RowsTensor& t = b.other(x.shared);
            if (x.src_bf16) {
                if (x.dst_bf16) scale_shared<uint16_t, uint16_t>(t, x.k, lane, f);
                else scale_shared<uint16_t, float>(t, x.k, lane, f);
            } else {
                if (x.dst_bf16) scale_shared<float, uint16_t>(t, x.k, lane, f);
                else scale_shared<float, float>(t, x.k, lane, f);
            }
        } else if (x.absent) {
            if (x.dst_bf16) {
                for (int i = lane; i < x.n; i += kWave) reinterpret_cast<uint16_t*>(x.dst)[i] = 0;
            } else {
                for (int i = lane; i < x.n; i += kWave) reinterpret_cast<float*>(x.dst)[i] = 0.0f;
            }
        }
    }
}

bool empty(const ember_grad& x) { return x.rows == 0 || x.cols == 0; }
bool contiguous(const ember_grad& x) {
    return x.rows_dev == nullptr && (x.rows == 1 || (x.lds == x.cols && x.ldd == x.cols));
}
bool is_flat(const ember_grad& x) { return contiguous(x) && x.rows * x.cols < ((int64_t)1 << 29); }

// Runs of n elements that begin `at` bytes behind a 16-byte boundary (2^40 elements
// at most: below 2^29).
int64_t runs_of(const ember_grad& x, int64_t n, int64_t at) {
    const int64_t es = x.src_dtype == EMBER_BF16 ? 2 : 4;
    return (n * es + at + kRunBytes - 1) / kRunBytes;
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
    t.src_bf16 = x.src_dtype == EMBER_BF16;
    t.dst_bf16 = x.dst_dtype == EMBER_BF16;
    const int64_t es = t.src_bf16 ? 2 : 4, esd = t.dst_bf16 ? 2 : 4;
    const uintptr_t at = reinterpret_cast<uintptr_t>(x.src) & 15;
    const int64_t chunk = 16 / es, out = std::min<int64_t>(16, chunk * esd);   // elements; bytes a chunk is stored in at once
    t.vec = at == 0 && x.lds * es % 16 == 0 && t.cols >= chunk;
    t.vec_dst = (reinterpret_cast<uintptr_t>(x.dst) | (uintptr_t)(x.ldd * esd)) % (uintptr_t)out == 0;
    if (t.rows > 1 && (t.vec ? t.cols / chunk : t.cols) <= kMaxPieces) {
        t.pieces = (int32_t)(t.vec ? t.cols / chunk : t.cols);
        t.inverse = ((1u << 20) + (uint32_t)t.pieces - 1) / (uint32_t)t.pieces;
        t.segs = 0;
        return (t.rows * t.pieces + kPerRun - 1) / kPerRun;
    }
    t.pieces = 0;
    t.inverse = 0;
    // rows that begin on different boundaries: as many runs as the worst of them
    t.segs = (int32_t)runs_of(x, t.cols, t.rows == 1 || x.lds * es % 16 == 0 ? at : 16 - es);
    return t.rows * t.segs;
}

// The tensors from g[i] on that one launch describes, empty ones aside; returns the next one's index.
int64_t batch_of(const ember_grad* g, int64_t n, int64_t i, Batch& b) {
    b.flats = b.others = 0;
    b.flat_runs = b.runs = 0;
    b.always = false;
    for (; i < n; ++i) {
        const ember_grad& x = g[i];
        if (empty(x)) continue;
        bool flat = is_flat(x);
        int64_t src = 0, dst = 0;
        if (flat) {
            if (b.flats == 0) {
                b.src = static_cast<const char*>(x.src);
                b.dst = static_cast<char*>(x.dst);
            }
            src = ((int64_t)reinterpret_cast<uintptr_t>(x.src) - (int64_t)reinterpret_cast<uintptr_t>(b.src)) / 2;
            dst = ((int64_t)reinterpret_cast<uintptr_t>(x.dst) - (int64_t)reinterpret_cast<uintptr_t>(b.dst)) / 2;
            flat = src == (int32_t)src && dst == (int32_t)dst;   // else too far from the first: described in full
        }
        const size_t used = b.flats * sizeof(FlatTensor) + b.others * sizeof(RowsTensor);
        if (used + (flat ? sizeof(FlatTensor) : sizeof(RowsTensor)) > (size_t)kSpace) break;
        b.always = b.always || x.src != x.dst || x.rows_dev != nullptr;
        if (flat) {
            const uint32_t count = (uint32_t)(x.rows * x.cols);
            const bool bf16 = x.src_dtype == EMBER_BF16;
            if (b.flats % kGroup == 0) b.group_run0[b.flats / kGroup] = (uint32_t)b.flat_runs;   // below 304 * 2^18
            const_cast<FlatTensor&>(b.flat(b.flats++)) = FlatTensor{
                (int32_t)src, (int32_t)dst, count | (bf16 ? 1u << 31 : 0) | (x.dst_dtype == EMBER_BF16 ? 1u << 30 : 0)};
            b.flat_runs += flat_runs_of(x.src, count, bf16);
        } else {
            b.runs += fill(const_cast<RowsTensor&>(b.other(b.others++)), x, b.runs);
        }
    }
    for (int k = 0; k < b.others; ++k) const_cast<RowsTensor&>(b.other(k)).run0 += b.flat_runs;
    b.runs += b.flat_runs;
    return i;
}

int blocks_of(const Batch& b, int most) {
    return (int)std::max<int64_t>(1, std::min<int64_t>((b.runs + kWaves - 1) / kWaves, most));
}

} // namespace

size_t clip_ws_bytes(int64_t n) {
    // the most sums that n tensors can have
    const int64_t launches = std::max<int64_t>(1, (n + kLeastPerLaunch - 1) / kLeastPerLaunch);
    const int64_t sums = std::max<int64_t>(launches * kMinClipBlocks, std::min<int64_t>(launches * kMaxClipBlocks,
                                                                                      kMaxSums));
    return ((size_t)sums * sizeof(double) + 255) / 256 * 256;
}

hipError_t launch_clip(const ember_grad* g, int64_t n, float max_norm, float* out, char* ws, hipStream_t s) {
    Batch b;
    int32_t first[kMaxLaunches];   // tensor of each launch
    int launches = 0;
    for (int64_t i = 0; i < n || launches == 0;) {   // no tensor that is not empty: one launch that writes the norm
        first[launches++] = (int32_t)i;
        i = batch_of(g, n, i, b);
    }
    const int most = std::max(kMinClipBlocks, std::min(kMaxClipBlocks, kMaxSums / launches));
    double* const sums = reinterpret_cast<double*>(ws);
    int total = 0;
    for (int k = 0; k < launches; ++k) {
        if (launches > 1) batch_of(g, n, first[k], b);
        const int blocks = blocks_of(b, most);
        ember_grad_squares<<<dim3((unsigned)blocks), kBlock, 0, s>>>(b, sums + total);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        total += blocks;
    }
    // the second pass, last launch first; the first one made writes the norm and the factor
    for (int k = launches - 1; k >= 0; --k) {
        if (k < launches - 1) batch_of(g, n, first[k], b);
        const bool work = b.always || !std::isinf(max_norm);
        if (!work && out == nullptr) continue;
        ember_grad_scale<<<dim3((unsigned)(work ? blocks_of(b, most) : 1)), kBlock, 0, s>>>(b, sums, total, max_norm, out);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        out = nullptr;
    }
    return hipSuccess;
}

} // namespace ember
