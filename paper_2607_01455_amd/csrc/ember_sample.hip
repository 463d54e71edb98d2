// A token drawn from each row of logits (gfx950), with temperature, top-k, top-p,
// min-p and a given random number.
//
// With z = (max - l) log2(e) / temperature a token's weight is 2^-z.  Weights are
// held in fixed point (64-bit integers, up to 48 bits behind the point, so that a
// row's sum fits), formed in fp64: their sums do not depend on any order, so
// blocks may share a row and add up with integer atomics, and a border that is
// met differently in fp64 is as rare as a difference of 2^-45.
//
// The three filters each keep a prefix of the tokens in falling order (equal logits
// by index), so what is kept is the shortest of three prefixes, and one (logit,
// index) says where it ends.  Four launches:
//   1  the largest and smallest logit of each part of a row;
//   2  weights, their sum for every chunk of 512 tokens, and, where top-k or top-p
//      is on, a histogram over z of counts and weights;
//   3  from the histogram the bins in which the prefixes end: their tokens go to
//      a list; sums of the tokens before them for every chunk;
//   4  a block a row sorts the list, finds the end of the prefix, finds the chunk
//      in which the random number falls, and in it the token.
// A list that does not fit (thousands of equal logits where a prefix ends) is
// replaced by a search for the prefix's end by halving, over the whole row.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "ember_device.h"
#include "ember_interface_launch.h"

namespace ember {
namespace {

typedef unsigned long long u64;

constexpr int kThreads = 512;                     // launches 1 to 3
constexpr int kWavesB = kThreads / kWave;
constexpr int kLastThreads = 1024;                // launch 4
constexpr int kPerLane = 8;                       // logits a lane
constexpr int kChunk = kWave * kPerLane;          // tokens of a chunk
constexpr int kBins = 1024;
constexpr int kList = 8192;                       // tokens of a row's list
constexpr int kMaxParts = 64;                     // of a row
constexpr int64_t kMaxRows = 512;                 // of a launch
constexpr double kLog2e = 1.4426950408889634;
constexpr double kLn2 = 0.6931471805599453;
constexpr double kFar = 64.0;                     // a z from which on a weight is 0

struct Part {            // of a row's logits
    float top, low;      // of those above minus infinity
    int some;            // how many these are
    int bad;             // a NaN or an infinity among them
};

struct RowState {
    u64 all;             // sum of the weights
    unsigned listed;     // tokens that belong to the list
    int near;            // tokens that min-p keeps
    // where the prefixes end, from the histogram
    u64 w_k, w_p;        // weights before bin_k, before bin_p
    int n_k, n_p;        // tokens there
    int bin_k;           // bin in which top-k ends (kBins: it is off)
    int bin_p, bin_p1;   // first and last bin in which top-p may end (kBins, -1: it is off)
    int sure;            // tokens of bins before it are kept by both
};

struct Space {           // a launch's rows in the workspace
    Part* parts;         // kMaxParts a row
    RowState* rows;
    u64* weight;         // kBins a row
    int* count;          // kBins a row
    u64* list;           // kList a row
    u64* chunk;          // chunks a row
};

struct Params {
    SampleArgs a;
    Space s;
    int chunks;          // of a row
    int parts;           // of a row, and their chunks
    int part_chunks;
    int bits;            // behind the weights' point
};

size_t up(size_t n) { return (n + 255) & ~(size_t)255; }
int64_t chunks_of(int64_t V) { return (V + kChunk - 1) / kChunk; }

size_t space_of(char* ws, int64_t rows, int64_t V, Space* s) {
    size_t at = 0;
    auto take = [&](size_t n) {
        char* p = ws + at;
        at += up(n);
        return p;
    };
    char* const parts = take((size_t)rows * kMaxParts * sizeof(Part));
    char* const state = take((size_t)rows * sizeof(RowState));
    char* const weight = take((size_t)rows * kBins * 8);
    char* const count = take((size_t)rows * kBins * 4);
    char* const list = take((size_t)rows * kList * 8);
    char* const chunk = take((size_t)rows * (size_t)chunks_of(V) * 8);
    if (s)
        *s = Space{reinterpret_cast<Part*>(parts), reinterpret_cast<RowState*>(state), reinterpret_cast<u64*>(weight),
                   reinterpret_cast<int*>(count),  reinterpret_cast<u64*>(list),       reinterpret_cast<u64*>(chunk)};
    return at;
}

// What one row asks for.
struct Ask {
    double heat;         // log2(e) / temperature
    int k;               // 0: off
    float p;
    float floor;         // min-p
    double far;          // the z up to which min-p keeps
    float u;
    bool right;          // parameters within their ranges
};
__device__ __forceinline__ Ask ask_of(const SampleArgs& a, int64_t t) {
    Ask q;
    const float temperature = a.temperature ? a.temperature[t] : 1.0f;
    q.k = a.top_k ? a.top_k[t] : 0;
    q.p = a.top_p ? a.top_p[t] : 1.0f;
    q.floor = a.min_p ? a.min_p[t] : 0.0f;
    q.u = a.u[t];
    q.right = temperature >= 0.0f && temperature < __builtin_inff() && q.k >= 0 && q.p >= 0.0f && q.p <= 1.0f &&
              q.floor >= 0.0f && q.floor <= 1.0f && q.u >= 0.0f && q.u < 1.0f;
    // temperature 0: the first of the largest logits
    if (temperature == 0.0f) q.k = 1;
    q.heat = kLog2e / (temperature == 0.0f ? 1.0 : (double)temperature);
    q.far = q.floor > 0.0f ? -log2((double)q.floor) : 1e300;
    return q;
}

// What is known of a row after launch 1.
struct Row {
    Ask ask;
    double top;
    double scale;        // bins a unit of z
    int some;
    bool fine;           // there is something to draw from
};
__device__ __forceinline__ Row row_of(const Params& p, int64_t t, int r) {
    Row x;
    x.ask = ask_of(p.a, t);
    float top = -__builtin_inff(), low = __builtin_inff();
    int some = 0, bad = 0;
    for (int c = threadIdx.x & (kWave - 1); c < p.parts; c += kWave) {
        const Part q = p.s.parts[(int64_t)r * kMaxParts + c];
        top = fmaxf(top, q.top);
        low = fminf(low, q.low);
        some += q.some;
        bad |= q.bad;
    }
    top = wave_all(top, [](float x, float y) { return fmaxf(x, y); });
    low = wave_all(low, [](float x, float y) { return fminf(x, y); });
    x.some = wave_all(some, [](int x, int y) { return x + y; });
    bad = wave_all(bad, [](int x, int y) { return x | y; });
    x.fine = x.ask.right && !bad && x.some > 0;
    x.top = top;
    const double span = fmin(((double)top - (double)low) * x.ask.heat, (double)p.bits + 1.0);
    x.scale = x.fine && span > 0.0 ? kBins / span : 0.0;
    return x;
}
__device__ __forceinline__ double z_of(const Row& x, float l) { return fmin((x.top - (double)l) * x.ask.heat, kFar); }
__device__ __forceinline__ int bin_of(const Row& x, double z) { return min(kBins - 1, (int)(z * x.scale)); }

// 2^-z in fixed point.  2^f for |f| <= 1/2 is the sum of (f ln 2)^n / n!, whose
// terms from the 13th on are below 2^-52; adding 2^52 leaves the integer in the
// low bits of the fp64 number, rounded to nearest.
__device__ __forceinline__ u64 weight_of(double z, int bits) {
    const double k = rint(-z);
    const double y = (-z - k) * kLn2;
    double e = 1.0 / 479001600.0;
    e = fma(e, y, 1.0 / 39916800.0);
    e = fma(e, y, 1.0 / 3628800.0);
    e = fma(e, y, 1.0 / 362880.0);
    e = fma(e, y, 1.0 / 40320.0);
    e = fma(e, y, 1.0 / 5040.0);
    e = fma(e, y, 1.0 / 720.0);
    e = fma(e, y, 1.0 / 120.0);
    e = fma(e, y, 1.0 / 24.0);
    e = fma(e, y, 1.0 / 6.0);
    e = fma(e, y, 0.5);
    e = fma(e, y, 1.0);
    e = fma(e, y, 1.0);
    const double v = ldexp(e, (int)k + bits) + 4503599627370496.0;
    return (u64)__double_as_longlong(v) & 0xFFFFFFFFFFFFFull;
}

// Place of a token in falling order: its logit, turned so that larger ones have
// smaller numbers, then its index.
__device__ __forceinline__ uint32_t fall_of(float l) {
    const uint32_t b = __float_as_uint(l == 0.0f ? 0.0f : l);     // both zeros are one
    return b & 0x80000000u ? b : ~(b | 0x80000000u);
}
__device__ __forceinline__ u64 place_of(float l, uint32_t i) { return (u64)fall_of(l) << 32 | i; }
__device__ __forceinline__ float logit_of(u64 place) {
    const uint32_t f = (uint32_t)(place >> 32);
    return __uint_as_float(f & 0x80000000u ? f : ~f & 0x7FFFFFFFu);
}

// Eight logits from an index on (a multiple of 8); minus infinity past the row.
template <typename T>
__device__ __forceinline__ void load8(const T* l, int64_t i, int64_t V, float (&x)[kPerLane]) {
    if (i + kPerLane <= V) {
#pragma unroll
        for (int q = 0; q < kPerLane / kChunkElems<T>; ++q) {
            const u32x4_t w = *reinterpret_cast<const u32x4_t*>(l + i + q * kChunkElems<T>);
#pragma unroll
            for (int e = 0; e < kChunkElems<T>; ++e) x[q * kChunkElems<T> + e] = elem<T>(w, e);
        }
    } else {
#pragma unroll
        for (int e = 0; e < kPerLane; ++e)
            x[e] = i + e < V ? load_elem(l, i + e, sizeof(T) == 2) : -__builtin_inff();
    }
}

__device__ __forceinline__ u64 wave_sum(u64 x) {
    return wave_all(x, [](u64 a, u64 b) { return a + b; });
}

// Inclusive sums over the threads of a block, and their total.  red: a slot a wave.
template <int kN, typename V>
__device__ __forceinline__ V block_scan(V x, V* red, V& total) {
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
#pragma unroll
    for (int m = 1; m < kWave; m <<= 1) {
        const V y = __shfl_up(x, m);
        if (lane >= m) x += y;
    }
    __syncthreads();
    if (lane == kWave - 1) red[wave] = x;
    __syncthreads();
    V before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kN / kWave; ++w) {
        if (w < wave) before += red[w];
        total += red[w];
    }
    return before + x;
}
template <int kN, typename V>
__device__ __forceinline__ V block_sum(V x, V* red) {
    V total;
    block_scan<kN>(x, red, total);
    return total;
}

// ---------------------------------------------------------------------------
// launches 1 to 3: part blockIdx.x of row blockIdx.y
// ---------------------------------------------------------------------------

template <typename T>
__global__ __launch_bounds__(kThreads) void ember_sample_range(Params p, int64_t t0) {
    __shared__ float redf[kWavesB];
    __shared__ int redi[kWavesB];
    const int c = blockIdx.x, r = blockIdx.y;
    const T* const l = static_cast<const T*>(p.a.L) + (t0 + r) * p.a.ldl;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x & (kWave - 1);
    // what launches 2 and 3 add to
    const int share = (kBins + p.parts - 1) / p.parts;
    for (int b = c * share + threadIdx.x; b < min((c + 1) * share, kBins); b += kThreads) {
        p.s.weight[(int64_t)r * kBins + b] = 0;
        p.s.count[(int64_t)r * kBins + b] = 0;
    }
    if (c == 0 && threadIdx.x == 0) {
        RowState& s = p.s.rows[r];
        s.all = 0;
        s.listed = 0;
        s.near = 0;
    }
    float top = -__builtin_inff(), low = __builtin_inff();
    int some = 0, bad = 0;
    const int end = min((c + 1) * p.part_chunks, p.chunks);
    for (int j = c * p.part_chunks + wave; j < end; j += kWavesB) {
        float x[kPerLane];
        load8(l, (int64_t)j * kChunk + lane * kPerLane, p.a.V, x);
#pragma unroll
        for (int e = 0; e < kPerLane; ++e) {
            const bool is = x[e] != -__builtin_inff();
            bad |= !(x[e] < __builtin_inff());
            top = fmaxf(top, x[e]);
            low = is ? fminf(low, x[e]) : low;
            some += is;
        }
    }
    top = row_all<kThreads>(top, [](float x, float y) { return fmaxf(x, y); }, redf);
    some = row_all<kThreads>(some, [](int x, int y) { return x + y; }, redi);
    __syncthreads();
    low = row_all<kThreads>(low, [](float x, float y) { return fminf(x, y); }, redf);
    bad = row_all<kThreads>(bad, [](int x, int y) { return x | y; }, redi);
    if (threadIdx.x == 0) p.s.parts[(int64_t)r * kMaxParts + c] = Part{top, low, some, bad};
}

__device__ __forceinline__ bool ranked(const Ask& q) { return q.k > 0 || q.p < 1.0f; }   // a histogram is needed

template <typename T>
__global__ __launch_bounds__(kThreads) void ember_sample_weights(Params p, int64_t t0) {
    __shared__ u64 weight[kBins];
    __shared__ int count[kBins];
    __shared__ u64 red[kWavesB];
    __shared__ int redi[kWavesB];
    const int c = blockIdx.x, r = blockIdx.y;
    const T* const l = static_cast<const T*>(p.a.L) + (t0 + r) * p.a.ldl;
    const Row row = row_of(p, t0 + r, r);
    if (!row.fine) return;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x & (kWave - 1);
    const bool hist = ranked(row.ask);
    if (hist) {
        for (int b = threadIdx.x; b < kBins; b += kThreads) {
            weight[b] = 0;
            count[b] = 0;
        }
        __syncthreads();
    }
    u64 all = 0;
    int near = 0;
    const int end = min((c + 1) * p.part_chunks, p.chunks);
    for (int j = c * p.part_chunks + wave; j < end; j += kWavesB) {
        float x[kPerLane];
        load8(l, (int64_t)j * kChunk + lane * kPerLane, p.a.V, x);
        u64 sum = 0;
#pragma unroll
        for (int e = 0; e < kPerLane; ++e) {
            const double z = z_of(row, x[e]);
            const u64 w = weight_of(z, p.bits);
            sum += w;
            near += x[e] != -__builtin_inff() && z <= row.ask.far;
            if (hist && w) {
                const int b = bin_of(row, z);
                atomicAdd(&weight[b], w);
                atomicAdd(&count[b], 1);
            }
        }
        sum = wave_sum(sum);
        if (lane == 0) p.s.chunk[(int64_t)r * p.chunks + j] = sum;
        all += sum;
    }
    all = block_sum<kThreads>(lane == 0 ? all : 0, red);
    near = block_sum<kThreads>(near, redi);
    if (threadIdx.x == 0) {
        atomicAdd(&p.s.rows[r].all, all);
        atomicAdd(&p.s.rows[r].near, near);
    }
    if (hist) {   // past the barriers of the sums
        for (int b = threadIdx.x; b < kBins; b += kThreads) {
            if (count[b]) {
                atomicAdd(&p.s.weight[(int64_t)r * kBins + b], weight[b]);
                atomicAdd(&p.s.count[(int64_t)r * kBins + b], count[b]);
            }
        }
    }
}

// The row's p-th part of a sum: what comes before a token that top-p keeps is below it.
__device__ __forceinline__ u64 part_of(u64 total, float p) { return (u64)ceil((double)total * (double)p); }

template <typename T>
__global__ __launch_bounds__(kThreads) void ember_sample_list(Params p, int64_t t0) {
    __shared__ u64 red[kWavesB];
    __shared__ int redi[kWavesB];
    __shared__ RowState found;
    const int c = blockIdx.x, r = blockIdx.y;
    const T* const l = static_cast<const T*>(p.a.L) + (t0 + r) * p.a.ldl;
    const Row row = row_of(p, t0 + r, r);
    const bool hist = ranked(row.ask);
    if (!row.fine || (!hist && row.ask.floor == 0.0f)) return;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x & (kWave - 1);

    if (threadIdx.x == 0) {
        found.bin_k = found.bin_p = kBins;
        found.bin_p1 = -1;
        found.w_k = found.w_p = 0;
        found.n_k = found.n_p = 0;
    }
    if (hist) {
        constexpr int kOwn = kBins / kThreads;     // bins a thread
        u64 w[kOwn], sw = 0;
        int n[kOwn], sn = 0;
#pragma unroll
        for (int q = 0; q < kOwn; ++q) {
            w[q] = p.s.weight[(int64_t)r * kBins + threadIdx.x * kOwn + q];
            n[q] = p.s.count[(int64_t)r * kBins + threadIdx.x * kOwn + q];
            sw += w[q];
            sn += n[q];
        }
        u64 all;
        int positive;
        const u64 w0 = block_scan<kThreads>(sw, red, all) - sw;    // before this thread's bins
        const int n0 = block_scan<kThreads>(sn, redi, positive) - sn;
        // top-k ends in the bin in which the count reaches k
        const int k = row.ask.k;
        const bool has_k = k > 0 && k < positive;
        if (has_k) {
            u64 wb = w0;
            int nb = n0;
#pragma unroll
            for (int q = 0; q < kOwn; ++q) {
                if (nb < k && nb + n[q] >= k) {
                    found.bin_k = threadIdx.x * kOwn + q;
                    found.w_k = wb;
                    found.n_k = nb;
                    red[0] = wb + w[q];
                }
                wb += w[q];
                nb += n[q];
            }
        }
        __syncthreads();
        // top-p ends between where it would with the smallest and the largest sum that top-k may keep
        if (row.ask.p < 1.0f) {
            const u64 least = part_of(has_k ? found.w_k : all, row.ask.p), most = part_of(has_k ? red[0] : all, row.ask.p);
            u64 wb = w0;
            int nb = n0;
#pragma unroll
            for (int q = 0; q < kOwn; ++q) {
                const int b = threadIdx.x * kOwn + q;
                if ((wb < least && wb + w[q] >= least) || (b == 0 && least == 0)) {
                    found.bin_p = b;
                    found.w_p = wb;
                    found.n_p = nb;
                }
                if ((wb < most && wb + w[q] >= most) || (b == 0 && most == 0)) found.bin_p1 = b;
                wb += w[q];
                nb += n[q];
            }
        }
        __syncthreads();
    } else {
        __syncthreads();
    }
    const int bin_k = found.bin_k, bin_p = found.bin_p, bin_p1 = found.bin_p1;
    const int sure = min(bin_k, bin_p);
    RowState& s = p.s.rows[r];
    if (c == 0 && threadIdx.x == 0) {
        s.w_k = found.w_k;
        s.w_p = found.w_p;
        s.n_k = found.n_k;
        s.n_p = found.n_p;
        s.bin_k = bin_k;
        s.bin_p = bin_p;
        s.bin_p1 = bin_p1;
        s.sure = sure;
    }
    const int end = min((c + 1) * p.part_chunks, p.chunks);
    for (int j = c * p.part_chunks + wave; j < end; j += kWavesB) {
        float x[kPerLane];
        const int64_t i = (int64_t)j * kChunk + lane * kPerLane;
        load8(l, i, p.a.V, x);
        u64 sum = 0;
#pragma unroll
        for (int e = 0; e < kPerLane; ++e) {
            const double z = z_of(row, x[e]);
            const int b = bin_of(row, z);
            if (b < sure) {
                if (z <= row.ask.far) sum += weight_of(z, p.bits);
            } else if ((b == bin_k || (b >= bin_p && b <= bin_p1)) && weight_of(z, p.bits)) {
                const unsigned at = atomicAdd(&s.listed, 1u);
                if (at < (unsigned)kList) p.s.list[(int64_t)r * kList + at] = place_of(x[e], (uint32_t)(i + e));
            }
        }
        sum = wave_sum(sum);
        if (lane == 0) p.s.chunk[(int64_t)r * p.chunks + j] = sum;
    }
}

// ---------------------------------------------------------------------------
// launch 4: row blockIdx.x
// ---------------------------------------------------------------------------

// Tokens up to a place in falling order, or (weights) their weights.
template <bool kWeights, typename T>
__device__ u64 up_to(const Params& p, const Row& row, const T* l, u64 place, u64* red) {
    u64 sum = 0;
    for (int64_t i = threadIdx.x * kPerLane; i < p.a.V; i += kLastThreads * kPerLane) {
        float x[kPerLane];
        load8(l, i, p.a.V, x);
#pragma unroll
        for (int e = 0; e < kPerLane; ++e) {
            if (x[e] != -__builtin_inff() && place_of(x[e], (uint32_t)(i + e)) <= place)
                sum += kWeights ? weight_of(z_of(row, x[e]), p.bits) : 1;
        }
    }
    return block_sum<kLastThreads>(sum, red);
}

// The first place up to which there is `need`, 1 at least, by halving: the logit, then the index.
template <bool kWeights, typename T>
__device__ u64 reach(const Params& p, const Row& row, const T* l, u64 need, u64* red) {
    u64 low = 0, high = ~(u64)0;      // the answer is in [low, high]
    for (int half = 0; half < 2; ++half) {
        // logits first: places that end in all ones
        const u64 fine = half == 0 ? 0xFFFFFFFFull : 0;
        while ((low | fine) < (high | fine)) {
            const u64 mid = (low + (high - low) / 2) | fine;
            if (up_to<kWeights>(p, row, l, mid, red) >= need) high = mid;
            else low = mid + 1;
        }
        if (half == 0) {
            low = high & ~0xFFFFFFFFull;
            high = low | (uint32_t)(p.a.V - 1);
        }
    }
    return high;
}

template <typename T>
__global__ __launch_bounds__(kLastThreads) void ember_sample_draw(Params p, int64_t t0) {
    __shared__ u64 entry[kList];
    __shared__ u64 red[kLastThreads / kWave];
    __shared__ int redi[kLastThreads / kWave];
    __shared__ u64 found_at;
    __shared__ u64 found_before;
    const int r = blockIdx.x;
    const int64_t t = t0 + r;
    const T* const l = static_cast<const T*>(p.a.L) + t * p.a.ldl;
    const Row row = row_of(p, t, r);
    if (!row.fine) {
        if (threadIdx.x == 0) {
            p.a.ids[t] = -1;
            if (p.a.logp) p.a.logp[t] = __uint_as_float(0x7FC00000u);
            if (p.a.kept) p.a.kept[t] = 0;
        }
        return;
    }
    const bool hist = ranked(row.ask), floored = row.ask.floor > 0.0f;
    u64* const chunk = p.s.chunk + (int64_t)r * p.chunks;
    const RowState& s = p.s.rows[r];
    u64 last = 0;                     // the last place that is kept, where the bins alone do not say it
    int sure = kBins;                 // tokens of bins before it are kept
    int kept = row.some;              // before min-p
    if (hist) {
        sure = s.sure;
        const int k = row.ask.k > 0 ? min(row.ask.k, row.some) : row.some;
        kept = k;
        const bool has_k = s.bin_k < kBins, has_p = s.bin_p < kBins;
        const int n = (int)min(s.listed, (unsigned)kList + 1);
        if (n > kList) {
            // too many for the list: search the row, then sum its chunks again
            last = ~(u64)0;
            u64 total = s.all;
            if (has_k) {
                last = reach<false>(p, row, l, (u64)row.ask.k, red);
                total = up_to<true>(p, row, l, last, red);
            }
            if (has_p) {
                const u64 need = part_of(total, row.ask.p);
                last = min(last, reach<true>(p, row, l, need > 0 ? need : 1, red));
                kept = (int)up_to<false>(p, row, l, last, red);
            }
            const int wave = threadIdx.x / kWave, lane = threadIdx.x & (kWave - 1);
            for (int j = wave; j < p.chunks; j += kLastThreads / kWave) {
                float x[kPerLane];
                const int64_t i = (int64_t)j * kChunk + lane * kPerLane;
                load8(l, i, p.a.V, x);
                u64 sum = 0;
#pragma unroll
                for (int e = 0; e < kPerLane; ++e) {
                    const double z = z_of(row, x[e]);
                    if (place_of(x[e], (uint32_t)(i + e)) <= last && z <= row.ask.far) sum += weight_of(z, p.bits);
                }
                sum = wave_sum(sum);
                if (lane == 0) __hip_atomic_store(&chunk[j], sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            sure = 0;
            __threadfence();
        } else if (n > 0) {
            int n2 = 2;
            while (n2 < n) n2 *= 2;
            for (int i = threadIdx.x; i < n2; i += kLastThreads)
                entry[i] = i < n ? p.s.list[(int64_t)r * kList + i] : ~(u64)0;
            __syncthreads();
            for (int size = 2; size <= n2; size *= 2) {
                for (int step = size / 2; step > 0; step /= 2) {
                    for (int q = threadIdx.x; q < n2 / 2; q += kLastThreads) {
                        const int i = (q / step) * 2 * step + q % step, j = i + step;
                        const u64 x = entry[i], y = entry[j];
                        if ((x > y) == ((i & size) == 0)) {
                            entry[i] = y;
                            entry[j] = x;
                        }
                    }
                    __syncthreads();
                }
            }
            // this thread's entries and their weights
            constexpr int kOwn = kList / kLastThreads;
            u64 w[kOwn], w_list = 0, w_k = 0;
            int bin[kOwn], before_k = 0;
#pragma unroll
            for (int q = 0; q < kOwn; ++q) {
                const int i = threadIdx.x * kOwn + q;
                const double z = i < n ? z_of(row, logit_of(entry[i])) : kFar;
                w[q] = i < n ? weight_of(z, p.bits) : 0;
                bin[q] = i < n ? bin_of(row, z) : kBins;
                before_k += bin[q] < s.bin_k;
                w_list += w[q];
            }
            int first_k = n, end_k = n;       // of the list: bin_k's first entry, and the first that top-k drops
            u64 total = s.all;
            if (has_k) {
                first_k = block_sum<kLastThreads>(before_k, redi);
                end_k = min(n, first_k + (row.ask.k - s.n_k));
#pragma unroll
                for (int q = 0; q < kOwn; ++q) {
                    const int i = threadIdx.x * kOwn + q;
                    if (i >= first_k && i < end_k) w_k += w[q];
                }
                total = s.w_k + block_sum<kLastThreads>(w_k, red);
            }
            int take = has_k ? end_k : 0;     // entries that are kept
            if (has_p) {
                const u64 need = part_of(total, row.ask.p);
                u64 all;
                u64 before = s.w_p + block_scan<kLastThreads>(w_list, red, all) - w_list;
                int mine = 0;
#pragma unroll
                for (int q = 0; q < kOwn; ++q) {
                    const int i = threadIdx.x * kOwn + q;
                    // the largest logit is kept whatever top-p is
                    mine += i < end_k && bin[q] <= s.bin_p1 && (before < need || (i == 0 && s.n_p == 0));
                    before += w[q];
                }
                take = block_sum<kLastThreads>(mine, redi);
                kept = s.n_p + take;
            }
            if (take > 0) last = entry[take - 1];
            // the kept entries join their chunks' sums
            __syncthreads();
#pragma unroll
            for (int q = 0; q < kOwn; ++q) {
                const int i = threadIdx.x * kOwn + q;
                if (i < take && z_of(row, logit_of(entry[i])) <= row.ask.far)
                    atomicAdd(&chunk[(uint32_t)entry[i] / kChunk], w[q]);
            }
            __threadfence();
        }
        __syncthreads();
    }
    if (floored) kept = min(kept, s.near);

    // the chunk in which u falls
    auto sum_of = [&](int64_t j) { return __hip_atomic_load(&chunk[j], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
    const int own = (p.chunks + kLastThreads - 1) / kLastThreads, j0 = threadIdx.x * own, j1 = min(j0 + own, p.chunks);
    u64 sum = 0, total;
    for (int j = j0; j < j1; ++j) sum += sum_of(j);
    u64 before = block_scan<kLastThreads>(sum, red, total) - sum;
    const u64 target = (u64)((double)total * (double)row.ask.u);
    if (before <= target && target < before + sum) {
        int j = j0;
        for (; j < j1 - 1; ++j) {
            const u64 x = sum_of(j);
            if (target < before + x) break;
            before += x;
        }
        found_at = j;
        found_before = before;
    }
    __syncthreads();
    // and the token: one a thread
    const int64_t i = (int64_t)found_at * kChunk + threadIdx.x;
    const u64 base = found_before;
    u64 w = 0;
    double z = 0.0;
    if (threadIdx.x < kChunk && i < p.a.V) {
        const float x = load_elem(l, i, sizeof(T) == 2);
        z = z_of(row, x);
        const bool keep = bin_of(row, z) < sure || place_of(x, (uint32_t)i) <= last;
        if (keep && z <= row.ask.far) w = weight_of(z, p.bits);
    }
    u64 in_chunk;
    const u64 end = base + block_scan<kLastThreads>(w, red, in_chunk);
    if (end - w <= target && target < end) {
        p.a.ids[t] = i;
        if (p.a.logp) p.a.logp[t] = (float)((p.bits - z) * kLn2 - log((double)s.all));
        if (p.a.kept) p.a.kept[t] = kept;
    }
}

template <typename T>
hipError_t launch(const Params& p, int64_t t0, int rows, bool list, hipStream_t s) {
    const dim3 grid((unsigned)p.parts, (unsigned)rows);
    ember_sample_range<T><<<grid, kThreads, 0, s>>>(p, t0);
    ember_sample_weights<T><<<grid, kThreads, 0, s>>>(p, t0);
    if (list) ember_sample_list<T><<<grid, kThreads, 0, s>>>(p, t0);
    ember_sample_draw<T><<<rows, kLastThreads, 0, s>>>(p, t0);
    return hipGetLastError();
}

} // namespace

size_t sample_ws_bytes(int64_t T, int64_t V) { return space_of(nullptr, std::min(T, kMaxRows), V, nullptr); }

hipError_t launch_sample(const SampleArgs& a, hipStream_t s) {
    Params p;
    p.a = a;
    const int64_t rows = std::min(a.T, kMaxRows);
    space_of(a.ws, rows, a.V, &p.s);
    p.chunks = (int)chunks_of(a.V);
    int width = 0;
    while (((int64_t)1 << width) < a.V) ++width;
    p.bits = std::min(48, 62 - width);
    // about 1024 blocks, of a chunk a wave at least
    const int64_t want = std::min<int64_t>({(1024 + rows - 1) / rows, (p.chunks + kWavesB - 1) / kWavesB, kMaxParts});
    p.part_chunks = (int)((p.chunks + want - 1) / want);
    p.parts = (p.chunks + p.part_chunks - 1) / p.part_chunks;
    const bool list = a.top_k || a.top_p || a.min_p || a.temperature;
    for (int64_t t0 = 0; t0 < a.T; t0 += kMaxRows) {
        const int n = (int)std::min(kMaxRows, a.T - t0);
        const hipError_t e = a.l_dtype == EMBER_F32 ? launch<float>(p, t0, n, list, s) : launch<uint16_t>(p, t0, n, list, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

} // namespace ember
