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
// by index), so what is kept is the shortest of three prefixes, and one place (logit
// and index in one number) says where it ends.  The token is then the one at which
// the running sum, by index, of the kept weights passes u times their sum.
//
// Rows of up to 8192 tokens: one launch, a block a row, which holds it in registers.
// Longer ones take four:
//   1  the largest and smallest logit of each part of a row, and, for a row that has a
//      filter, the largest of every chunk of 1024 tokens;
//   2  weights and their sum, of every chunk where no filter is on, and, where top-k or
//      top-p is, a histogram over z of counts and weights;
//   3  from the histogram the bins in which the prefixes end: their tokens go to
//      a list; for every chunk the sum of the tokens before them;
//   4  a block a row finds the prefix's end among the listed, the chunk in which
//      the random number falls, and in it the token.
// In the bin an end is found by rank where few tokens are there, or else by histograms over
// the places, each over one bin of the last: of the listed, or, where they do not fit
// (thousands of equal logits at a prefix's end), of the whole row.  (Histograms over places
// alone have most of their bins about 0, where floats are dense: 256 rows of 8192 with top-k
// and top-p take 20 us, and 31 so.)
//
// Bound by: a short row by one block's chain of latencies (8 us for 64 logits as for 8191, 9 for 256 such rows: by clocks
// kept along the way a third goes to the joined range and the row's parameters in fp64, an eighth to the logits' loads, a
// fifth to the last token with its logarithm, a sixth to the two sums over the block and their barriers), with filters
// by that of finding the ends (17 to 23 us, 1 or 256 rows); few long rows by the chain of the four launches (16 x 128256
// bf16: 4 + 9 + 8 + 11 us); many by HBM in launch 1 (256 x 128256 fp32: 23 us, 5.8 TB/s), the vector units and LDS
// atomics in 2 (41 us: 70% and 40% busy), loads and the rows that keep the most tokens in 3 (37 to 40 us; 4 takes 13).

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
constexpr int kRowThreads = 1024;                 // a block that has a row
constexpr int kPerLane = 8;                       // logits a lane
constexpr int kSub = kWave * kPerLane;            // tokens of a wave's loads
constexpr int kChunk = 2 * kSub;                  // and of a chunk
constexpr int kBins = 1024;
constexpr int kList = 8192;                       // tokens of a row's list
constexpr int kPartList = 1280;                   // of a part's (launch 3: four blocks a compute unit)
constexpr int kRanked = kWave;                    // candidates that a wave ranks
constexpr int kMaxParts = 64;                     // of a row
constexpr int64_t kMaxRows = 512;                 // of a launch
constexpr int64_t kOneBlock = kRowThreads * kPerLane;   // tokens of a row that a block holds
constexpr size_t kLeastBytes = 4096;              // of a workspace
constexpr int kSteps = 32;                        // of a halving of the weight: z counts these
constexpr double kLog2e = 1.4426950408889634;
constexpr double kLn2 = 0.6931471805599453;
constexpr double kFar = 64.0 * kSteps;            // a z from which on a weight is 0
constexpr double kWhole = 6755399441055744.0;     // 1.5 * 2^52: numbers about it are whole
static_assert(kBins == kRowThreads, "a bin a thread");

struct Part {            // of a row's logits
    float top, low;      // of those above minus infinity
    int some;            // how many these are
    int bad;             // a NaN or an infinity among them
};

struct Bins {            // where the prefixes end, from a row's histogram
    u64 w_k, w_p;        // weights before bin_k, before bin_p
    int n_k, n_p;        // tokens there
    int in_k, to_p;      // tokens in bin_k; up to bin_p1's end
    int bin_k;           // bin in which top-k ends (kBins: it is off)
    int bin_p, bin_p1;   // first and last bin in which top-p may end (kBins, -1: it is off)
};

struct RowState {
    u64 all;             // sum of the weights
    unsigned listed;     // tokens that belong to the list
    int near;            // tokens that min-p keeps
    Bins bins;
};

struct Space {           // a launch's rows in the workspace
    Part* parts;         // kMaxParts a row
    RowState* rows;
    u64* weight;         // kBins a row
    int* count;          // kBins a row
    u64* list;           // kList a row
    u64* chunk;          // chunks a row: sums of weights
    float* peak;         // chunks a row: largest logits
};

struct Params {
    SampleArgs a;
    Space s;
    int chunks;          // of a row
    int parts;           // of a row, and their chunks
    int part_chunks;
    int weight_chunks;   // of a block of launch 2
    int bits;            // behind the weights' point
    int width;           // bits of an index
    bool list;           // a row may have a filter: launch 3
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
    char* const peak = take((size_t)rows * (size_t)chunks_of(V) * 4);
    if (s)
        *s = Space{reinterpret_cast<Part*>(parts), reinterpret_cast<RowState*>(state), reinterpret_cast<u64*>(weight),
                   reinterpret_cast<int*>(count),  reinterpret_cast<u64*>(list),       reinterpret_cast<u64*>(chunk),
                   reinterpret_cast<float*>(peak)};
    return at;
}

// The value of another lane of the row of 16, or of an earlier row's end; `none` where there is none.
template <int kCtrl, int kRows>
__device__ __forceinline__ int from_lane(int x, int none) {
    return __builtin_amdgcn_update_dpp(none, x, kCtrl, kRows, 0xF, false);
}
template <int kCtrl, int kRows>
__device__ __forceinline__ float from_lane(float x, float none) {
    return __int_as_float(from_lane<kCtrl, kRows>(__float_as_int(x), __float_as_int(none)));
}
template <int kCtrl, int kRows>
__device__ __forceinline__ u64 from_lane(u64 x, u64 none) {
    const uint32_t lo = (uint32_t)from_lane<kCtrl, kRows>((int)(uint32_t)x, (int)(uint32_t)none);
    const uint32_t hi = (uint32_t)from_lane<kCtrl, kRows>((int)(uint32_t)(x >> 32), (int)(uint32_t)(none >> 32));
    return (u64)hi << 32 | lo;
}
// Inclusive sums over a wave: shifts by 1, 2, 4 and 8 within rows of 16 lanes, then the
// sums of the row before and of the half before.  (Exchanges through the LDS took most
// of launch 4's time.)
template <typename V>
__device__ __forceinline__ V wave_scan(V x) {
    x += from_lane<0x111, 0xF>(x, (V)0);
    x += from_lane<0x112, 0xF>(x, (V)0);
    x += from_lane<0x114, 0xF>(x, (V)0);
    x += from_lane<0x118, 0xF>(x, (V)0);
    x += from_lane<0x142, 0xA>(x, (V)0);
    x += from_lane<0x143, 0xC>(x, (V)0);
    return x;
}
__device__ __forceinline__ int last_lane(int x) { return __builtin_amdgcn_readlane(x, kWave - 1); }
__device__ __forceinline__ float last_lane(float x) { return __int_as_float(last_lane(__float_as_int(x))); }
__device__ __forceinline__ u64 last_lane(u64 x) {
    return (u64)(uint32_t)last_lane((int)(uint32_t)(x >> 32)) << 32 | (uint32_t)last_lane((int)(uint32_t)x);
}
template <typename V>
__device__ __forceinline__ V wave_sum(V x) { return last_lane(wave_scan(x)); }
// The result over a wave of an operation for which twice the same is once, such as a maximum.
template <typename V, typename Op>
__device__ __forceinline__ V wave_one(V x, Op op) {
    x = op(x, from_lane<0x111, 0xF>(x, x));
    x = op(x, from_lane<0x112, 0xF>(x, x));
    x = op(x, from_lane<0x114, 0xF>(x, x));
    x = op(x, from_lane<0x118, 0xF>(x, x));
    x = op(x, from_lane<0x142, 0xA>(x, x));
    x = op(x, from_lane<0x143, 0xC>(x, x));
    return last_lane(x);
}

// What one row asks for.
struct Ask {
    double heat;         // steps of z a unit of logit
    double cool;         // and units of logit a step
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
    const double by = temperature == 0.0f ? 1.0 : (double)temperature;
    q.heat = kSteps * kLog2e / by;
    q.cool = by * (1.0 / (kSteps * kLog2e));
    q.far = q.floor > 0.0f ? -kSteps * log2((double)q.floor) : 1e300;
    return q;
}

// What is known of a row once its range is.
struct Row {
    Ask ask;
    double top;
    double reach;        // logits further below the largest count as this far
    double none;         // and from here on have no weight
    double scale;        // bins a unit of logit
    int some;
    bool fine;           // there is something to draw from
};
// The same in all lanes: kept in scalar registers.
__device__ __forceinline__ double uniform(double x) {
    const u64 b = (u64)__double_as_longlong(x);
    const uint32_t lo = __builtin_amdgcn_readfirstlane((int)(uint32_t)b);
    const uint32_t hi = __builtin_amdgcn_readfirstlane((int)(uint32_t)(b >> 32));
    return __longlong_as_double((long long)((u64)hi << 32 | lo));
}
__device__ __forceinline__ Row row_of(const Params& p, int64_t t, const Part& q) {
    Row x;
    x.ask = ask_of(p.a, t);
    x.ask.heat = uniform(x.ask.heat);
    x.ask.far = uniform(x.ask.far);
    x.some = __builtin_amdgcn_readfirstlane(q.some);
    x.fine = __builtin_amdgcn_readfirstlane(x.ask.right && !q.bad && q.some > 0);
    x.top = uniform(q.top);
    x.reach = uniform(kFar * x.ask.cool);
    x.none = uniform((p.bits + 1.0) * kSteps * x.ask.cool);
    const double span = fmin((double)q.top - (double)q.low, x.none);
    x.scale = uniform(x.fine && span > 0.0 ? kBins * (1.0 - 0x1p-20) / span : 0.0);
    return x;
}
__device__ __forceinline__ Part join(const Part& a, const Part& b) {
    return Part{fmaxf(a.top, b.top), fminf(a.low, b.low), a.some + b.some, a.bad | b.bad};
}
__device__ __forceinline__ Part wave_join(Part x) {
    return Part{wave_one(x.top, [](float a, float b) { return fmaxf(a, b); }),
                wave_one(x.low, [](float a, float b) { return fminf(a, b); }), wave_sum(x.some),
                wave_one(x.bad, [](int a, int b) { return a | b; })};
}
template <int kN>
__device__ __forceinline__ Part block_join(Part x, Part* red) {
    x = wave_join(x);
    if ((threadIdx.x & (kWave - 1)) == 0) red[threadIdx.x / kWave] = x;
    __syncthreads();
    x = red[0];
#pragma unroll
    for (int w = 1; w < kN / kWave; ++w) x = join(x, red[w]);
    return x;
}
constexpr float kInf = __builtin_inff();
__device__ __forceinline__ void see(Part& q, float l) {
    q.bad |= !(l < kInf);
    q.top = fmaxf(q.top, l);
    q.low = l != -kInf ? fminf(q.low, l) : q.low;
    q.some += l != -kInf;
}
// Launches 2 to 4: from the parts of launch 1.
__device__ __forceinline__ Row row_at(const Params& p, int64_t t, int r) {
    const int c = threadIdx.x & (kWave - 1);
    static_assert(kMaxParts == kWave, "a part a lane");
    return row_of(p, t, wave_join(c < p.parts ? p.s.parts[(int64_t)r * kMaxParts + c] : Part{-kInf, kInf, 0, 0}));
}
// How far a logit is below the largest, z times a step, and whether min-p keeps it.
__device__ __forceinline__ double gap_of(const Row& x, float l) { return fmin(x.top - (double)l, x.reach); }
__device__ __forceinline__ bool near_of(const Row& x, float l) { return (x.top - (double)l) * x.ask.heat <= x.ask.far; }
// (up to a gap that has a weight the bins are 0 .. kBins - 1 by the scale alone)
__device__ __forceinline__ int bin_of(const Row& x, double gap) { return (int)fmin(gap * x.scale, kBins - 1.0); }

// 2^(-z / kSteps) in fixed point, z = gap heat.  With n the whole number of steps nearest -z, in
// the low bits of a sum with 1.5 * 2^52, it is the table's 2^(bits + (n mod kSteps) / kSteps), times a
// power of two, times e^(c y) with y = -z - n, |y| <= 1/2, c = ln 2 / 32, whose series' terms
// from the 7th on are below 2^-58.  Adding 2^52 leaves the integer in the low bits of the
// fp64 number, rounded to nearest.  (A table of 256 saves two terms, but its reads meet in the
// LDS banks; 32 numbers of 8 bytes lie in one each.)
__device__ __forceinline__ u64 weight_of(const Row& x, double gap, const double* table) {
    constexpr double c = kLn2 / kSteps;
    const double t = fma(gap, -x.ask.heat, kWhole);
    const double y = fma(gap, -x.ask.heat, kWhole - t);
    double e = c * c * c * c * c * c / 720.0;
    e = fma(e, y, c * c * c * c * c / 120.0);
    e = fma(e, y, c * c * c * c / 24.0);
    e = fma(e, y, c * c * c / 6.0);
    e = fma(e, y, c * c / 2.0);
    e = fma(e, y, c);
    e = fma(e, y, 1.0);
    const uint32_t n = (uint32_t)(u64)__double_as_longlong(t);
    u64 two = (u64)__double_as_longlong(table[n & (kSteps - 1)]);
    two += (u64)((n & ~(kSteps - 1u)) << 15) << 32;
    const double v = fma(e, __longlong_as_double((long long)two), 4503599627370496.0);
    return (u64)__double_as_longlong(v) & 0xFFFFFFFFFFFFFull;
}
static_assert(kSteps == 32, "a shift by 20 - 5");
__device__ __forceinline__ void fill_table(double* table, int bits) {
    if (threadIdx.x < kSteps) table[threadIdx.x] = exp2(bits + threadIdx.x * (1.0 / kSteps));
}

// Place of a token in falling order: its logit, turned so that larger ones have
// smaller numbers, then its index.
__device__ __forceinline__ uint32_t fall_of(float l) {
    const uint32_t b = __float_as_uint(l == 0.0f ? 0.0f : l);     // both zeros are one
    return b & 0x80000000u ? b : ~(b | 0x80000000u);
}
__device__ __forceinline__ float logit_of_fall(uint32_t f) { return __uint_as_float(f & 0x80000000u ? f : ~f & 0x7FFFFFFFu); }
// (of a bf16 logit's turned bits the lower half follows from the upper)
template <typename T> constexpr int kFallBits = 8 * (int)sizeof(T);
template <typename T>
__device__ __forceinline__ u64 place_of(float l, uint32_t i, int width) {
    return (u64)(fall_of(l) >> (32 - kFallBits<T>)) << width | i;
}
template <typename T>
__device__ __forceinline__ float logit_of(u64 place, int width) {
    const uint32_t f = (uint32_t)(place >> width);
    if constexpr (sizeof(T) == 4) return logit_of_fall(f);
    else return logit_of_fall(f << 16 | (f & 0x8000u ? 0u : 0xFFFFu));
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

// Inclusive sums over the threads of a block, and their total.  red: a slot a wave.
template <int kN, typename V>
__device__ __forceinline__ V block_scan(V x, V* red, V& total) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    x = wave_scan(x);
    __syncthreads();
    if ((threadIdx.x & (kWave - 1)) == kWave - 1) red[wave] = x;
    __syncthreads();
    V before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kN / kWave; ++w) {
        const V y = red[w];
        before += w < wave ? y : 0;
        total += y;
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
// where a prefix ends
// ---------------------------------------------------------------------------

struct Select {
    u64 weight[kBins];
    u64 place[kRanked];
    int count[kBins];
    u64 red[kRowThreads / kWave];
    int redi[kRowThreads / kWave];
    u64 lo, hi;                  // places among which the end is
    u64 w;                       // weights before them
    int n;                       // tokens there
    int in;                      // tokens among them, then those ranked
};
constexpr u64 kNone = ~(u64)0;   // past every place

// The first place up to which the candidates' count (or their weights) reaches
// `need`, of 1 at least and at most what there is.  each(f) calls f(place, weight) for
// the candidates of a thread, `most` of all threads at most.  Every pass makes a histogram
// over one bin of the last, until a bin holds no more than a wave ranks: a lane each,
// which goes through the others.  n, w: what there is up to the place, it included.
template <bool kWeights, typename Each>
__device__ u64 end_of(Each each, int most, u64 need, Select& s, int& n, u64& w) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x & (kWave - 1);
    u64 from = 0, to = kNone, w0 = 0;
    int n0 = 0;
    __syncthreads();
    if (most > kRanked) {
        u64 lo = kNone, hi = 0;
        each([&](u64 place, auto) {
            lo = min(lo, place);
            hi = max(hi, place);
        });
        lo = wave_one(lo, [](u64 a, u64 b) { return a < b ? a : b; });
        hi = wave_one(hi, [](u64 a, u64 b) { return a > b ? a : b; });
        if (threadIdx.x == 0) {
            s.lo = kNone;
            s.hi = 0;
        }
        s.weight[threadIdx.x] = 0;
        s.count[threadIdx.x] = 0;
        __syncthreads();
        if (lane == 0) {
            atomicMin(&s.lo, lo);
            atomicMax(&s.hi, hi);
        }
        __syncthreads();
        from = s.lo;
        to = s.hi;
        // a pass leaves ten bits less of at most 56
        for (int pass = 0; pass < 6; ++pass) {
            const u64 wide = to - from;
            const int shift = wide < kBins ? 0 : 64 - __clzll(wide) - 10;
            each([&](u64 place, auto weight) {
                if (place < from || place > to) return;
                const int b = (int)((place - from) >> shift);
                atomicAdd(&s.weight[b], weight());
                atomicAdd(&s.count[b], 1);
            });
            __syncthreads();
            const u64 wb = s.weight[threadIdx.x];
            const int nb = s.count[threadIdx.x];
            s.weight[threadIdx.x] = 0;
            s.count[threadIdx.x] = 0;
            u64 w1 = wave_scan(wb);
            int n1 = wave_scan(nb);
            if (lane == kWave - 1) {
                s.red[wave] = w1;
                s.redi[wave] = n1;
            }
            __syncthreads();
            w1 += w0;
            n1 += n0;
#pragma unroll
            for (int q = 0; q < kRowThreads / kWave; ++q) {
                w1 += q < wave ? s.red[q] : 0;
                n1 += q < wave ? s.redi[q] : 0;
            }
            const u64 before = kWeights ? w1 - wb : (u64)(n1 - nb), after = kWeights ? w1 : (u64)n1;
            if (nb > 0 && before < need && after >= need) {
                s.lo = from + ((u64)threadIdx.x << shift);
                s.hi = min(to, s.lo + (((u64)1 << shift) - 1));
                s.w = w1 - wb;
                s.n = n1 - nb;
                s.in = nb;
            }
            __syncthreads();
            from = s.lo;
            to = s.hi;
            w0 = s.w;
            n0 = s.n;
            if (s.in <= kRanked) break;
        }
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        s.lo = kNone;
        s.in = 0;
    }
    __syncthreads();
    each([&](u64 place, auto weight) {
        if (place < from || place > to) return;
        const int q = atomicAdd(&s.in, 1);
        if (q >= kRanked) return;
        s.place[q] = place;
        s.weight[q] = weight();
    });
    __syncthreads();
    if (wave == 0) {
        const int m = min(s.in, kRanked);
        const u64 at = lane < m ? s.place[lane] : 0;
        u64 before = w0;
        int rank = n0;
        for (int q = 0; q < m; ++q) {
            const bool less = s.place[q] < at;
            before += less ? s.weight[q] : 0;
            rank += less;
        }
        const u64 after = before + (lane < m ? s.weight[lane] : 0);
        if (lane < m && (kWeights ? before < need && after >= need : (u64)rank < need && (u64)rank + 1 >= need)) {
            s.lo = at;
            s.w = after;
            s.n = rank + 1;
        }
    }
    __syncthreads();
    n = s.n;
    w = s.w;
    return s.lo;
}

// The row's p-th part of a sum: what comes before a token that top-p keeps is below it.
__device__ __forceinline__ u64 part_of(u64 total, float p) { return (u64)ceil((double)total * (double)p); }
__device__ __forceinline__ bool ranked(const Ask& q) { return q.k > 0 || q.p < 1.0f; }   // an end has to be found

// The bins in which the prefixes end, from a histogram of which each of a block's kN threads
// has kBins / kN bins side by side.  In LDS after the next barrier.
template <int kN>
__device__ __forceinline__ void bins_of(const Ask& q, const u64 (&w)[kBins / kN], const int (&n)[kBins / kN], u64* red, int* redi,
                                        Bins& found) {
    constexpr int kOwn = kBins / kN;
    if (threadIdx.x == 0) found = Bins{0, 0, 0, 0, 0, 0, kBins, kBins, -1};
    u64 sw = 0, all;
    int sn = 0, positive;
#pragma unroll
    for (int o = 0; o < kOwn; ++o) {
        sw += w[o];
        sn += n[o];
    }
    const u64 w0 = block_scan<kN>(sw, red, all) - sw;        // before this thread's bins
    const int n0 = block_scan<kN>(sn, redi, positive) - sn;
    // top-k ends in the bin in which the count reaches k
    const bool has_k = q.k > 0 && q.k < positive;
    if (has_k) {
        u64 wb = w0;
        int nb = n0;
#pragma unroll
        for (int o = 0; o < kOwn; ++o) {
            if (nb < q.k && nb + n[o] >= q.k) {
                found.bin_k = threadIdx.x * kOwn + o;
                found.w_k = wb;
                found.n_k = nb;
                found.in_k = n[o];
                red[0] = wb + w[o];
            }
            wb += w[o];
            nb += n[o];
        }
    }
    __syncthreads();
    if (q.p >= 1.0f) return;
    // top-p ends between where it would with the smallest and the largest sum that top-k may keep
    const u64 least = part_of(has_k ? found.w_k : all, q.p), most = part_of(has_k ? red[0] : all, q.p);
    u64 wb = w0;
    int nb = n0;
#pragma unroll
    for (int o = 0; o < kOwn; ++o) {
        const int b = threadIdx.x * kOwn + o;
        if ((wb < least && wb + w[o] >= least) || (b == 0 && least == 0)) {
            found.bin_p = b;
            found.w_p = wb;
            found.n_p = nb;
        }
        if ((wb < most && wb + w[o] >= most) || (b == 0 && most == 0)) {
            found.bin_p1 = b;
            found.to_p = nb + n[o];
        }
        wb += w[o];
        nb += n[o];
    }
}

// The last place that is kept (kNone: all); `kept` comes as what top-k alone keeps.
// each(first, last bin, f): a thread's tokens of a weight in these, as end_of takes them.
template <typename Each>
__device__ __forceinline__ u64 last_of(const Ask& q, const Bins& b, u64 all, Each each, Select& s, int& kept) {
    u64 last = kNone, total = all, sum;
    int n;
    if (b.bin_k < kBins) {
        last = end_of<false>([&](auto f) { each(b.bin_k, b.bin_k, f); }, b.in_k, (u64)(q.k - b.n_k), s, n, sum);
        total = b.w_k + sum;
    }
    if (b.bin_p < kBins) {
        // what the bins before keep is below this part, and at bin_p1's end it is reached
        const u64 need = part_of(total, q.p);
        last = end_of<true>([&](auto f) { each(b.bin_p, b.bin_p1, f); }, b.to_p - b.n_p, need > b.w_p ? need - b.w_p : 1, s, n, sum);
        kept = b.n_p + n;
    }
    return last;
}

__device__ __forceinline__ void no_token(const SampleArgs& a, int64_t t) {
    a.ids[t] = -1;
    if (a.logp) a.logp[t] = __uint_as_float(0x7FC00000u);
    if (a.kept) a.kept[t] = 0;
}
__device__ __forceinline__ void token(const Params& p, const Row& x, int64_t t, int64_t i, float l, u64 all, int kept) {
    p.a.ids[t] = i;
    if (p.a.logp) p.a.logp[t] = (float)((p.bits - gap_of(x, l) * x.ask.heat / kSteps) * kLn2 - log((double)all));
    if (p.a.kept) p.a.kept[t] = kept;
}

// ---------------------------------------------------------------------------
// one launch: a block a row, eight tokens a thread side by side
// ---------------------------------------------------------------------------

template <typename T>
__global__ __launch_bounds__(kRowThreads) void ember_sample_row(Params p, int64_t t0) {
    __shared__ Select s;
    __shared__ Bins bins;
    __shared__ double table[kSteps];
    __shared__ Part redp[kRowThreads / kWave];
    const int64_t t = t0 + blockIdx.x;
    const T* const l = static_cast<const T*>(p.a.L) + t * p.a.ldl;
    fill_table(table, p.bits);
    s.weight[threadIdx.x] = 0;
    s.count[threadIdx.x] = 0;
    float x[kPerLane];
    Part part{-kInf, kInf, 0, 0};
    const uint32_t i0 = threadIdx.x * kPerLane;
    load8(l, i0, p.a.V, x);
#pragma unroll
    for (int e = 0; e < kPerLane; ++e) see(part, x[e]);
    const Row row = row_of(p, t, block_join<kRowThreads>(part, redp));
    if (!row.fine) {
        if (threadIdx.x == 0) no_token(p.a, t);
        return;
    }
    const bool hist = ranked(row.ask);
    u64 w[kPerLane], all = 0;
    int b[kPerLane];
    uint32_t mask = 0;                    // tokens of this thread that have a weight, then those that are kept
    int near = 0;
#pragma unroll
    for (int e = 0; e < kPerLane; ++e) {
        const double gap = gap_of(row, x[e]);
        w[e] = weight_of(row, gap, table);
        b[e] = bin_of(row, gap);
        all += w[e];
        mask |= (uint32_t)(w[e] != 0) << e;
        near += x[e] != -kInf && near_of(row, x[e]);
        if (e % 4 == 3) __builtin_amdgcn_sched_barrier(0);      // eight at once take more registers
    }
    if (hist) {
#pragma unroll
        for (int e = 0; e < kPerLane; ++e) {
            if (!w[e]) continue;
            atomicAdd(&s.weight[b[e]], w[e]);
            atomicAdd(&s.count[b[e]], 1);
        }
    }
    all = block_sum<kRowThreads>(all, s.red);
    int kept = row.some;
    if (hist) {
        const u64 own_w[1] = {s.weight[threadIdx.x]};
        const int own_n[1] = {s.count[threadIdx.x]};
        bins_of<kRowThreads>(row.ask, own_w, own_n, s.red, s.redi, bins);
        __syncthreads();
        if (row.ask.k > 0) kept = min(kept, row.ask.k);
        const auto place = [&](int e) { return place_of<T>(x[e], i0 + e, p.width); };
        const auto each = [&](int first, int last, auto f) {
#pragma unroll
            for (int e = 0; e < kPerLane; ++e)
                if ((mask >> e & 1) && b[e] >= first && b[e] <= last) f(place(e), [&] { return w[e]; });
        };
        const u64 last = last_of(row.ask, bins, all, each, s, kept);
#pragma unroll
        for (int e = 0; e < kPerLane; ++e) mask &= ~((uint32_t)(place(e) > last) << e);
    }
    if (row.ask.floor > 0.0f) {
        kept = min(kept, block_sum<kRowThreads>(near, s.redi));
#pragma unroll
        for (int e = 0; e < kPerLane; ++e) mask &= ~((uint32_t)!near_of(row, x[e]) << e);
    }
    // running sums by index
    u64 sum = 0, total;
#pragma unroll
    for (int e = 0; e < kPerLane; ++e) sum += mask >> e & 1 ? w[e] : 0;
    u64 run = block_scan<kRowThreads>(sum, s.red, total);
    const u64 target = (u64)((double)total * (double)row.ask.u);
#pragma unroll
    for (int e = kPerLane - 1; e >= 0; --e) {
        const u64 after = run;
        run -= mask >> e & 1 ? w[e] : 0;
        if (run <= target && target < after) token(p, row, t, i0 + e, x[e], all, kept);
    }
}

// ---------------------------------------------------------------------------
// launches 1 to 3 of longer rows: part blockIdx.x of row blockIdx.y
// ---------------------------------------------------------------------------

// A wave's chunks from j on, every kWavesB-th: f(this lane's logits) for both of its halves, with
// the next loads ahead, then g(chunk).
template <typename T, typename F, typename G>
__device__ __forceinline__ void each_chunk(const T* l, int64_t V, int j, int end, F f, G g) {
    const int at = threadIdx.x % kWave * kPerLane;
    float x[kPerLane], y[kPerLane];
    if (j < end) load8(l, (int64_t)j * kChunk + at, V, x);
    for (; j < end; j += kWavesB) {
        load8(l, (int64_t)j * kChunk + kSub + at, V, y);
        f(x);
        if (j + kWavesB < end) load8(l, (int64_t)(j + kWavesB) * kChunk + at, V, x);
        f(y);
        g(j);
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void ember_sample_range(Params p, int64_t t0) {
    __shared__ Part redp[kWavesB];
    const int c = blockIdx.x, r = blockIdx.y;
    const T* const l = static_cast<const T*>(p.a.L) + (t0 + r) * p.a.ldl;
    const int wave = threadIdx.x / kWave;
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
    Part part{-kInf, kInf, 0, 0};
    const int end = min((c + 1) * p.part_chunks, p.chunks);
    float peak = -kInf;
    each_chunk(
        l, p.a.V, c * p.part_chunks + wave, end,
        [&](const float (&x)[kPerLane]) {
#pragma unroll
            for (int e = 0; e < kPerLane; ++e) {
                see(part, x[e]);
                peak = fmaxf(peak, x[e]);
            }
        },
        [&](int j) {
            if (!p.list) return;
            peak = wave_one(peak, [](float a, float b) { return fmaxf(a, b); });
            if (threadIdx.x % kWave == 0) p.s.peak[(int64_t)r * p.chunks + j] = peak;
            peak = -kInf;
        });
    part = block_join<kThreads>(part, redp);
    if (threadIdx.x == 0) p.s.parts[(int64_t)r * kMaxParts + c] = part;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void ember_sample_weights(Params p, int64_t t0) {
    __shared__ u64 weight[kBins];
    __shared__ int count[kBins];
    __shared__ double table[kSteps];
    __shared__ u64 red[kWavesB];
    __shared__ int redi[kWavesB];
    const int c = blockIdx.x, r = blockIdx.y;
    const T* const l = static_cast<const T*>(p.a.L) + (t0 + r) * p.a.ldl;
    const Row row = row_at(p, t0 + r, r);
    if (!row.fine) return;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x & (kWave - 1);
    const bool hist = ranked(row.ask), floored = row.ask.floor > 0.0f;
    fill_table(table, p.bits);
    if (hist) {
        for (int b = threadIdx.x; b < kBins; b += kThreads) {
            weight[b] = 0;
            count[b] = 0;
        }
    }
    __syncthreads();
    u64 all = 0, sum = 0;
    int near = 0;
    const int end = min((c + 1) * p.weight_chunks, p.chunks);
    each_chunk(
        l, p.a.V, c * p.weight_chunks + wave, end,
        [&](const float (&x)[kPerLane]) {
            u64 w[kPerLane];
            int b[kPerLane];
#pragma unroll
            for (int e = 0; e < kPerLane; ++e) {
                const double gap = gap_of(row, x[e]);
                w[e] = weight_of(row, gap, table);
                b[e] = (int)(gap * row.scale);
                sum += w[e];
            }
            if (hist) {
#pragma unroll
                for (int e = 0; e < kPerLane; ++e) {
                    if (!w[e]) continue;
                    atomicAdd(&weight[b[e]], w[e]);
                    atomicAdd(&count[b[e]], 1);
                }
            }
            if (floored) {
#pragma unroll
                for (int e = 0; e < kPerLane; ++e) near += x[e] != -kInf && near_of(row, x[e]);
            }
        },
        [&](int j) {
            if (hist || floored) return;      // launch 3 does it
            sum = wave_sum(sum);
            if (lane == 0) {
                p.s.chunk[(int64_t)r * p.chunks + j] = sum;
                all += sum;
            }
            sum = 0;
        });
    all = block_sum<kThreads>(all + sum, red);
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

template <typename T>
__global__ __launch_bounds__(kThreads, 8) void ember_sample_list(Params p, int64_t t0) {
    __shared__ double table[kSteps];
    __shared__ u64 red[kWavesB];
    __shared__ int redi[kWavesB];
    __shared__ Bins found;
    __shared__ float dense[kWavesB][kSub + kWave];
    __shared__ uint16_t index[kWavesB][kSub + kWave];
    __shared__ u64 list[kPartList];
    __shared__ int listed;
    __shared__ unsigned joined;
    const int c = blockIdx.x, r = blockIdx.y;
    const T* const l = static_cast<const T*>(p.a.L) + (t0 + r) * p.a.ldl;
    const Row row = row_at(p, t0 + r, r);
    const bool hist = ranked(row.ask);
    if (!row.fine || (!hist && row.ask.floor == 0.0f)) return;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x & (kWave - 1);
    fill_table(table, p.bits);

    if (threadIdx.x == 0) {
        listed = 0;
        found = Bins{0, 0, 0, 0, 0, 0, kBins, kBins, -1};
    }
    if (hist) {
        constexpr int kOwn = kBins / kThreads;     // bins a thread
        u64 w[kOwn];
        int n[kOwn];
#pragma unroll
        for (int q = 0; q < kOwn; ++q) {
            w[q] = p.s.weight[(int64_t)r * kBins + threadIdx.x * kOwn + q];
            n[q] = p.s.count[(int64_t)r * kBins + threadIdx.x * kOwn + q];
        }
        bins_of<kThreads>(row.ask, w, n, red, redi, found);
    }
    __syncthreads();
    const int bin_k = found.bin_k, bin_p = found.bin_p, bin_p1 = found.bin_p1;
    const int sure = min(bin_k, bin_p);      // tokens of bins before it are kept by both
    RowState& s = p.s.rows[r];
    if (c == 0 && threadIdx.x == 0) s.bins = found;
    // A logit below which nothing counts, with margins for the border's rounding and its own:
    // whether a token counts its bin says.
    const auto gap_to = [&](int b) { return row.scale > 0.0 ? b / row.scale : row.none; };
    double gap = fmin(gap_to(sure), row.ask.far * row.ask.cool);
    if (bin_k < kBins) gap = fmax(gap, gap_to(bin_k + 1));
    if (bin_p < kBins) gap = fmax(gap, gap_to(bin_p1 + 1));
    float least = (float)(row.top - fmin(gap, row.none) * (1.0 + 0x1p-40));
    least = fmaxf(least - fabsf(least) * 0x1p-22f - 1e-37f, -3.4028235e38f);
    const int end = min((c + 1) * p.part_chunks, p.chunks);
    // A wave's chunks, every kWavesB-th, 64 at a time; those with a logit that counts are
    // gone through: their tokens that count side by side in LDS, then a token a lane.
    for (int j0 = c * p.part_chunks + wave; j0 < end; j0 += kWavesB * kWave) {
        const int mine = j0 + lane * kWavesB;
        const int64_t at = (int64_t)r * p.chunks + mine;
        const bool some = mine < end && p.s.peak[at] >= least;
        if (mine < end && !some) p.s.chunk[at] = 0;
        u64 todo = __ballot(some);
        auto chunk_of = [&](u64 m) { return j0 + (__ffsll(m) - 1) * kWavesB; };
        u64 sum = 0;
        int n = 0, j = 0;
        // a half's tokens that count join the n there are
        auto put = [&](const float (&x)[kPerLane], int first) {
#pragma unroll
            for (int e = 0; e < kPerLane; ++e) {
                const u64 m = __ballot(x[e] >= least);
                if (x[e] >= least) {
                    const int to = n + __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0));
                    dense[wave][to] = x[e];
                    index[wave][to] = (uint16_t)(first + lane * kPerLane + e);
                }
                n += __popcll(m);
            }
        };
        auto take = [&] {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            for (int q = lane; q < n; q += kWave) {
                const float v = dense[wave][q];
                const double gap = gap_of(row, v);
                const int b = bin_of(row, gap);
                const u64 w = weight_of(row, gap, table);
                if (b < sure) {
                    sum += near_of(row, v) ? w : 0;
                } else if (w && (b == bin_k || (b >= bin_p && b <= bin_p1))) {
                    const int to = atomicAdd(&listed, 1);
                    if (to < kPartList) list[to] = place_of<T>(v, (uint32_t)(j * kChunk + index[wave][q]), p.width);
                }
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            n = 0;
        };
        float x[kPerLane], y[kPerLane];
        const int own = lane * kPerLane;
        if (todo) load8(l, (int64_t)chunk_of(todo) * kChunk + own, p.a.V, x);
        while (todo) {
            j = chunk_of(todo);
            todo &= todo - 1;
            load8(l, (int64_t)j * kChunk + kSub + own, p.a.V, y);
            put(x, 0);
            if (todo) load8(l, (int64_t)chunk_of(todo) * kChunk + own, p.a.V, x);
            if (n > kWave) take();
            put(y, kSub);
            take();
            sum = wave_sum(sum);
            if (lane == 0) p.s.chunk[(int64_t)r * p.chunks + j] = sum;
            sum = 0;
        }
    }
    // the block's list joins the row's
    __syncthreads();
    const int n = listed;
    if (n == 0) return;
    if (threadIdx.x == 0) joined = atomicAdd(&s.listed, n > kPartList ? (unsigned)kList + 1 : (unsigned)n);
    __syncthreads();
    for (int q = threadIdx.x; q < min(n, kPartList); q += kThreads)
        if (joined + q < (unsigned)kList) p.s.list[(int64_t)r * kList + joined + q] = list[q];
}

// ---------------------------------------------------------------------------
// launch 4: row blockIdx.x
// ---------------------------------------------------------------------------

template <typename T>
__global__ __launch_bounds__(kRowThreads) void ember_sample_draw(Params p, int64_t t0) {
    __shared__ Select s;
    __shared__ double table[kSteps];
    __shared__ u64 more[kRowThreads];      // what is kept of a thread's chunks beside their sums
    const int r = blockIdx.x;
    const int64_t t = t0 + r;
    const T* const l = static_cast<const T*>(p.a.L) + t * p.a.ldl;
    const Row row = row_at(p, t, r);
    if (!row.fine) {
        if (threadIdx.x == 0) no_token(p.a, t);
        return;
    }
    // what is needed later, ahead: this thread's chunks, the first of the list
    const bool hist = ranked(row.ask);
    const int own = (p.chunks + kRowThreads - 1) / kRowThreads;      // chunks a thread
    u64 sum = 0;
    for (int j = threadIdx.x * own; j < min((int)(threadIdx.x + 1) * own, p.chunks); ++j)
        sum += p.s.chunk[(int64_t)r * p.chunks + j];
    const u64 first = hist ? p.s.list[(int64_t)r * kList + threadIdx.x] : 0;
    const RowState st = p.s.rows[r];
    fill_table(table, p.bits);
    more[threadIdx.x] = 0;
    __syncthreads();
    const u64 all = st.all;
    u64 last = 0;                     // the last place that is kept, where the bins alone do not say it
    int sure = kBins;                 // tokens of bins before it are kept
    int kept = row.some;              // before min-p
    if (hist) {
        sure = min(st.bins.bin_k, st.bins.bin_p);
        if (row.ask.k > 0) kept = min(kept, row.ask.k);
        const int n = (int)min(st.listed, (unsigned)kList + 1);
        if (n > kList) {
            const auto each = [&](int first, int last, auto f) {
                for (int64_t i = threadIdx.x * kPerLane; i < p.a.V; i += kRowThreads * kPerLane) {
                    float x[kPerLane];
                    load8(l, i, p.a.V, x);
#pragma unroll
                    for (int e = 0; e < kPerLane; ++e) {
                        const double gap = gap_of(row, x[e]);
                        const int b = bin_of(row, gap);
                        if (b < first || b > last) continue;
                        const u64 w = weight_of(row, gap, table);
                        if (w) f(place_of<T>(x[e], (uint32_t)(i + e), p.width), [&] { return w; });
                    }
                }
            };
            last = last_of(row.ask, st.bins, all, each, s, kept);
            each(sure, kBins - 1, [&](u64 at, auto weight) {
                if (at <= last && near_of(row, logit_of<T>(at, p.width)))
                    atomicAdd(&more[(uint32_t)(at & (((u64)1 << p.width) - 1)) / (kChunk * own)], weight());
            });
        } else if (n > 0) {
            constexpr int kOwn = kList / kRowThreads;
            u64 at[kOwn], w[kOwn];
            int bin[kOwn];
            const auto logit = [&](int q) { return logit_of<T>(at[q], p.width); };
#pragma unroll
            for (int q = 0; q < kOwn; ++q) {
                at[q] = kNone;
                w[q] = 0;
                bin[q] = kBins;
                if (q * kRowThreads >= n) continue;
                const int i = q * kRowThreads + threadIdx.x;
                if (i >= n) continue;
                at[q] = q == 0 ? first : p.s.list[(int64_t)r * kList + i];
                const double gap = gap_of(row, logit(q));
                w[q] = weight_of(row, gap, table);
                if (w[q]) bin[q] = bin_of(row, gap);
                else at[q] = kNone;
            }
            const auto each = [&](int first, int last, auto f) {
#pragma unroll
                for (int q = 0; q < kOwn; ++q)
                    if (bin[q] >= first && bin[q] <= last) f(at[q], [&] { return w[q]; });
            };
            last = last_of(row.ask, st.bins, all, each, s, kept);
            // the kept ones join their chunks' sums
#pragma unroll
            for (int q = 0; q < kOwn; ++q) {
                if (at[q] <= last && near_of(row, logit(q)))
                    atomicAdd(&more[(uint32_t)(at[q] & (((u64)1 << p.width) - 1)) / (kChunk * own)], w[q]);
            }
        }
    }
    __syncthreads();
    if (row.ask.floor > 0.0f) kept = min(kept, st.near);

    // the thread in whose chunks u falls
    u64 kept_sum;
    sum = (sure > 0 ? sum : 0) + more[threadIdx.x];
    if (threadIdx.x == 0) s.lo = kNone;
    const u64 end = block_scan<kRowThreads>(sum, s.red, kept_sum);
    const u64 target = (u64)((double)kept_sum * (double)row.ask.u);
    if (end - sum <= target && target < end) {
        s.lo = threadIdx.x;
        s.w = end - sum;
    }
    __syncthreads();
    if (s.lo == kNone) {      // not met: the largest logit is always kept
        if (threadIdx.x == 0) no_token(p.a, t);
        return;
    }
    // and the token in them, one a thread
    int64_t i = (int64_t)s.lo * own * kChunk + threadIdx.x;
    u64 before = s.w;
    for (int q = 0; q < own * kChunk; q += kRowThreads, i += kRowThreads) {
        u64 w = 0;
        float x = 0.0f;
        if (q + (int)threadIdx.x < own * kChunk && i < p.a.V) {
            x = load_elem(l, i, sizeof(T) == 2);
            const double gap = gap_of(row, x);
            const bool keep = bin_of(row, gap) < sure || place_of<T>(x, (uint32_t)i, p.width) <= last;
            if (keep && near_of(row, x)) w = weight_of(row, gap, table);
        }
        u64 piece;
        const u64 to = before + block_scan<kRowThreads>(w, s.red, piece);
        if (to - w <= target && target < to) token(p, row, t, i, x, all, kept);
        before += piece;
        if (target < before) break;
    }
}

template <typename T>
hipError_t launch(const Params& p, int64_t t0, int rows, hipStream_t s) {
    const dim3 grid((unsigned)p.parts, (unsigned)rows);
    ember_sample_range<T><<<grid, kThreads, 0, s>>>(p, t0);
    ember_sample_weights<T><<<dim3((unsigned)((p.chunks + p.weight_chunks - 1) / p.weight_chunks), (unsigned)rows), kThreads, 0, s>>>(p, t0);
    if (p.list) ember_sample_list<T><<<grid, kThreads, 0, s>>>(p, t0);
    ember_sample_draw<T><<<rows, kRowThreads, 0, s>>>(p, t0);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_row(const Params& p, hipStream_t s) {
    for (int64_t t0 = 0; t0 < p.a.T; t0 += kMaxGridBlocks) {
        ember_sample_row<T><<<(unsigned)std::min(kMaxGridBlocks, p.a.T - t0), kRowThreads, 0, s>>>(p, t0);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

} // namespace

// (a block's rows need none of it: 4 KiB for any number of them, so that a call's workspace is never empty)
size_t sample_ws_bytes(int64_t T, int64_t V) {
    return V <= kOneBlock ? kLeastBytes : std::max(kLeastBytes, space_of(nullptr, std::min(T, kMaxRows), V, nullptr));
}

hipError_t launch_sample(const SampleArgs& a, hipStream_t s) {
    Params p;
    p.a = a;
    p.width = 0;
    while (((int64_t)1 << p.width) < a.V) ++p.width;
    p.bits = std::min(48, 62 - p.width);
    if (a.V <= kOneBlock) return a.l_dtype == EMBER_F32 ? launch_row<float>(p, s) : launch_row<uint16_t>(p, s);
    const int64_t rows = std::min(a.T, kMaxRows);
    space_of(a.ws, rows, a.V, &p.s);
    p.chunks = (int)chunks_of(a.V);
    // about 1024 blocks (launch 2: 512, which are there at once), of a chunk a wave at least
    const auto chunks_a_block = [&](int64_t blocks) {
        const int64_t n = std::min<int64_t>({(blocks + rows - 1) / rows, (p.chunks + kWavesB - 1) / kWavesB, kMaxParts});
        return (int)((p.chunks + n - 1) / n);
    };
    p.part_chunks = chunks_a_block(1024);
    p.weight_chunks = chunks_a_block(512);
    p.parts = (p.chunks + p.part_chunks - 1) / p.part_chunks;
    p.list = a.top_k || a.top_p || a.min_p || a.temperature;
    for (int64_t t0 = 0; t0 < a.T; t0 += kMaxRows) {
        const int n = (int)std::min(kMaxRows, a.T - t0);
        const hipError_t e = a.l_dtype == EMBER_F32 ? launch<float>(p, t0, n, s) : launch<uint16_t>(p, t0, n, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

} // namespace ember
