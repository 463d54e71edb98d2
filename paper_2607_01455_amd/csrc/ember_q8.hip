// Logits of an LM head held in 8 bits (gfx950):
//   Y_tv = (sum_k Xq_tk Wq_vk) xscale_t wscale_v + bias_v,
// with int8 matrix instructions.  The sum is exact in int32 (D is limited to
// EMBER_NORM_MAX_D), so neither tiling nor order changes a bit of it; it is
// rounded to fp32 once, scaled, and rounded to the type of Y.
//
// Tiling: a block computes BM tokens x BN channels; its wavefronts hold their
// parts of the tile as 32 x 32 MFMA accumulators.  Both operands have the
// contraction contiguous, so a step's slices (BM and BN rows of KS bytes) go from
// global memory straight into LDS (16-byte buffer loads with an LDS destination)
// and are read from there as MFMA operands, 16 consecutive columns a lane.  A ring
// of LDS stages keeps the loads of the next steps in flight; the operands of
// each 32-column sub-step are read behind the previous sub-step's MFMAs, across
// the step barrier too.  In the small tilings several groups of wavefronts share a
// tile's steps, each with a ring of its own, and their sums are added at the end.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "ember_device.h"
#include "ember_interface_launch.h"
#include "ember_tile.h"

namespace ember {
namespace {

constexpr uint32_t kRotate = 5;            // steps between the first steps of neighbouring tiles

struct Params {
    LogitsArgs a;
    int nk;              // steps of the contraction
    int MT;              // tiles of tokens
    int64_t NT;          // tiles of channels
    int64_t tile0;       // this launch's tiles: [tile0, tile1) of the MT * NT
    int64_t tile1;
    int64_t per_xcd;     // tiles per XCD
    int64_t blocks;      // blocks per XCD: each takes every blocks-th of its tiles
    int group_m;         // token tiles a group of the tile order
    int in_step;         // log2 of the channel tiles that begin at the same step
};

template <int BM_, int BN_, int WM_, int WN_, int KS_, int STAGES_, int KG_ = 1>
struct Tile {
    static constexpr int BM = BM_, BN = BN_;       // tokens, channels a block
    static constexpr int WM = WM_, WN = WN_;       // wavefronts over them
    static constexpr int KS = KS_;                 // columns (bytes) a step
    static constexpr int kStages = STAGES_;
    static constexpr int KG = KG_;                 // groups of wavefronts that share the steps, each with a ring
    static constexpr int kWavesB = WM * WN;        // of a group
    static constexpr int kThreads = KG * kWavesB * kWave;
    static constexpr int MT = BM / WM / 32, NT = BN / WN / 32;   // MFMA tiles a wave
    static constexpr int kSub = KS / 32;
    static constexpr int kChunks = KS / 16;        // 16-byte chunks of a slice's row
    static constexpr int kRowsPerLoad = kWave / kChunks;
    static constexpr int kLoadsA = BM / kRowsPerLoad, kLoadsB = BN / kRowsPerLoad;
    static constexpr int kLoads = (kLoadsA + kLoadsB) / kWavesB;   // a wave and step
    static constexpr int kStageBytes = (BM + BN) * KS;
    static constexpr int kRing = kStages * kStageBytes;
    static constexpr int kLds = KG * kRing;
    static_assert((kLoadsA + kLoadsB) % kWavesB == 0, "equal loads a wave");
    static_assert(kSub >= 2 && kSub % 2 == 0, "a step ends on the register set it began with");
    static_assert(kStages >= 2 && (kStages - 2) * kLoads < 64, "vmcnt range");
    static_assert((int64_t)std::max(BM, BN) * EMBER_Q8_MAX_LD < (int64_t)1 << 31, "32-bit load offsets");
    static_assert(kLds <= 160 * 1024, "LDS of one CU");
};

// The epilogue's use of the LDS: a strip a wave, then the channels' scales and biases.
template <typename C, typename YT>
struct Epilogue {
    static constexpr int kGroup = std::min(C::NT, 256 / (32 * (int)sizeof(YT)));   // MFMA tiles side by side in a strip
    static constexpr int kCols = kGroup * 32;
    static constexpr int kPitch = kCols * (int)sizeof(YT) + 16;   // bytes a token
    static constexpr int kStrips = C::kWavesB * 32 * kPitch;
    static constexpr int kBytes = kStrips + 2 * C::BN * 4;
};

// Where a compute unit holds one block, the block goes through several tiles, and the
// next one's first stage is loaded while an epilogue works behind it (us, a tile a
// block / like this, 256 x 256 tiles: 4096 x 128256 x 4096 2115 / 2001, 955 x 33990 x
// 3381 fp32 165 / 161, 1500 x 50000 x 1024 106 / 103).
template <typename C>
constexpr bool kGoesOn = C::KG == 1 && C::kLds > 80 * 1024;
template <typename C>
constexpr int kEpilogueAt = kGoesOn<C> ? C::kStageBytes : 0;   // in the LDS
template <typename C, typename YT>
constexpr int kLdsBytes = std::max(C::kLds, kEpilogueAt<C> + Epilogue<C, YT>::kBytes);

// kMask: D is not a multiple of 16, so the last chunk of a row holds columns
// that do not count; they are cleared in the tokens' operand.
template <typename C, typename YT, bool kMask>
__global__ __launch_bounds__(C::kThreads) void ember_logits_q8(Params p) {
    __shared__ __attribute__((aligned(1024))) uint8_t lds[kLdsBytes<C, YT>];
    const LogitsArgs& a = p.a;
    const int lane = threadIdx.x & (kWave - 1);
    const int wave_all = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int group = wave_all / C::kWavesB, wave = wave_all % C::kWavesB;
    const int wm = wave % C::WM, wn = wave / C::WM;
    const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds + group * C::kRing;

    // blocks of one XCD take consecutive tiles
    const int64_t first = p.tile0 + (int64_t)(blockIdx.x % kXcds) * p.per_xcd;
    const int64_t end = min(first + p.per_xcd, p.tile1);
    int64_t l = first + blockIdx.x / kXcds;
    if (l >= end) return;
    const int nk = p.nk, D = (int)a.D;
    const int steps = (nk + C::KG - 1) / C::KG;   // of each group; past the last they are zeros
    struct At {
        int64_t t0, v0;
        int rot;
    };
    // Blocks with other channels begin at other steps (the sum has no order): in
    // step, all of them would read the same columns of rows that lie a power of
    // two apart, and so a few of the memory's channels at a time (64 tokens x
    // 128256 x 4096: 127 us in step, 105 like this; one token: 110 and 91).  With
    // several token tiles, eight channel tiles are in step: an XCD's blocks then
    // read the tokens' slices together, not each from beyond its L2, which costs
    // power and so clock (4096 x 128256 x 4096: 1997 us with one in step, groups of
    // eight token tiles; 1885 with eight in step; 1867 with groups of four too).
    auto tile_at = [&](int64_t i) {
        int tm;
        int64_t tn;
        ember::tile_at(p.MT, p.NT, p.group_m, i, tm, tn);
        return At{(int64_t)tm * C::BM, tn * C::BN, (int)((uint64_t)(tn >> p.in_step) * kRotate % (uint32_t)nk)};
    };
    At at = tile_at(l);

    // load j of this wave fills rows [kRowsPerLoad q, ..) of the tokens' slice, q =
    // wave + kWavesB j, then of the channels'; a lane's chunk is the same in all of them
    static_assert(C::kWavesB % 2 == 0 && C::kLoadsA % C::kWavesB == 0, "one load_k for all loads, each of one operand");
    const int load_row = wave * C::kRowsPerLoad + lane / C::kChunks;
    const int load_k = ((lane % C::kChunks) ^ swizzle<C::kChunks>(load_row)) * 16;
    const uint32_t load_a = load_row * (uint32_t)a.ldx + load_k, load_b = load_row * (uint32_t)a.ldw + load_k;
    struct StepLoads {
        i32x4 ra, rb;
        uint32_t oa, ob;
    };
    // step i of this wave's group
    auto loads_of = [&](int i) {
        const int kt = i * C::KG + group;
        const bool in = kt < nk;
        const int ks = kt + at.rot < nk ? kt + at.rot : kt + at.rot - nk;
        const int64_t k0 = in ? (int64_t)ks * C::KS : 0;
        StepLoads sl;
        sl.ra = rsrc(a.Xq + at.t0 * a.ldx + k0, in ? (a.T - at.t0) * a.ldx - k0 : 0);
        sl.rb = rsrc(a.Wq + at.v0 * a.ldw + k0, in ? (a.V - at.v0) * a.ldw - k0 : 0);
        // Chunks past column D are zeros (no row's offset brings kBufferMax back).
        // The offsets of a step's loads are formed anew in each, hidden from the
        // compiler, which would keep all of them in registers.
        const bool whole = load_k < D - (int)k0;
        sl.oa = whole ? load_a : kBufferMax;
        sl.ob = whole ? load_b : kBufferMax;
        asm volatile("" : "+v"(sl.oa), "+v"(sl.ob));
        return sl;
    };
    auto issue_one = [&](const StepLoads& sl, uint32_t st, int j) {
        constexpr int kA = C::kLoadsA / C::kWavesB, kRows = C::kWavesB * C::kRowsPerLoad;
        const uint32_t o = j < kA ? sl.oa + j * (kRows * (uint32_t)a.ldx) : sl.ob + (j - kA) * (kRows * (uint32_t)a.ldw);
        load_to_lds(j < kA ? sl.ra : sl.rb, st + (wave + C::kWavesB * j) * (C::kRowsPerLoad * C::KS), o);
    };

    // operand reads: lane l takes row l % 32 of an MFMA tile, columns
    // 16 (l / 32) .. + 15 of the sub-step
    auto frag = [&](uint32_t st, int row, int kk) {
        const int c = 2 * kk + (lane >> 5);
        const uint32_t at = st + row * C::KS + ((c ^ swizzle<C::kChunks>(row)) * 16);
        return *(const __attribute__((address_space(3))) i32x4*)(uintptr_t)at;
    };
    const int row_a = wm * (C::MT * 32) + (lane & 31), row_b = C::BM + wn * (C::NT * 32) + (lane & 31);
    static_assert(C::BM % 16 == 0, "the channels' rows have the swizzle of their number");
    auto mask_a = [&](int kt, int kk, i32x4& x) {
        const int n = D - kt * C::KS - 32 * kk - 16 * (lane >> 5);   // columns that count of these 16
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const int b = n - 4 * w;
            x[w] &= b >= 4 ? -1 : b <= 0 ? 0 : (int)((1u << (8 * b)) - 1);
        }
    };

    auto issue = [&](int q) {
        const StepLoads sl = loads_of(q);
#pragma unroll
        for (int j = 0; j < C::kLoads; ++j) issue_one(sl, lds_base + q * C::kStageBytes, j);
    };
    issue(0);
    for (bool fresh = true;; fresh = false) {
        i32x16 acc[C::MT][C::NT];
#pragma unroll
        for (int mt = 0; mt < C::MT; ++mt)
#pragma unroll
            for (int nt = 0; nt < C::NT; ++nt)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[mt][nt][i] = 0;

        // the scales the epilogue needs, ahead of the operands
        const int64_t t0 = at.t0, v0 = at.v0;
        float xs[C::MT];
#pragma unroll
        for (int m = 0; m < C::MT; ++m) {
            const int64_t t = t0 + (wm * C::MT + m) * 32 + (lane & 31);
            xs[m] = t < a.T ? a.xscale[t] : 0.0f;
        }
        const int64_t my_v = v0 + threadIdx.x;
        const bool has_v = (int)threadIdx.x < C::BN && my_v < a.V;
        const float my_wscale = has_v ? a.wscale[my_v] : 0.0f, my_bias = has_v && a.bias ? a.bias[my_v] : 0.0f;

#pragma unroll
        for (int q = 1; q < C::kStages; ++q) issue(q);
        l += p.blocks;
        const bool more = kGoesOn<C> && l < end;
        At then = at;
        if (more) then = tile_at(l);
        if (fresh) wait_step<(C::kStages - 1) * C::kLoads>();
        i32x4 af[2][C::MT], bf[2][C::NT];
#pragma unroll
        for (int m = 0; m < C::MT; ++m) af[0][m] = frag(lds_base, row_a + 32 * m, 0);
#pragma unroll
        for (int n = 0; n < C::NT; ++n) bf[0][n] = frag(lds_base, row_b + 32 * n, 0);

        // Step kt multiplies its stage in kSub sub-steps; while the MFMAs of one run,
        // the operands of the next are read into the other register set.  The step
        // barrier sits before the last sub-step, whose operands are in registers by
        // then: past it no wave reads this stage any more, so the loads of step
        // kt + kStages may fill it; and at most (kStages - 2) kLoads loads of each
        // wave are outstanding, which are those of steps kt + 2 and later, so step
        // kt + 1 lies in its stage.
        uint32_t st = lds_base;
        for (int i = 0; i < steps; ++i) {
            const uint32_t next = st + C::kStageBytes == lds_base + C::kRing ? lds_base : st + C::kStageBytes;
            const StepLoads sl = loads_of(i + C::kStages);
#pragma unroll
            for (int kk = 0; kk < C::kSub; ++kk) {
                const int cur = kk & 1;
                const bool last = kk == C::kSub - 1;
                if constexpr (kMask) {
                    const int kt = i * C::KG + group, ks = kt + at.rot < nk ? kt + at.rot : kt + at.rot - nk;
                    if (ks == nk - 1) {
#pragma unroll
                        for (int m = 0; m < C::MT; ++m) mask_a(ks, kk, af[cur][m]);
                    }
                }
                if (last) wait_step<(C::kStages - 2) * C::kLoads>();
                __builtin_amdgcn_sched_barrier(0);
                constexpr int kSlots = C::MT * C::NT > C::MT + C::NT ? C::MT * C::NT : C::MT + C::NT;
                constexpr int kAll = kSlots > C::kLoads ? kSlots : C::kLoads;
#pragma unroll
                for (int x = 0; x < kAll; ++x) {
                    if (x < C::MT * C::NT) {
                        const int m = x / C::NT, n = x % C::NT;
                        acc[m][n] = __builtin_amdgcn_mfma_i32_32x32x32_i8(bf[cur][n], af[cur][m], acc[m][n], 0, 0, 0);
                    }
                    // operands in the order the MFMAs first use them: A 0, all of B, the rest of A
                    if (x < C::MT + C::NT) {
                        const bool is_b = x >= 1 && x <= C::NT;
                        const int f = x == 0 ? 0 : is_b ? x - 1 : x - C::NT;
                        const i32x4 w = frag(last ? next : st, (is_b ? row_b : row_a) + 32 * f, last ? 0 : kk + 1);
                        if (is_b) bf[cur ^ 1][f] = w;
                        else af[cur ^ 1][f] = w;
                    }
                    if (last && x < C::kLoads) issue_one(sl, st, x);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            st = next;
        }
        // the zero-filling loads past the end have landed and every wave is done with the stages
        wait_step<0>();
        if (more) {
            at = then;
            issue(0);
        }

        if constexpr (C::KG > 1) {
            // the other groups' sums join the first one's
            constexpr int kSums = C::kWavesB * C::MT * C::NT * 16 * kWave;
            static_assert((C::KG - 1) * kSums * 4 <= C::kLds, "the sums of the groups");
            int* const sums = reinterpret_cast<int*>(lds) + (wave * C::MT * C::NT * 16) * kWave + lane;
#pragma unroll
            for (int m = 0; m < C::MT; ++m)
#pragma unroll
                for (int n = 0; n < C::NT; ++n)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (group > 0) sums[(group - 1) * kSums + ((m * C::NT + n) * 16 + i) * kWave] = acc[m][n][i];
            wait_step<63>();
            if (group == 0) {
#pragma unroll
                for (int q = 0; q < C::KG - 1; ++q)
#pragma unroll
                    for (int m = 0; m < C::MT; ++m)
#pragma unroll
                        for (int n = 0; n < C::NT; ++n)
#pragma unroll
                            for (int i = 0; i < 16; ++i)
                                acc[m][n][i] += sums[q * kSums + ((m * C::NT + n) * 16 + i) * kWave];
            }
            wait_step<63>();
        }

        // Epilogue: the channels are the rows of the MFMA tiles, so a lane holds four
        // consecutive ones of a token.  Each wave takes its part in strips of 32 tokens
        // x up to 256 bytes of channels: the values go to a wave-private LDS strip
        // and are stored from it row by row, 16 bytes a lane.
        using E = Epilogue<C, YT>;
        constexpr int kEs = (int)sizeof(YT), kGroup = E::kGroup, kCols = E::kCols, kPitch = E::kPitch;
        constexpr int kLanesPerRow = kCols * kEs / 16;
        constexpr int kRowsPerPass = kWave / kLanesPerRow;
        constexpr int kEpc = 16 / kEs;
        static_assert(C::NT % kGroup == 0 && 32 % kRowsPerPass == 0 && C::kThreads >= C::BN, "whole strips");
        uint8_t* const strip = lds + kEpilogueAt<C> + wave * (32 * kPitch);
        float* const sw = reinterpret_cast<float*>(lds + kEpilogueAt<C> + E::kStrips);
        float* const sb = sw + C::BN;
        if ((int)threadIdx.x < C::BN) {
            sw[threadIdx.x] = my_wscale;
            sb[threadIdx.x] = my_bias;
        }
        wait_step<63>();
        if (C::KG > 1 && group > 0) break;
        int el = lane;
        asm volatile("" : "+v"(el));   // what follows from it is not kept in registers over the loop above
        const int half = el >> 5, tok = el & 31;
        typedef float f32x4 __attribute__((ext_vector_type(4)));
#pragma unroll
        for (int m = 0; m < C::MT; ++m) {
            const int64_t ts = t0 + (wm * C::MT + m) * 32;
#pragma unroll
            for (int g = 0; g < C::NT / kGroup; ++g) {
                const int c0 = wn * (C::NT * 32) + g * kCols;   // the strip's first channel in the tile
#pragma unroll
                for (int n = 0; n < kGroup; ++n) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int at = n * 32 + 8 * q + 4 * half;   // registers 4 q .. 4 q + 3
                        const f32x4 w = *reinterpret_cast<const f32x4*>(sw + c0 + at);
                        const f32x4 b = *reinterpret_cast<const f32x4*>(sb + c0 + at);
                        float y[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            y[e] = (float)acc[m][g * kGroup + n][4 * q + e] * (xs[m] * w[e]) + b[e];
                        store_values<YT, 4>(reinterpret_cast<YT*>(strip + tok * kPitch) + at, 0, 4, y);
                    }
                }
                wave_lds_order();
                // this wave's share of the next tile's first stage has landed before its
                // stores are on their way, so that no one waits for these
                if (kGoesOn<C> && m == 0 && g == 0) __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
#pragma unroll
                for (int ps = 0; ps < 32 / kRowsPerPass; ++ps) {
                    const int r = ps * kRowsPerPass + el / kLanesPerRow;
                    const int c = el % kLanesPerRow;
                    const int64_t t = ts + r, v = v0 + c0 + c * kEpc;
                    const u32x4_t w = *reinterpret_cast<const u32x4_t*>(strip + r * kPitch + c * 16);
                    if (t < a.T) {
                        YT* y = static_cast<YT*>(a.Y) + t * a.ldy + v;
                        if (v + kEpc <= a.V) {
                            *reinterpret_cast<u32x4_t*>(y) = w;
                        } else {
#pragma unroll
                            for (int e = 0; e < kEpc; ++e) {
                                if (v + e < a.V) {
                                    if constexpr (kEs == 2)
                                        reinterpret_cast<uint16_t*>(y)[e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
                                    else
                                        reinterpret_cast<uint32_t*>(y)[e] = w[e];
                                }
                            }
                        }
                    }
                }
                wave_lds_order();   // the strip is rewritten next
            }
        }
        if (!more) break;
        // every wave is done with its strip and has its share of the stage
        wait_step<63>();
    }
}

// ---------------------------------------------------------------------------
// few tokens
// ---------------------------------------------------------------------------

constexpr int kFewWaves = 8;                 // wavefronts that share the contraction, and one that adds up
constexpr int kFewThreads = (kFewWaves + 1) * kWave;
constexpr int kStrip = 16;                   // channels of a strip
constexpr int kFewBlocks = 256;              // one a compute unit

struct FewParams {
    LogitsArgs a;
    int64_t rounds;      // rounds of SB strips over the table
    int per_xcd;         // rounds of one pass of the grid, per XCD
};

// Up to 16 NB tokens: bound by the table's bytes.  Eight waves share the columns
// (KF blocks of 64 each) and hold their part of all the tokens as MFMA operands in
// registers, loaded once; then they stream the table, SB strips of 16 channels a
// round, straight from memory into the other operand, two rounds in flight.
// They leave their sums of a round in LDS, where a ninth wave adds them up,
// scales and stores them while the others go on (the streaming waves have no
// memory operations but their loads, which return in order).  Columns past D are
// zeros in the tokens' operand, so what the table's operand holds there (some
// column before D) does not matter.
template <int KF, int KP, int SB, int NB, typename YT>
__global__ __launch_bounds__(kFewThreads) void ember_logits_few(FewParams p) {
    const LogitsArgs& a = p.a;
    constexpr int N = kChunkElems<YT>;
    constexpr int kPitch = SB * kStrip + N;
    __shared__ __attribute__((aligned(16))) int part[2][SB][NB][kFewWaves][4 * kWave];
    __shared__ __attribute__((aligned(16))) YT ybuf[16 * NB][kPitch];
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int D = (int)a.D;
    const int row = lane & 15, quarter = lane >> 4;

    // rounds of one pass of the grid: consecutive ones within an XCD
    const int64_t pass = (int64_t)p.per_xcd * kXcds;
    const int64_t first = (int64_t)(blockIdx.x % kXcds) * p.per_xcd + blockIdx.x / kXcds;
    if (first >= p.rounds) return;   // the whole block: no meeting is missed
    // this block's rounds, made even: one past the table reads and stores nothing
    const int rounds = (int)((p.rounds - first + pass - 1) / pass + 1) & ~1;
    auto channel = [&](int i) { return (first + i * pass) * SB * kStrip; };   // first one of the block's round i

    // The block's waves meet once a round, the streaming ones with their loads in
    // flight.  Half `buf` of part is written before the round's meeting, read
    // before the next one and written again after that.
    auto meet = [&] {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    auto buffer = [&](const void* base, int64_t bytes) {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0,
                                                 (int)(bytes < kBufferMax ? bytes : kBufferMax), kBufferWord3);
    };

    if (wave == kFewWaves) {
        float xs[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) xs[b] = 16 * b + row < a.T ? a.xscale[16 * b + row] : 0.0f;
        struct Scales {
            float ws[SB][4], bias[SB][4];
        };
        // lane: token lane % 16, channels 4 (lane / 16) .. + 3 of a strip; zeros past the table
        auto load = [&](int i, Scales& x) {
            const int64_t v = channel(i);
            const int64_t left = v < a.V ? a.V - v : 0;
            const auto rw = buffer(a.wscale + (v < a.V ? v : 0), left * 4);
            const auto rb = buffer(a.bias ? a.bias + (v < a.V ? v : 0) : a.wscale, a.bias ? left * 4 : 0);
#pragma unroll
            for (int s = 0; s < SB; ++s) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int at = (s * kStrip + 4 * quarter + e) * 4;
                    x.ws[s][e] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rw, at, 0, 0));
                    x.bias[s][e] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rb, at, 0, 0));
                }
            }
        };
        auto sum = [&](int i, int buf, const Scales& x, Scales& next) {
            meet();
            load(i + 1, next);   // a round ahead
#pragma unroll
            for (int s = 0; s < SB; ++s) {
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    i32x4 acc = {0, 0, 0, 0};
#pragma unroll
                    for (int q = 0; q < kFewWaves; ++q)
                        acc += *reinterpret_cast<const i32x4*>(&part[buf][s][b][q][4 * lane]);
                    float y[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[e] = (float)acc[e] * (xs[b] * x.ws[s][e]) + x.bias[s][e];
                    store_values<YT, 4>(&ybuf[16 * b + row][s * kStrip + 4 * quarter], 0, 4, y);
                }
            }
            // 16 bytes a lane, row by row
            wave_lds_order();
            constexpr int kPerRow = SB * kStrip / N;
            const int64_t v0 = channel(i);
#pragma unroll
            for (int q = lane; q < 16 * NB * kPerRow; q += kWave) {
                const int t = q / kPerRow, c = q % kPerRow * N;
                if (t >= a.T || v0 + c >= a.V) continue;
                const u32x4_t w = *reinterpret_cast<const u32x4_t*>(&ybuf[t][c]);
                YT* y = static_cast<YT*>(a.Y) + t * a.ldy + v0 + c;
                if (v0 + c + N <= a.V) {
                    *reinterpret_cast<u32x4_t*>(y) = w;
                } else {
                    for (int e = 0; e < N; ++e)
                        if (v0 + c + e < a.V) y[e] = ybuf[t][c + e];
                }
            }
            wave_lds_order();
        };
        Scales s0, s1;
        load(0, s0);
        for (int i = 0; i < rounds; i += 2) {
            sum(i, 0, s0, s1);
            sum(i + 1, 1, s1, s0);
        }
        return;
    }

    // The loads of part h (of KP) of a round's columns: zeros for columns past D and
    // rows past the table (a round past the last one reads nothing), so that
    // every round has the same loads.
    const int col0 = wave * (KF * 64) + 16 * quarter;
    const uint32_t row_off = row * (uint32_t)a.ldw + col0;
    const int64_t row_end = (a.D + 15) / 16 * 16;   // of the last row that is read
    auto load = [&](int i, int h, i32x4 (&w)[SB][KF]) {
        const int64_t v0 = channel(i);
#pragma unroll
        for (int s = 0; s < SB; ++s) {
            const int64_t v = v0 + s * kStrip;
            const auto rs = buffer(a.Wq + (v < a.V ? v * a.ldw : 0), v < a.V ? (a.V - 1 - v) * a.ldw + row_end : 0);
#pragma unroll
            for (int f = 0; f < KF; ++f) {
                // all of the column in the offset that the buffer's range is checked against
                const int at = (h * kFewWaves * KF + f) * 64;
                const uint32_t off = (col0 + at < D ? row_off : kBufferMax) + at;
                w[s][f] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, off, 0, 0));
            }
        }
    };
    i32x4 x[KP][NB][KF];
    const int64_t xt = a.T - 1;
#pragma unroll
    for (int h = 0; h < KP; ++h) {
#pragma unroll
        for (int f = 0; f < KF; ++f) {
            const int k = col0 + (h * kFewWaves * KF + f) * 64;
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                // lanes without a column or a token read others and are cleared below
                const int64_t t = min((int64_t)(16 * b + row), xt);
                x[h][b][f] = *reinterpret_cast<const i32x4*>(a.Xq + t * a.ldx + (k < D ? k : 0));
            }
        }
    }
    i32x4 w0[SB][KF], w1[SB][KF];
    load(0, 0, w0);
    if constexpr (KP == 2) load(0, 1, w1);
    else load(1, 0, w1);
#pragma unroll
    for (int h = 0; h < KP; ++h) {
#pragma unroll
        for (int f = 0; f < KF; ++f) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int n = D - col0 - (h * kFewWaves * KF + f) * 64 - 4 * q;   // columns that count of these four
                const int m = n >= 4 ? -1 : n <= 0 ? 0 : (int)((1u << (8 * n)) - 1);
#pragma unroll
                for (int b = 0; b < NB; ++b) x[h][b][f][q] &= 16 * b + row < a.T ? m : 0;
            }
        }
    }
    i32x4 acc[SB][NB];
    auto multiply = [&](int h, const i32x4 (&w)[SB][KF]) {
#pragma unroll
        for (int s = 0; s < SB; ++s) {
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                if (h == 0) acc[s][b] = i32x4{0, 0, 0, 0};
#pragma unroll
                for (int f = 0; f < KF; ++f)
                    acc[s][b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[s][f], x[h][b][f], acc[s][b], 0, 0, 0);
            }
        }
    };
    auto leave = [&](int buf) {
#pragma unroll
        for (int s = 0; s < SB; ++s)
#pragma unroll
            for (int b = 0; b < NB; ++b) *reinterpret_cast<i32x4*>(&part[buf][s][b][wave][4 * lane]) = acc[s][b];
    };
    // the next loads go out before the MFMAs behind them wait for theirs
    auto refill = [&](int i, int h, i32x4 (&w)[SB][KF]) {
        __builtin_amdgcn_sched_barrier(0);
        load(i, h, w);
        __builtin_amdgcn_sched_barrier(0);
    };
    for (int i = 0; i < rounds; i += 2) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if constexpr (KP == 2) {
                multiply(0, w0);
                refill(i + u + 1, 0, w0);
                multiply(1, w1);
                leave(u);
                refill(i + u + 1, 1, w1);
            } else {
                multiply(0, u == 0 ? w0 : w1);
                leave(u);
                refill(i + u + 2, 0, u == 0 ? w0 : w1);
            }
            meet();
        }
    }
}

template <int KF, int KP, int SB, int NB>
hipError_t launch_few(const LogitsArgs& a, hipStream_t s) {
    FewParams p;
    p.a = a;
    p.rounds = (a.V + SB * kStrip - 1) / (SB * kStrip);
    p.per_xcd = (int)std::min<int64_t>((p.rounds + kXcds - 1) / kXcds, kFewBlocks / kXcds);
    const dim3 grid((unsigned)(p.per_xcd * kXcds));
    if (a.y_dtype == EMBER_F32) ember_logits_few<KF, KP, SB, NB, float><<<grid, kFewThreads, 0, s>>>(p);
    else ember_logits_few<KF, KP, SB, NB, uint16_t><<<grid, kFewThreads, 0, s>>>(p);
    return hipGetLastError();
}

template <typename C>
hipError_t launch_tiles(const LogitsArgs& a, hipStream_t s) {
    Params p;
    p.a = a;
    p.nk = (int)((a.D + C::KS - 1) / C::KS);
    p.MT = (int)((a.T + C::BM - 1) / C::BM);
    p.NT = (a.V + C::BN - 1) / C::BN;
    p.group_m = 4;
    p.in_step = p.MT > 1 ? 3 : 0;
    const int64_t total = (int64_t)p.MT * p.NT;
    const bool mask = a.D % 16 != 0;
    for (int64_t t0 = 0; t0 < total; t0 += kMaxGridBlocks) {
        p.tile0 = t0;
        p.tile1 = std::min(t0 + kMaxGridBlocks, total);
        p.per_xcd = (p.tile1 - t0 + kXcds - 1) / kXcds;
        p.blocks = kGoesOn<C> ? std::min<int64_t>(p.per_xcd, kCus / kXcds) : p.per_xcd;
        const dim3 grid((unsigned)(p.blocks * kXcds));
        if (a.y_dtype == EMBER_F32) {
            if (mask) ember_logits_q8<C, float, true><<<grid, C::kThreads, 0, s>>>(p);
            else ember_logits_q8<C, float, false><<<grid, C::kThreads, 0, s>>>(p);
        } else {
            if (mask) ember_logits_q8<C, uint16_t, true><<<grid, C::kThreads, 0, s>>>(p);
            else ember_logits_q8<C, uint16_t, false><<<grid, C::kThreads, 0, s>>>(p);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

using T64x128 = Tile<64, 128, 2, 2, 128, 3>;
using T32x64 = Tile<32, 64, 1, 2, 128, 3, 4>;    // four and three groups of wavefronts share the steps
using T64x64 = Tile<64, 64, 2, 2, 128, 3, 3>;
using T128x128 = Tile<128, 128, 4, 2, 128, 2>;
using T128x128s = Tile<128, 128, 2, 2, 64, 3>;   // 48 KB of shared memory: three a compute unit
using T128x256 = Tile<128, 256, 4, 2, 128, 3>;
using T256x256 = Tile<256, 256, 4, 2, 128, 2>;

// What a launch of a tiling takes, in us, fitted to 50 shapes of 10 to 4096 tokens,
// 1000 to 128256 channels and 128 to 8192 columns (rms error 10 to 20%): one
// fill of the pipeline, then the tiles of a compute unit one after the other, each
// its columns at the rate of a full chip (us per 4096) and its epilogue, which
// is twice as long for fp32 logits.  Where one tile has a compute unit to itself
// the last ones are a whole round; where several share it they are about half of one.
struct TileCost {
    int bm, bn;
    bool alone;
    double fill, columns, epilogue;
};
constexpr TileCost kTiles[] = {
    {64, 128, false, 3.6, 12.0, 1.5},  {32, 64, true, 2.0, 5.0, 2.6},     {64, 64, true, 3.5, 9.0, 1.9},
    {128, 128, false, 3.6, 20.4, 1.6}, {128, 128, false, 5.1, 21.5, 1.1}, {128, 256, true, 2.5, 33.0, 4.0},
    {256, 256, true, 2.5, 52.0, 6.2},
};
constexpr double kTableBytesPerUs = 5.8e6;   // no tiling reads the table faster
double tile_us(const TileCost& c, const LogitsArgs& a) {
    const double tiles = (double)((a.T + c.bm - 1) / c.bm) * (double)((a.V + c.bn - 1) / c.bn) / 256.0;
    const double rounds = c.alone ? std::ceil(tiles) : std::max(1.0, tiles + 0.5);
    const double tile = c.columns * (double)a.D / 4096.0 + c.epilogue * (a.y_dtype == EMBER_F32 ? 2 : 1);
    return std::max(c.fill + rounds * tile, (double)a.V * (double)a.D / kTableBytesPerUs);
}

} // namespace

// Few tokens take the streaming form while their operands fit its registers (us,
// streaming / best tiling: 1 token x 128256 x 4096 82 / 91, 16 tokens 90 / 94, 32
// tokens 96 / 98, 20 x 50000 x 3000 32 / 37, 64 x 100000 x 1000 29 / 39, 64 x 30000 x
// 2000 18 / 21; past those limits 10 x 32768 x 8192 62 / 47, 50 x 200000 x 500 50 /
// 42).  Others the tiling that should take least (us): 333 x 8191 x 1000 12 with
// 128 x 128 tiles and 21 with 256 x 256, 330 x 110820 x 128 26 with 128 x 128 three a
// compute unit, 28 with two and 33 with 256 x 256, 128 x 128256 x 4096 112 with 128 x 256
// and 133 with 256 x 256, 211 x 36770 x 2896 49 with 256 x 256 and 76 with 128 x 128,
// 40 x 128256 x 4096 98 with 64 x 128 and 126 with 256 x 256.  Where few tiles are
// there and D is long, one tile's chain of steps is what counts, and groups of
// wavefronts that share it help (64 x 1500 x 4096 9 with 32 x 64 tiles and four groups,
// 15 with 32 x 128 and none; 500 x 2000 x 4096 12 with 64 x 64 and three, 16; more
// stages instead of groups 16 and 16).
hipError_t launch_logits(const LogitsArgs& a, hipStream_t s) {
    if (a.T <= 16) {
        if (a.D <= 512) return launch_few<1, 1, 4, 1>(a, s);
        if (a.D <= 1024) return launch_few<2, 1, 2, 1>(a, s);
        if (a.D <= 2048) return launch_few<4, 1, 1, 1>(a, s);
        if (a.D <= 4096) return launch_few<4, 2, 1, 1>(a, s);
    } else if (a.T <= 32) {
        if (a.D <= 512) return launch_few<1, 1, 2, 2>(a, s);
        if (a.D <= 1024) return launch_few<2, 1, 2, 2>(a, s);
        if (a.D <= 2048) return launch_few<4, 1, 1, 2>(a, s);
        if (a.D <= 4096) return launch_few<4, 2, 1, 2>(a, s);
    } else if (a.T <= 64 && a.D > 512) {
        if (a.D <= 1024) return launch_few<2, 1, 1, 4>(a, s);
        if (a.D <= 2048) return launch_few<2, 2, 1, 4>(a, s);
    }
    int best = 0;
    for (int i = 1; i < (int)(sizeof kTiles / sizeof kTiles[0]); ++i)
        if (tile_us(kTiles[i], a) < tile_us(kTiles[best], a)) best = i;
    switch (best) {
    case 0: return launch_tiles<T64x128>(a, s);
    case 1: return launch_tiles<T32x64>(a, s);
    case 2: return launch_tiles<T64x64>(a, s);
    case 3: return launch_tiles<T128x128>(a, s);
    case 4: return launch_tiles<T128x128s>(a, s);
    case 5: return launch_tiles<T128x256>(a, s);
    default: return launch_tiles<T256x256>(a, s);
    }
}

} // namespace ember
