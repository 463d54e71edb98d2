// Token tables in 4 bits (gfx950): rows rounded to them, rows read back, and the
// logits of an LM head held so,
//   Y_tv = xscale_t sum_g wscale_vg (sum_{k in g} Xq_tk c_vk) + bias_v,
// the sum over a group with int8 matrix instructions.
//
// Packing.  128 columns are a block of 64 bytes.  Byte 16 q + 4 w + b of it holds
// the code of column 32 w + 4 q + b in its lower half and that of the column 16
// further in its upper half, in two's complement.  A byte's halves become 8-bit
// operands by one mask (upper) or a shift and a mask (lower), both times 16, and
// every dword holds columns of one group of 32, so that whole operands belong to
// one group whatever its size:
//   - 16 bytes a lane (q: the lane's quarter) are, dword by dword, the operands of
//     16 x 16 tiles of 32 columns;
//   - one dword of each q, one half, is 16 consecutive columns: 32 x 32 tiles.
// The sum of a group is at most 16 * 8 * 128 * 128 < 2^24: exact in int32 and in
// the fp32 it is turned into before it is scaled and added to the other groups'.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "ember_device.h"
#include "ember_interface_launch.h"
#include "ember_tile.h"

namespace ember {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kBlockCols = 128;      // columns of a block of codes
constexpr int kBlockBytes = 64;
constexpr float kTiny = 1e-36f;      // a group below it is zeros

__device__ __forceinline__ uint32_t low_codes(uint32_t w) { return (w << 4) & 0xF0F0F0F0u; }   // times 16
__device__ __forceinline__ uint32_t high_codes(uint32_t w) { return w & 0xF0F0F0F0u; }

// n / d for n < 2^16 and the magic number of d < 2^16 (0: of one).
__device__ __forceinline__ uint32_t div_small(uint32_t n, uint32_t magic) { return magic ? __umulhi(n, magic) : n; }
uint32_t magic_of(uint32_t d) { return d == 1 ? 0 : (uint32_t)((((uint64_t)1 << 32) + d - 1) / d); }

// ---------------------------------------------------------------------------
// rows to 4 bits and back
// ---------------------------------------------------------------------------

constexpr int kRowThreads = 256;
constexpr int64_t kPastBytes = (int64_t)96 << 20;         // of rows: from here on they are stored past the caches
constexpr int kUnitLanes = 16;                            // lanes a block of codes, one dword each
constexpr int kUnitsPerPass = kRowThreads / kUnitLanes;   // blocks of codes side by side
constexpr int kAhead = 4;                                 // of a thread, whose loads go out together
constexpr float kSmall = 1e-28f;                          // below it a quotient's remainder may not be exact

// A lane (w, q) of a block has dword 16 q + 4 w of its codes.  In memory order the pair of lanes with q
// = 2 i and 2 i + 1 has 16 columns: the even lane takes the 8 from 32 w + 8 i on (the lower halves of both
// dwords), the odd one the 8 from 32 w + 16 + 8 i on (the upper halves), 16 bytes of bf16 each.
__device__ __forceinline__ int first_col(int s, int lane) {
    return s * kBlockCols + 32 * (lane >> 2) + 4 * (lane & 2) + 16 * (lane & 1);
}

// The value of another lane of the row of 16.
template <int kCtrl>
__device__ __forceinline__ uint32_t of_lane(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kCtrl, 0xF, 0xF, true);
}
constexpr int kPair = 0xB1, kQuad = 0x4E, kHalfRow = 0x141, kRow = 0x140;    // lane ^ 1, ^ 2; mirrored in 8, in 16

struct QuantParams {
    Quant4Args a;
    int nblk;            // blocks of codes a row
    int groups;          // groups a row
    uint32_t magic;      // of nblk
    int rows_per_block;
};

// A group is 4, 8 or 16 lanes.  The quotient x / s is rounded correctly, and so is the code at a
// tie: with r = 1 / s correctly rounded, q = x r and the remainder e = x - q s (exact), q + e r is
// (Markstein).  Bound by HBM: 128256 x 4096 bf16 (1.3 GB read and written) 219 to 245 us, 5.4 to
// 6.0 TB/s; with divisions 390.
template <typename T, int G>
__global__ __launch_bounds__(kRowThreads) void ember_quantize_q4(QuantParams p) {
    const Quant4Args& a = p.a;
    constexpr int kChunks = 8 / kChunkElems<T>;
    const int lane = threadIdx.x % kUnitLanes, w = lane / 4, q = lane % 4;
    const int64_t row0 = (int64_t)blockIdx.x * p.rows_per_block;
    const int rows = (int)min((int64_t)p.rows_per_block, a.rows - row0);
    const int units = rows * p.nblk, D = (int)a.D;
    for (int u0 = threadIdx.x / kUnitLanes; u0 < units; u0 += kAhead * kUnitsPerPass) {
        u32x4_t x[kAhead][kChunks];
        int r[kAhead], s[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int u = min(u0 + i * kUnitsPerPass, units - 1);
            r[i] = (int)div_small(u, p.magic);
            s[i] = u - r[i] * p.nblk;
            const T* row = static_cast<const T*>(a.X) + (row0 + r[i]) * a.ldx;
            const bool follows = row0 + r[i] + 1 < a.rows;
            const int col = first_col(s[i], lane);
#pragma unroll
            for (int c = 0; c < kChunks; ++c) x[i][c] = load_chunk(row, col + c * kChunkElems<T>, D, follows);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (u0 + i * kUnitsPerPass >= units) break;
            const int col = first_col(s[i], lane);
            float v[8];
            uint32_t top = 0;              // of the magnitudes' bits: those of a NaN are above infinity's
#pragma unroll
            for (int c = 0; c < kChunks; ++c) {
                if (col + (c + 1) * kChunkElems<T> > D) x[i][c] &= kept_words<T>(col + c * kChunkElems<T>, D);
#pragma unroll
                for (int e = 0; e < kChunkElems<T>; ++e) {
                    v[c * kChunkElems<T> + e] = elem<T>(x[i][c], e);
                    top = max(top, __float_as_uint(v[c * kChunkElems<T> + e]) & 0x7FFFFFFFu);
                }
            }
            top = max(top, of_lane<kPair>(top));
            top = max(top, of_lane<kQuad>(top));
            if constexpr (G >= 64) top = max(top, of_lane<kHalfRow>(top));
            if constexpr (G == 128) top = max(top, of_lane<kRow>(top));
            const float most = __uint_as_float(top);
            const uint32_t bits = pack_bf16(most * (1.0f / 7.0f), 0.0f) & 0xFFFFu;
            const float scale = bf16_bits_f32(bits), inv = 1.0f / scale;
            const bool fine = top < 0x7F800000u, some = fine && most >= kTiny;
            uint32_t half[2] = {0, 0};     // codes of the first four columns, of the others, in the lower halves of bytes
            // (whole numbers by adding 1.5 * 2^23, whose low bits then are the code's)
            if (__ballot(most < kSmall && most > 0.0f)) {
#pragma unroll 1
                for (int e = 0; e < 8; ++e) half[e / 4] |= (__float_as_uint(v[e] / scale + 12582912.0f) & 15u) << (8 * (e % 4));
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float y = v[e] * inv, more = fmaf(fmaf(-y, scale, v[e]), inv, y);
                    half[e / 4] |= (__float_as_uint(more + 12582912.0f) & 15u) << (8 * (e % 4));
                }
            }
            // the even lane gives its second half for the odd one's first
            const uint32_t other = of_lane<kPair>(q & 1 ? half[0] : half[1]);
            const uint32_t codes = q & 1 ? other | half[1] << 4 : half[0] | other << 4;
            uint8_t* out = a.Q + (row0 + r[i]) * a.ldq + s[i] * kBlockBytes + 16 * q + 4 * w;
            *reinterpret_cast<uint32_t*>(out) = some ? codes : 0u;
            const int g = (s[i] * kBlockCols + 32 * w) / G;
            if (lane % (G / 8) == 0 && g < p.groups)
                a.gscale[(row0 + r[i]) * a.ldg + g] = (uint16_t)(some ? bits : fine ? 0u : 0x7FC0u);
        }
    }
}

struct RowsParams {
    Rows4Args a;
    int64_t first;       // row of the first, without tokens
    int nblk;
    uint32_t magic;
    int rows_per_block;
};

// Rows of the table, or those of given tokens: the exact product of a code (4 bits)
// and its scale (8), rounded once.  A token outside the table has NaN.  Each store of
// a block's 16 lanes is 256 bytes side by side: of bf16 the pairs' eight columns a lane;
// of fp32 four, for which a lane loads two dwords.  Bound by the stores: 16384 tokens of
// 128256 x 4096, bf16 (169 MB), 26 us, 6.5 TB/s.
// kPast: stored past the caches, which is the faster form at every size where nothing reads the rows next, but a
// reader that does finds them in the memory-side cache otherwise.  The limit is where the rows and the norm of them with
// its residual, as a model goes on, together stop losing by it.  Time through the caches against past them, mean (least to
// most) of ten tables of 32000 to 262144 rows and 1000 to 8192 columns, bf16 and fp32; the same buffers every time or
// others make no difference with a reader:
//   rows         80 MiB              96                   128                  144                 192
//   alone        +10% (0 to +22)     +17 (+10 to +25)     +23 (+8 to +32)      +27 (+8 to +37)     +36 (+12 to +48)
//   norm of sum  -0.6 (-5 to +4)     -0.2 (-4 to +5)      0.0 (-4 to +5)       +1.2 (-4 to +6)     +5 (-3 to +10)
//   norm alone   -3.3 (-7 to +1)     -3.0 (-7 to +2)      -1.9 (-7 to +4)      +0.3 (-6 to +7)     +7 (-3 to +14)
// The most is lost with 8192 columns of 128256 rows: of 128 MiB, and a norm alone, 86 us, 80 through the caches.
template <typename T, int G, bool kPast>
__global__ __launch_bounds__(kRowThreads) void ember_rows_q4(RowsParams p) {
    const Rows4Args& a = p.a;
    constexpr int kPieces = sizeof(T) / 2, kCols = 8 / kPieces;      // stores a lane, columns of each
    const int lane = threadIdx.x % kUnitLanes, q = lane % 4, w = kPieces == 1 ? lane / 4 : lane / 8;
    const int64_t row0 = (int64_t)blockIdx.x * p.rows_per_block;
    const int rows = (int)min((int64_t)p.rows_per_block, a.n - row0);
    const int units = rows * p.nblk, D = (int)a.D;
    for (int u0 = threadIdx.x / kUnitLanes; u0 < units; u0 += kAhead * kUnitsPerPass) {
        uint32_t codes[kAhead][kPieces], scale[kAhead][kPieces];
        int r[kAhead], s[kAhead];
        int64_t v[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int u = min(u0 + i * kUnitsPerPass, units - 1);
            r[i] = (int)div_small(u, p.magic);
            s[i] = u - r[i] * p.nblk;
            v[i] = a.tok ? a.tok[row0 + r[i]] : p.first + row0 + r[i];
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const bool in = v[i] >= 0 && v[i] < a.V;
            const int64_t at = in ? v[i] : 0;
#pragma unroll
            for (int j = 0; j < kPieces; ++j) {
                const int wj = w + 2 * j, g = min((s[i] * kBlockCols + 32 * wj) / G, (D - 1) / G);     // past the row: not used
                codes[i][j] = *reinterpret_cast<const uint32_t*>(a.Wq + at * a.ldw + s[i] * kBlockBytes + 16 * q + 4 * wj);
                scale[i][j] = in ? a.wscale[at * a.ldg + g] : 0x7FC0u;
            }
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (u0 + i * kUnitsPerPass >= units) break;
            T* const y = static_cast<T*>(a.Y) + (row0 + r[i]) * a.ldy;
            float x[kPieces][kCols];
#pragma unroll
            for (int j = 0; j < kPieces; ++j) {
                // the codes in the upper halves of bytes: of the pair's dwords the same half, or that of lanes 4 .. 7 of 8
                uint32_t c[2];
                if constexpr (kPieces == 1) {
                    const uint32_t other = of_lane<kPair>(codes[i][j]);
                    c[0] = q & 1 ? other : codes[i][j] << 4;
                    c[1] = q & 1 ? codes[i][j] : other << 4;
                } else {
                    c[0] = lane & 4 ? codes[i][j] : codes[i][j] << 4;
                }
                const float f = bf16_bits_f32(scale[i][j]);
#pragma unroll
                for (int e = 0; e < kCols; ++e) x[j][e] = (float)((int)(c[e / 4] << (24 - 8 * (e % 4))) >> 28) * f;
                const int col = kPieces == 1 ? first_col(s[i], lane) : s[i] * kBlockCols + 64 * j + 4 * lane;
                store_values<T, kCols, kPast>(y, col, D, x[j]);
            }
        }
    }
}

// Rows of a launch's blocks: about 64 blocks of codes each.
int rows_per_block(int nblk) { return std::max(1, 64 / nblk); }

template <typename T>
void launch_quantize(const QuantParams& p, unsigned grid, hipStream_t s) {
    if (p.a.group == 32) ember_quantize_q4<T, 32><<<grid, kRowThreads, 0, s>>>(p);
    else if (p.a.group == 64) ember_quantize_q4<T, 64><<<grid, kRowThreads, 0, s>>>(p);
    else ember_quantize_q4<T, 128><<<grid, kRowThreads, 0, s>>>(p);
}
template <typename T, bool kPast>
void launch_rows(const RowsParams& p, unsigned grid, hipStream_t s) {
    if (p.a.group == 32) ember_rows_q4<T, 32, kPast><<<grid, kRowThreads, 0, s>>>(p);
    else if (p.a.group == 64) ember_rows_q4<T, 64, kPast><<<grid, kRowThreads, 0, s>>>(p);
    else ember_rows_q4<T, 128, kPast><<<grid, kRowThreads, 0, s>>>(p);
}

// ---------------------------------------------------------------------------
// logits of few tokens
// ---------------------------------------------------------------------------

constexpr int kUnit = 4;                       // blocks of codes a unit: 512 columns
constexpr int kFewLds = 152 * 1024;

// kWide: 32 x 32 tiles, MT of them over the tokens; else one of 16 x 16.
template <bool kWide_, int MT_>
struct Stream {
    static constexpr bool kWide = kWide_;
    static constexpr int MT = MT_;
    static constexpr int kRows = kWide ? 32 : 16;           // channels of a strip, tokens of a tile
    static constexpr int kTokens = kRows * MT;
    static constexpr int kWaves = kWide ? 8 : 16;           // at most
    static constexpr int kThreads = kWaves * kWave;
    static constexpr int kDepth = 2;                        // units in registers
    static constexpr int kLoadsW = kWide ? 2 * kUnit : kUnit;    // 16-byte loads of a unit's codes
    static constexpr int kAcc = kWide ? 16 : 4;             // values of a tile a lane
    static constexpr int kLanes = kWide ? 2 : 4;            // lanes of a row
};

struct Few4Params {
    Logits4Args a;
    int nblk;            // blocks of codes a row
    int groups;
    int units;           // of a row
    int pitch;           // bytes of a token in LDS
    int window;          // units that the LDS holds of each token
    int share;           // waves that share a strip: each takes every share-th unit
    int waves;           // of a block
    int64_t strips;
    int together;        // neighbouring strips of a block (where a wave goes through several)
    bool several;        // a wave goes through several strips
    int tiles;           // of tokens
    int blocks;          // of a tile of tokens
};

// Few tokens, 16 to 64 a block: bound by the table's bytes.  A block holds the tokens'
// codes in LDS, in the order of the table's operands (all columns, or a window of them
// after the other); each wave streams strips of 16 or 32 channels straight from memory
// into registers, the next units' loads in flight.  The tokens are the rows of the
// MFMA tiles, so a lane's values are all of one channel, the one whose codes it
// loads, and need that channel's scale alone.  Where a table has few strips several
// waves share one, unit by unit, and add up in LDS.  Blocks of the same channels and
// other tokens are neighbours on one XCD, whose L2 then has the codes.  The order of
// a logit's sum depends on V and D, not on the number of tokens.
// 128256 x 4096: 1 token, groups of 128, 44 to 48 us (271 MB, 5.6 to 6.1 TB/s; reading alone 6.9); 16 tokens,
// groups of 32, 54 to 63, where no unit is full: the vector units work for 40% of the time (half of it on the sums'
// scaling), the matrix units for 10%, and a wave's loads, operands, MFMAs and scaling follow each other; 64 x 100000 x
// 1000, groups of 64, 26.
template <typename C, int G, typename YT>
__global__ __launch_bounds__(C::kThreads) void ember_logits_q4_few(Few4Params p) {
    const Logits4Args& a = p.a;
    constexpr int kPer = kBlockCols / G;                    // groups a block
    constexpr int kScaleBytes = kUnit * kPer * 2;           // of a unit: 8, 16 or 32
    constexpr int kScaleWords = kScaleBytes / 4;
    // A row's lanes load a part of its scales each, where all of them are more than 8 bytes (16 x 128256 x
    // 4096, groups of 32: 57 us, 59 when each loads all 32 bytes).
    constexpr int kScaleParts = kScaleWords == 2 ? 1 : C::kWide ? 2 : 4;
    typedef int acc_t __attribute__((ext_vector_type(C::kAcc)));
    typedef float facc_t __attribute__((ext_vector_type(C::kAcc)));
    __shared__ __attribute__((aligned(16))) uint8_t lds[kFewLds];
    __shared__ float xs[64];
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int row = lane % C::kRows, part = lane / C::kRows;
    const int nblk = p.nblk, D = (int)a.D;
    // block -> tile of tokens and block of channels: on an XCD the tiles of the same channels side by side
    const int in_xcd = blockIdx.x / kXcds, block = in_xcd / p.tiles * kXcds + blockIdx.x % kXcds;
    const int64_t t0 = (int64_t)(in_xcd % p.tiles) * C::kTokens;
    const int T = (int)min((int64_t)C::kTokens, a.T - t0);
    if (block >= p.blocks) return;

    // this wave's strips and units
    const int per_block = p.waves / p.share, mate = wave % p.share, place = wave / p.share;
    int64_t first, pass;
    if (p.several) {
        // `together` neighbours, then those of the grid's other blocks
        first = ((int64_t)block + (int64_t)p.blocks * (place / p.together)) * p.together + place % p.together;
        pass = (int64_t)p.blocks * per_block;
    } else {
        first = (int64_t)block * per_block + place;
        pass = p.strips;
    }
    const int mine = first < p.strips ? (int)((p.strips - 1 - first) / pass) + 1 : 0;
    auto channel = [&](int i) { return (first + i * pass) * C::kRows; };
    const int64_t row_bytes = (int64_t)nblk * kBlockBytes;
    const uint32_t off_w = (uint32_t)row * (uint32_t)a.ldw + part * (kBlockBytes / C::kLanes);
    const uint32_t off_s = (uint32_t)row * (uint32_t)a.ldg * 2 + lane / (kWave / kScaleParts) * (kScaleBytes / kScaleParts);
    auto buffer = [&](const void* base, int64_t bytes) {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0,
                                                 (int)(bytes < kBufferMax ? bytes : kBufferMax), kBufferWord3);
    };
    struct Unit {
        i32x4 w[C::kLoadsW];
        uint32_t s[kScaleWords / kScaleParts];
        float bias;
    };
    // unit u of strip i: zeros past the table (also for strips past it) and past the row
    auto load = [&](int i, int u, Unit& k) {
        const int64_t v = channel(i);
        const bool in = i < mine && v < a.V;
        const int64_t v_in = in ? v : 0, left = in ? a.V - 1 - v : 0;
        const auto rw = buffer(a.Wq + v_in * a.ldw, in ? left * a.ldw + row_bytes : 0);
        const auto rs = buffer(a.wscale + v_in * a.ldg, in ? (left * a.ldg + (p.groups + 7) / 8 * 8) * 2 : 0);
        const auto rb = buffer(a.bias ? a.bias + v_in : a.xscale, in && a.bias ? (left + 1) * 4 : 0);
#pragma unroll
        for (int b = 0; b < C::kLoadsW; ++b) {
            const int s = u * kUnit + b / (C::kLoadsW / kUnit);
            const uint32_t off = s < nblk ? off_w + s * kBlockBytes + b % (C::kLoadsW / kUnit) * 16 : kBufferMax;
            k.w[b] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rw, off, 0, 0));
        }
        // (groups past the row's are not used)
        const uint32_t off = u * kUnit * kPer < p.groups ? off_s + u * kScaleBytes : kBufferMax;
        constexpr int kWords = kScaleWords / kScaleParts;      // 1, 2 or 4
        if constexpr (kWords == 1) {
            k.s[0] = __builtin_amdgcn_raw_buffer_load_b32(rs, off, 0, 0);
        } else if constexpr (kWords == 2) {
            const u32x2_t d = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_raw_buffer_load_b64(rs, off, 0, 0));
            k.s[0] = d[0];
            k.s[1] = d[1];
        } else {
            const u32x4_t d = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rs, off, 0, 0));
#pragma unroll
            for (int e = 0; e < 4; ++e) k.s[e] = d[e];
        }
        k.bias = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rb, row * 4, 0, 0));
    };

    uint32_t at_x[C::MT];
#pragma unroll
    for (int m = 0; m < C::MT; ++m)       // rows past T: any token
        at_x[m] = (uint32_t)(min(C::kRows * m + row, T - 1) * p.pitch + part * 16);

    facc_t f[C::MT];
    auto clear = [&] {
#pragma unroll
        for (int m = 0; m < C::MT; ++m)
#pragma unroll
            for (int e = 0; e < C::kAcc; ++e) f[m][e] = 0.0f;
    };
    // u0: the unit that the LDS begins with
    auto multiply = [&](int u, int u0, const Unit& k) {
        // all lanes of a row get all of its scales: halves of the wave, then quarters exchanged
        uint32_t sw[kScaleWords];
        constexpr int kWords = kScaleWords / kScaleParts;
#pragma unroll
        for (int r = 0; r < kWords; ++r) {
            if constexpr (kScaleParts == 1) {
                sw[r] = k.s[r];
                continue;
            }
            const auto h = __builtin_amdgcn_permlane32_swap(k.s[r], k.s[r], false, false);
            if constexpr (kScaleParts == 2) {
                sw[r] = h[0];
                sw[kWords + r] = h[1];
            } else {
                const auto q0 = __builtin_amdgcn_permlane16_swap(h[0], h[0], false, false);
                const auto q2 = __builtin_amdgcn_permlane16_swap(h[1], h[1], false, false);
                sw[r] = q0[0];
                sw[kWords + r] = q0[1];
                sw[2 * kWords + r] = q2[0];
                sw[3 * kWords + r] = q2[1];
            }
        }
#pragma unroll
        for (int b = 0; b < kUnit; ++b) {
            const int s = u * kUnit + b;
            if (s >= nblk) continue;
            // A block's operands.  16 x 16 tiles: two of 64 columns, or four of 32; a lane's quarter
            // of the block's bytes holds them.  32 x 32 tiles: four of 32 columns, each a dword of
            // both quarters that a lane has.
            i32x4 op[C::kWide ? 4 : 2];
#pragma unroll
            for (int h = 0; h < (C::kWide ? 4 : 2); ++h) {
                const uint32_t d0 = C::kWide ? k.w[2 * b][h] : k.w[b][2 * h % 4];
                const uint32_t d1 = C::kWide ? k.w[2 * b + 1 < C::kLoadsW ? 2 * b + 1 : 0][h] : k.w[b][(2 * h + 1) % 4];
                op[h] = i32x4{(int)low_codes(d0), (int)high_codes(d0), (int)low_codes(d1), (int)high_codes(d1)};
            }
            float scale[kPer];
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                const int g = b * kPer + j;
                scale[j] = __uint_as_float((g & 1) ? sw[g / 2] & 0xFFFF0000u : sw[g / 2] << 16);
            }
#pragma unroll
            for (int m = 0; m < C::MT; ++m) {
                const uint8_t* x = lds + at_x[m] + (s - u0 * kUnit) * kBlockCols;
                acc_t zero;
#pragma unroll
                for (int e = 0; e < C::kAcc; ++e) zero[e] = 0;
                acc_t sum[kPer];
                if constexpr (C::kWide) {
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const i32x4 xw = *reinterpret_cast<const i32x4*>(x + 32 * w);
                        const int j = w * kPer / 4;
                        sum[j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(xw, op[w], w % (4 / kPer) == 0 ? zero : sum[j], 0, 0, 0);
                    }
                } else {
                    const i32x4 x0 = *reinterpret_cast<const i32x4*>(x);
                    const i32x4 x1 = *reinterpret_cast<const i32x4*>(x + 64);
                    if constexpr (G == 128) {
                        sum[0] = __builtin_amdgcn_mfma_i32_16x16x64_i8(x0, op[0], zero, 0, 0, 0);
                        sum[0] = __builtin_amdgcn_mfma_i32_16x16x64_i8(x1, op[1], sum[0], 0, 0, 0);
                    } else if constexpr (G == 64) {
                        sum[0] = __builtin_amdgcn_mfma_i32_16x16x64_i8(x0, op[0], zero, 0, 0, 0);
                        sum[1] = __builtin_amdgcn_mfma_i32_16x16x64_i8(x1, op[1], zero, 0, 0, 0);
                    } else {
                        typedef int i32x2 __attribute__((ext_vector_type(2)));
                        auto half = [](const i32x4& r, int h) {
                            return __builtin_bit_cast(long, h ? i32x2{r[2], r[3]} : i32x2{r[0], r[1]});
                        };
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            sum[j] = __builtin_amdgcn_mfma_i32_16x16x32_i8(half(j < 2 ? x0 : x1, j & 1),
                                                                           half(op[j >> 1], j & 1), zero, 0, 0, 0);
                    }
                }
#pragma unroll
                for (int j = 0; j < kPer; ++j) {
                    // no group: what stands in its place is not a scale
                    if (kPer > 1 && s * kPer + j >= p.groups) continue;
#pragma unroll
                    for (int e = 0; e < C::kAcc; ++e) f[m][e] = fmaf((float)sum[j][e], scale[j], f[m][e]);
                }
                if (C::kWide) __builtin_amdgcn_sched_barrier(0);    // more tiles at once take more registers
            }
        }
    };
    auto store = [&](int i, float bias) {
        int l = lane;
        asm volatile("" : "+v"(l));   // what follows from it is not kept in registers over the loop
        const int64_t v = channel(i) + l % C::kRows;
        if (i >= mine || v >= a.V) return;
        const int tl = l / C::kRows * 4;
        YT* const y0 = static_cast<YT*>(a.Y) + t0 * a.ldy + v;
#pragma unroll
        for (int m = 0; m < C::MT; ++m) {
#pragma unroll
            for (int e = 0; e < C::kAcc; ++e) {
                const int t = C::kWide ? 32 * m + 8 * (e / 4) + tl + e % 4 : tl + e;
                if (t >= T) continue;
                const float y = fmaf(f[m][e], xs[t], bias);
                if constexpr (sizeof(YT) == 4) y0[t * a.ldy] = y;
                else y0[t * a.ldy] = (uint16_t)pack_bf16(y, 0.0f);
            }
        }
    };

    Unit k[C::kDepth];
    int i = 0, u = mate;         // the next unit to multiply
    int il = 0, ul = mate;       // and to load
    const int slots = p.several ? p.units : (p.units + p.window - 1) / p.window * p.window;
    auto next = [&](int& i, int& u) {
        if ((u += p.share) >= slots) u = mate, ++i;
    };
#pragma unroll
    for (int d = 0; d < C::kDepth - 1; ++d) {
        load(il, ul, k[d]);
        next(il, ul);
    }
    if ((int)threadIdx.x < T) xs[threadIdx.x] = a.xscale[t0 + threadIdx.x] * 0.0625f;    // operands are 16 times the codes
    clear();
    float bias = 0.0f;
    for (int u0 = 0; u0 < p.units; u0 += p.window) {
        // the tokens' codes of the window, 16 columns a thread: columns 4 q .. of the 16 go to
        // the 16 bytes that their lane reads
        if (u0 > 0) __syncthreads();
        const int cols = min(p.window, p.units - u0) * kUnit * 8;     // of 16 columns
        const int all = T * cols, threads = p.waves * kWave;
        for (int n0 = threadIdx.x; n0 < all; n0 += 4 * threads) {      // four loads in flight
            i32x4 x[4];
            uint32_t to[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if (__builtin_amdgcn_readfirstlane(n0) + q * threads >= all) break;      // for the whole wave
                const int n = min(n0 + q * threads, all - 1), t = n / cols, c = n - t * cols;
                const int k0 = (u0 * kUnit * 8 + c) * 16;
                // (the padding up to 16 columns is readable)
                x[q] = *reinterpret_cast<const i32x4*>(a.Xq + (t0 + t) * a.ldx + (k0 < D ? k0 : 0));
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int left = D - k0 - 4 * j;
                    x[q][j] &= left >= 4 ? -1 : left <= 0 ? 0 : (int)((1u << (8 * left)) - 1);
                }
                const int w = c % 8 / 2, h = c % 2;
                to[q] = t * p.pitch + c / 8 * kBlockCols + (C::kWide ? w * 32 : (w >> 1) * 64 + (w & 1) * 8) + h * 4;
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if (n0 + q * threads >= all) continue;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    *reinterpret_cast<int*>(lds + to[q] + (C::kWide ? (j >> 1) * 16 + (j & 1) * 8 : j * 16)) = x[q][j];
            }
        }
        __syncthreads();
        // as many steps for each wave, a multiple of the depth: past its units (of its strips) they are empty
        const int total = p.several ? mine * p.units : p.window / p.share;
        for (int n = 0; n < total; n += C::kDepth) {
#pragma unroll
            for (int d = 0; d < C::kDepth; ++d) {
                load(il, ul, k[(d + C::kDepth - 1) % C::kDepth]);
                next(il, ul);
                __builtin_amdgcn_sched_barrier(0);
                multiply(u, u0, k[d]);
                if (u < p.units && u + p.share >= p.units) {
                    bias = k[d].bias;
                    if (p.share == 1) {
                        store(i, bias);
                        clear();
                    }
                }
                next(i, u);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
    if (p.share > 1) {
        // the others' sums join the first's, in order
        float* const sums = reinterpret_cast<float*>(lds);
        __syncthreads();
#pragma unroll
        for (int m = 0; m < C::MT; ++m)
#pragma unroll
            for (int e = 0; e < C::kAcc; ++e) sums[((wave * C::MT + m) * C::kAcc + e) * kWave + lane] = f[m][e];
        __syncthreads();
        if (mate > 0) return;
        const int64_t v = channel(0) + row;
        bias = a.bias && v < a.V && mine ? a.bias[v] : 0.0f;
        for (int q = 1; q < p.share; ++q) {
#pragma unroll
            for (int m = 0; m < C::MT; ++m)
#pragma unroll
                for (int e = 0; e < C::kAcc; ++e) f[m][e] += sums[(((wave + q) * C::MT + m) * C::kAcc + e) * kWave + lane];
        }
        store(0, bias);
    }
}

// ---------------------------------------------------------------------------
// logits of many tokens
// ---------------------------------------------------------------------------

struct Tile4Params {
    Logits4Args a;
    int nk;              // blocks of codes a row: steps
    int groups;
    int MT;
    int64_t NT;
    int64_t tiles, per_xcd;
    int group_m;
};

// BM tokens x 32 channels a wave, WN waves side by side, GROUPS times: each group of waves
// takes every GROUPS-th step.
template <int BM_, int WN_, int STAGES_, int GROUPS_ = 1>
struct Tile4 {
    static constexpr int BM = BM_, BN = 32 * WN_;  // tokens, channels a block
    static constexpr int kStages = STAGES_;
    static constexpr int kWaves = WN_, kGroups = GROUPS_;
    static constexpr int kThreads = kGroups * kWaves * kWave;
    static constexpr int MT = BM / 32;             // MFMA tiles a wave
    static constexpr int kX = BM * kBlockCols, kW = BN * kBlockBytes;                 // bytes of a stage
    static constexpr int kS = BN * 16, kScales = 3;                                   // of a period's scales, and of these
    static constexpr int kLoadsX = BM / 8 / kWaves, kLoadsW = BN / 16 / kWaves;       // a wave and step
    static constexpr int kLoads = kLoadsX + kLoadsW + 1;
    static constexpr int kStageBytes = kX + kW;
    static constexpr int kRing = kStages * kStageBytes, kNone = kRing + kScales * kS;    // kNone: what loads outside a buffer write
    static constexpr int kGroupLds = kNone + 1024;                                    // a group's
    static constexpr int kXs = kGroups * kGroupLds, kLds = kXs + BM * 4;
    static constexpr int kSumBytes = kWaves * MT * 16 * kWave * 4;                    // a group's sums
    static_assert(BM % (8 * kWaves) == 0 && kWaves % 2 == 0 && MT % 2 == 0, "equal loads a wave, even tiles");
    static_assert(kStages >= 2 && kStages <= 4 && (kStages - 2) * kLoads < 64, "vmcnt range, scales of the steps ahead");
    static_assert(kGroups == 1 || (kGroups == 2 && kSumBytes <= kGroupLds), "whole periods of scales; the second group's sums");
    static_assert(BN % kWave == 0 && BN / kWave <= kWaves, "the scales' loads");
    static_assert((int64_t)std::max(BM, BN) * EMBER_Q8_MAX_LD < (int64_t)1 << 31, "32-bit load offsets");
    static constexpr int kBlocks = 160 * 1024 / kLds;    // a compute unit
    static_assert(kBlocks > 0, "LDS of one CU");
};

// BM tokens x BN channels a block, a block of 128 columns a step.  A ring of LDS
// stages holds the tokens' codes and the table's; beside it are 16 bytes of scales a
// channel (eight groups: two to eight steps), loaded with the first of their steps.
// Every group's sum has to be turned into fp32, scaled and added: 32 vector instructions
// for each 32 x 32 tile, as long as the MFMAs of 128 columns take.  So these are laid
// between the next sum's MFMAs, each wave has all of the block's tokens (the codes' halves
// are taken apart once), and the step barrier sits before the last tile of tokens, whose
// operands are in registers by then.  1024 x 128256 x 4096, groups of 128, bf16 logits: 660 to
// 720 us by card (the first dozen launches up to 780), 1.5 to 1.6 POPS (the int8 library product, without scales:
// 2.0); the vector units have 55% of the time, the matrix units 36%, and they hardly overlap.
template <typename C, int G, typename YT>
__global__ __launch_bounds__(C::kThreads) void ember_logits_q4(Tile4Params p) {
    __shared__ __attribute__((aligned(1024))) uint8_t lds[C::kLds];
    const Logits4Args& a = p.a;
    constexpr int kPer = kBlockCols / G;
    const int lane = threadIdx.x & (kWave - 1);
    const int group = C::kGroups == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / (C::kWaves * kWave));
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave) - group * C::kWaves;      // of the group
    uint8_t* const own = lds + group * C::kGroupLds;
    const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)own;
    // this block's tiles: every gridDim.x / kXcds-th of its XCD's
    const int64_t xcd = blockIdx.x % kXcds, end = min((xcd + 1) * p.per_xcd, p.tiles);
    int64_t l = xcd * p.per_xcd + blockIdx.x / kXcds;
    if (l >= end) return;
    const int D = (int)a.D;

    const int row_x = wave * 8 + lane / 8, row_w = wave * 16 + lane / 4;
    const int k_x = ((lane % 8) ^ swizzle<8>(row_x)) * 16, k_w = ((lane % 4) ^ swizzle<4>(row_w)) * 16;
    const int row_s = wave < C::BN / kWave ? wave * kWave + lane : 0;      // the first waves load the scales
    const uint32_t off_x = row_x * (uint32_t)a.ldx + k_x, off_w = row_w * (uint32_t)a.ldw + k_w;
    const uint32_t off_s = row_s * (uint32_t)(2 * a.ldg);
    // all of a load's place in the offset that the buffer's range is checked against; past the
    // last step they are outside it
    int64_t t0, v0;
    i32x4 rx, rw, rs;
    auto go_to = [&](int64_t l) {
        int tm;
        int64_t tn;
        tile_at(p.MT, p.NT, p.group_m, l, tm, tn);
        t0 = (int64_t)tm * C::BM, v0 = tn * C::BN;
        rx = rsrc(a.Xq + t0 * a.ldx, (a.T - t0) * a.ldx);
        rw = rsrc(a.Wq + v0 * a.ldw, (a.V - v0) * a.ldw);
        rs = rsrc(a.wscale + v0 * a.ldg, (a.V - v0) * a.ldg * 2);
    };
    // step i of the group: the row's step kt
    auto step_of = [&](int i) { return C::kGroups * i + group; };
    const int steps = (p.nk + C::kGroups - 1) / C::kGroups;
    auto issue = [&](int i, uint32_t st) {
        const int kt = step_of(i);
        const uint32_t ox = kt * kBlockCols + k_x < D ? off_x + kt * kBlockCols : kBufferMax;
        const uint32_t ow = off_w + (kt < p.nk ? (uint32_t)kt * kBlockBytes : kBufferMax);
        // Scales: 16 bytes of a row each, so 64 rows a load, and slow.  In the other steps (and waves)
        // the load stays, outside the buffer, so that all steps have as many.
        constexpr int kPeriod = 8 / kPer;
        const bool scales = kt % kPeriod == group && kt < p.nk && wave < C::BN / kWave;
        const uint32_t os = off_s + (scales ? (uint32_t)(kt / kPeriod * 16) : kBufferMax);
        const uint32_t to_s = scales ? C::kRing + kt / kPeriod % C::kScales * C::kS + wave * 1024 : C::kNone;
        load_to_lds(rs, lds_base + to_s, os);
#pragma unroll
        for (int j = 0; j < C::kLoadsX; ++j)
            load_to_lds(rx, lds_base + st + (wave + C::kWaves * j) * 1024, ox + j * (C::kWaves * 8 * (uint32_t)a.ldx));
#pragma unroll
        for (int j = 0; j < C::kLoadsW; ++j)
            load_to_lds(rw, lds_base + st + C::kX + (wave + C::kWaves * j) * 1024, ow + j * (C::kWaves * 16 * (uint32_t)a.ldw));
    };
    const int half = lane >> 5, sh = half ? 0 : 4, col = lane & 31, ch = wave * 32 + col;
    const auto* const ring = (const __attribute__((address_space(3))) uint8_t*)own;      // stages: offsets in it
    auto lds_at = [&](uint32_t at, int more) { return *(const __attribute__((address_space(3))) i32x4*)(ring + at + more); };
    // operands: a tile's tokens, 32 columns each; a block's codes, dword w of quarter t; scales
    uint32_t at_x[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) at_x[w] = col * kBlockCols + (((2 * w + half) ^ swizzle<8>(col)) * 16);
    uint32_t at_w[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) at_w[t] = ch * kBlockBytes + ((t ^ swizzle<4>(ch)) * 16);
    // (masked: the group's last step, where a D that is not a multiple of 16 has a chunk of columns that do not count)
    uint32_t here[4];       // of the stage
    auto read_x = [&](int m, i32x4 (&x)[4], bool masked) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            x[w] = lds_at(here[w], m * (32 * kBlockCols));
            if (!masked) continue;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int b = D - step_of(steps - 1) * kBlockCols - 32 * w - 16 * half - 4 * e;
                x[w][e] &= b >= 4 ? -1 : b <= 0 ? 0 : (int)((1u << (8 * b)) - 1);
            }
        }
    };
    auto read_w = [&](uint32_t st, i32x4 (&wd)[4]) {
#pragma unroll
        for (int t = 0; t < 4; ++t) wd[t] = lds_at(st + at_w[t], C::kX);
    };
    auto read_s = [&](int i, float (&s)[kPer]) {
        const int kt = step_of(i);
        const uint32_t at = kt * kPer / 8 % C::kScales * C::kS + ch * 16 + kt * kPer % 8 * 2;
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const uint32_t h = *(const __attribute__((address_space(3))) uint16_t*)(ring + at + (C::kRing + 2 * j));
            // no group: what stands in its place is not a scale
            s[j] = (kPer == 1 && C::kGroups == 1) || kt * kPer + j < p.groups ? bf16_bits_f32(h) : 0.0f;
        }
    };
    auto take_apart = [&](const i32x4 (&wd)[4], i32x4 (&op)[4]) {
#pragma unroll
        for (int w = 0; w < 4; ++w)
#pragma unroll
            for (int t = 0; t < 4; ++t) op[w][t] = (int)(((uint32_t)wd[t][w] << sh) & 0xF0F0F0F0u);
    };

    f32x16 f[C::MT];
    i32x16 sum[2], zero;
#pragma unroll
    for (int e = 0; e < 16; ++e) zero[e] = 0;

    // for the epilogue; the operands are 16 times the codes
    float* const xs = reinterpret_cast<float*>(lds + C::kXs);
    float my_xs, bias;
    auto factors = [&] {
        const int64_t my_t = t0 + threadIdx.x, my_v = v0 + ch;
        my_xs = (int)threadIdx.x < C::BM && my_t < a.T ? a.xscale[my_t] * 0.0625f : 0.0f;
        bias = a.bias && my_v < a.V ? a.bias[my_v] : 0.0f;
    };
    i32x4 op[4], wd[4], x[2][4];
    float scale[kPer], last;         // this step's, and that of the sum that is not added yet
    uint32_t st;
    auto step = [&](int i, auto is_last) {
        constexpr bool kLast = decltype(is_last)::value;
        const uint32_t next = st + C::kStageBytes == C::kRing ? 0 : st + C::kStageBytes;
        float then[kPer];
#pragma unroll
        for (int m = 0; m < C::MT; ++m) {
            if (m + 1 < C::MT) {
                read_x(m + 1, x[(m + 1) & 1], kLast);
            } else if (!kLast) {
                // Everyone's operands of this stage are in registers, so step i + kStages may fill
                // it; of each wave's loads those of step i + 2 and later may be out.
                wait_step<(C::kStages - 2) * C::kLoads>();
                issue(i + C::kStages, st);
                read_w(next, wd);
                read_s(i + 1, then);
#pragma unroll
                for (int w = 0; w < 4; ++w) here[w] = next + at_x[w];
                read_x(0, x[0], false);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                constexpr int kRun = 4 / kPer;                 // MFMAs of a group
                const int n = (m * 4 + w) / kRun, cur = n & 1;
                sum[cur] = __builtin_amdgcn_mfma_i32_32x32x32_i8(x[m & 1][w], op[w], w % kRun == 0 ? zero : sum[cur], 0, 0, 0);
                // a part of the sum before
                const int before = (n + C::MT * kPer - 1) % (C::MT * kPer);
                const float s = n == 0 ? last : scale[before % kPer];
#pragma unroll
                for (int e = 0; e < 16 / kRun; ++e) {
                    const int q = w % kRun * (16 / kRun) + e;
                    f[before / kPer][q] = fmaf((float)sum[cur ^ 1][q], s, f[before / kPer][q]);
                }
                asm volatile("" : "+v"(f[before / kPer]));     // here, not past the step
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        last = scale[kPer - 1];
        if (kLast) return;
#pragma unroll
        for (int j = 0; j < kPer; ++j) scale[j] = then[j];
        take_apart(wd, op);
        st = next;
    };
    // A lane holds 16 tokens of a channel: through a strip of LDS of the wave's own, 32
    // tokens x 32 channels, each token's are stored side by side.  The strips take the ring's
    // last stages; the first of the next tile are loaded meanwhile.
    constexpr int kEs = (int)sizeof(YT), kPitch = 32 * kEs + 16, kEpc = 16 / kEs, kPerRow = 32 / kEpc;
    constexpr int kAhead = C::kStages - (C::kWaves * 32 * kPitch + C::kStageBytes - 1) / C::kStageBytes;
    static_assert(C::kGroups == 1 || C::kSumBytes + C::kWaves * 32 * kPitch <= C::kGroups * C::kGroupLds, "sums and strips");
    static_assert(kAhead >= 1, "the strips");
    uint8_t* const strip = lds + (C::kGroups == 1 ? kAhead * C::kStageBytes : C::kSumBytes) + wave * (32 * kPitch);
    int el = lane;
    auto store = [&](int64_t t0, int64_t v0, float bias) {
        asm volatile("" : "+v"(el));   // what follows from it is not kept in registers over the steps
        const int eh = el >> 5, ec = el & 31;
#pragma unroll
        for (int m = 0; m < C::MT; ++m) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int r = 8 * (e / 4) + 4 * eh + e % 4;
                const float y = fmaf(f[m][e], xs[32 * m + r], bias);
                if constexpr (kEs == 4) *reinterpret_cast<float*>(strip + r * kPitch + ec * 4) = y;
                else *reinterpret_cast<uint16_t*>(strip + r * kPitch + ec * 2) = (uint16_t)pack_bf16(y, 0.0f);
            }
            wave_lds_order();
#pragma unroll
            for (int q = 0; q < 32 * kPerRow / kWave; ++q) {
                const int r = (q * kWave + el) / kPerRow, c = el % kPerRow * kEpc;
                const int64_t t = t0 + 32 * m + r, v = v0 + wave * 32 + c;
                const u32x4_t y = *reinterpret_cast<const u32x4_t*>(strip + r * kPitch + c * kEs);
                if (t >= a.T) continue;
                YT* const to = static_cast<YT*>(a.Y) + t * a.ldy + v;
                if (v + kEpc <= a.V) {
                    *reinterpret_cast<u32x4_t*>(to) = y;
                } else {
#pragma unroll
                    for (int e = 0; e < kEpc; ++e) {
                        if (v + e >= a.V) continue;
                        if constexpr (kEs == 4) reinterpret_cast<uint32_t*>(to)[e] = y[e];
                        else reinterpret_cast<uint16_t*>(to)[e] = (uint16_t)(y[e >> 1] >> (16 * (e & 1)));
                    }
                }
            }
            wave_lds_order();
        }
    };

    go_to(l);
    factors();
#pragma unroll
    for (int q = 0; q < C::kStages; ++q) issue(q, q * C::kStageBytes);
    for (;;) {
        if ((int)threadIdx.x < C::BM) xs[threadIdx.x] = my_xs;
#pragma unroll
        for (int e = 0; e < 16; ++e) sum[0][e] = sum[1][e] = 0;
#pragma unroll
        for (int m = 0; m < C::MT; ++m)
#pragma unroll
            for (int e = 0; e < 16; ++e) f[m][e] = 0.0f;
        last = 0.0f;
        st = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) here[w] = at_x[w];
        wait_step<(C::kStages - 1) * C::kLoads>();
        read_w(0, wd);
        read_s(0, scale);
        read_x(0, x[0], steps == 1);
        take_apart(wd, op);
        for (int i = 0; i < steps - 1; ++i) step(i, std::false_type());
        if (steps > 1) read_x(0, x[0], true);
        step(steps - 1, std::true_type());
#pragma unroll
        for (int e = 0; e < 16; ++e) f[C::MT - 1][e] = fmaf((float)sum[1][e], last, f[C::MT - 1][e]);
        wait_step<0>();    // the zero-filling loads past the end have landed, and everyone is done with the stages
        if constexpr (C::kGroups > 1) {
            // one tile: the second group's sums join the first's
            float* const sums = reinterpret_cast<float*>(lds) + wave * (C::MT * 16 * kWave) + lane;
            if (group > 0) {
#pragma unroll
                for (int m = 0; m < C::MT; ++m)
#pragma unroll
                    for (int e = 0; e < 16; ++e) sums[(m * 16 + e) * kWave] = f[m][e];
            }
            __syncthreads();
            if (group > 0) return;
#pragma unroll
            for (int m = 0; m < C::MT; ++m)
#pragma unroll
                for (int e = 0; e < 16; ++e) f[m][e] += sums[(m * 16 + e) * kWave];
            store(t0, v0, bias);
            return;
        }
        const int64_t t_done = t0, v_done = v0;
        const float bias_done = bias;
        l += gridDim.x / kXcds;
        const bool more = l < end;
        if (more) {
            go_to(l);
            factors();
#pragma unroll
            for (int q = 0; q < kAhead; ++q) issue(q, q * C::kStageBytes);
        }
        store(t_done, v_done, bias_done);
        if (!more) return;
        wait_step<63>();   // everyone is done with the strips and xs (no load is waited for)
#pragma unroll
        for (int q = kAhead; q < C::kStages; ++q) issue(q, q * C::kStageBytes);
    }
}

// Bytes of a token's units in LDS.  They end 16 bytes past a multiple of the banks: the
// lanes of a part read different ones.
int64_t few_pitch(int64_t units) { return (units * kUnit * kBlockCols + 255) / 256 * 256 + 16; }
static_assert(16 * (4 * 2 * kUnit * kBlockCols + 16) <= kFewLds, "16 tokens: a window for four waves, two units deep");

template <typename C, int G>
hipError_t launch_few(const Logits4Args& a, hipStream_t s) {
    Few4Params p;
    p.a = a;
    p.nblk = (int)((a.D + kBlockCols - 1) / kBlockCols);
    p.groups = (int)((a.D + G - 1) / G);
    p.units = (p.nblk + kUnit - 1) / kUnit;
    // Waves that share a strip of 32 channels (of 16: as many, so that the order of the sums
    // is the same): up to four, where there would be fewer than 1024 at work.
    const int64_t strips32 = (a.V + 31) / 32;
    p.share = 1;
    while (p.share < 4 && p.share * 2 <= p.units && strips32 * p.share < 1024) p.share *= 2;
    p.strips = (a.V + C::kRows - 1) / C::kRows;
    p.tiles = (int)((a.T + C::kTokens - 1) / C::kTokens);
    const int64_t T = std::min<int64_t>(a.T, C::kTokens);
    p.several = p.share == 1 && T * few_pitch(p.units) <= kFewLds;
    const int step = p.share * C::kDepth;      // a window has whole rounds of the registers' units
    p.window = p.several ? p.units : (p.units + step - 1) / step * step;
    while (!p.several && p.window > 0 && T * few_pitch(p.window) > kFewLds) p.window -= step;
    if (p.window < step && !p.several) return hipErrorInvalidValue;
    p.pitch = (int)few_pitch(p.window);
    // few waves to a block where there would be less than a block for each compute unit
    p.waves = C::kWaves;
    while (p.waves > 8 && p.strips * p.share * p.tiles < (int64_t)p.waves * kCus * 3 / 4) p.waves /= 2;
    const int64_t per_block = p.waves / p.share;
    p.together = p.strips >= 4 * kCus ? 4 : 1;
    const int64_t all = p.several ? (p.strips + p.together - 1) / p.together : (p.strips + per_block - 1) / per_block;
    p.blocks = (int)(p.several ? std::min<int64_t>(all, std::max(1, kCus / p.tiles)) : all);
    const dim3 grid((unsigned)((p.blocks + kXcds - 1) / kXcds * kXcds * p.tiles));
    if (a.y_dtype == EMBER_F32) ember_logits_q4_few<C, G, float><<<grid, p.waves * kWave, 0, s>>>(p);
    else ember_logits_q4_few<C, G, uint16_t><<<grid, p.waves * kWave, 0, s>>>(p);
    return hipGetLastError();
}

template <typename C, int G, typename YT>
void launch_tile(const Tile4Params& p, unsigned grid, hipStream_t s) {
    ember_logits_q4<C, G, YT><<<grid, C::kThreads, 0, s>>>(p);
}

template <typename C, int G>
hipError_t launch_tiles(const Logits4Args& a, hipStream_t s) {
    Tile4Params p;
    p.a = a;
    p.nk = (int)((a.D + kBlockCols - 1) / kBlockCols);
    p.groups = (int)((a.D + G - 1) / G);
    p.MT = (int)((a.T + C::BM - 1) / C::BM);
    p.NT = (a.V + C::BN - 1) / C::BN;
    p.group_m = 4;
    p.tiles = (int64_t)p.MT * p.NT;
    p.per_xcd = (p.tiles + kXcds - 1) / kXcds;
    // The blocks that are there at once go through the tiles, so that the next one's first loads are
    // out while one is stored (1024 x 131072: 690 us at D = 4096 and 230 at 1024; a tile a block 720
    // and 245); of few steps, with nothing to hide the stores behind, a tile a block (172 at 512; 181).
    const int64_t blocks = p.nk < 6 || C::kGroups > 1 ? kMaxGridBlocks : kCus * C::kBlocks;
    const unsigned grid = (unsigned)(std::min<int64_t>(p.per_xcd, blocks / kXcds) * kXcds);
    if (a.y_dtype == EMBER_F32) launch_tile<C, G, float>(p, grid, s);
    else launch_tile<C, G, uint16_t>(p, grid, s);
    return hipGetLastError();
}

using T128x256 = Tile4<128, 8, 4>;
using T64x128 = Tile4<64, 4, 3>;       // two a compute unit
using T64x128Two = Tile4<64, 4, 3, 2>;

// Whether the large tiling is the faster one: by rounds of the chip's compute units, of which
// the small tiling's hold two blocks (the second costs 0.6 of the first), a round of large
// tiles being 2.2 of its own (fitted to 96 to 1024 tokens, 2000 to 100000 channels, D = 1000 and
// 4096, all group sizes: what it takes is never more than 1% slower than the other; 512 x 32000
// x 4096, groups of 128: 82 us, 115 in small tiles; 333 x 8191 x 1000, groups of 64, in small ones: bf16 logits
// 14.8, 19.4 in large; fp32 with a bias 16.9 and 21.7).
bool large_tiles(const Logits4Args& a) {
    const auto tiles = [&](int BM, int BN) { return (double)((a.T + BM - 1) / BM) * (double)((a.V + BN - 1) / BN) / kCus; };
    const double small = tiles(T64x128::BM, T64x128::BN);
    return 2.2 * std::ceil(tiles(T128x256::BM, T128x256::BN)) <= (small <= 1.0 ? 1.0 : 0.8 * std::ceil(small));
}

// Up to 16 tokens the streaming form.  Up to 64 it is the faster one
//   - in tiles of 16 tokens for small tables, as long as these are few: several tiles' blocks fill the
//     chip and the codes come from the caches (us, D = 2048, groups of 128: 64 x 4000 8.4, 12.5 with the
//     tiling; 64 x 8000 15.3 and 12.5; groups of 32 16.8 and 17.8, but 64 x 16000 32 and 18);
//   - in tiles of 32 or 64 tokens whose codes fit the LDS for large ones: of up to 32 tokens (32 x 60000 x
//     2048 17.7, 19.0 with the tiling), of more where the small tiling takes more than one round (64 x 60000
//     x 2048 24 and 20, 64 x 128256 x 2048, groups of 64, 42 and 44);
//   - in tiles of 16 for up to 32 tokens that do not fit, where groups of 32 or 64 keep the tiling's vector
//     units (32 x 60000 x 8192: groups of 32 88 and 104, of 64 82 and 75, of 128 81 and 57; of 64 it is the
//     faster one in 14 of 20 shapes of 34000 to 128256 channels and 4700 to 8192 columns, 32 x 34000 x 8192 54 and 74,
//     and 13% slower at most).
template <int G>
hipError_t launch_group(const Logits4Args& a, hipStream_t s) {
    const int64_t pitch = few_pitch((a.D + kUnit * kBlockCols - 1) / (kUnit * kBlockCols));
    const int64_t strips = (a.T + 15) / 16 * ((a.V + 15) / 16);
    const int64_t tiles = (a.T + T64x128::BM - 1) / T64x128::BM * ((a.V + T64x128::BN - 1) / T64x128::BN);
    if (a.T <= 16) return launch_few<Stream<false, 1>, G>(a, s);
    if (a.T <= 64 && a.V < 16384 && strips < (G == 128 ? 1500 : 3000)) return launch_few<Stream<false, 1>, G>(a, s);
    if (a.T <= 32 && a.V >= 16384) {
        if (32 * pitch <= kFewLds) return launch_few<Stream<true, 1>, G>(a, s);
        if (G < 128 && tiles > kCus) return launch_few<Stream<false, 1>, G>(a, s);
    }
    if (a.T <= 64 && 64 * pitch <= kFewLds && tiles > 2 * kCus) return launch_few<Stream<true, 2>, G>(a, s);
    if (a.T > 64 && large_tiles(a)) return launch_tiles<T128x256, G>(a, s);
    // where each compute unit has one small tile at most, two groups of waves share its steps (us: 200 x
    // 8000 x 8192, groups of 32, 55, one group 84; 96 x 8191 x 1000, groups of 64, 10.2 and 11.6)
    return tiles <= kCus ? launch_tiles<T64x128Two, G>(a, s) : launch_tiles<T64x128, G>(a, s);
}

} // namespace

// (a launch's blocks are limited, so rows go in parts)
hipError_t launch_quantize4(const Quant4Args& a, hipStream_t s) {
    QuantParams p;
    p.a = a;
    p.nblk = (int)((a.D + kBlockCols - 1) / kBlockCols);
    p.groups = (int)((a.D + a.group - 1) / a.group);
    p.magic = magic_of(p.nblk);
    p.rows_per_block = rows_per_block(p.nblk);
    const int64_t part = kMaxGridBlocks * p.rows_per_block;
    for (int64_t row = 0; row < a.rows; row += part) {
        p.a.X = static_cast<const char*>(a.X) + row * a.ldx * (a.x_dtype == EMBER_F32 ? 4 : 2);
        p.a.Q = a.Q + row * a.ldq;
        p.a.gscale = a.gscale + row * a.ldg;
        p.a.rows = std::min(part, a.rows - row);
        const unsigned grid = (unsigned)((p.a.rows + p.rows_per_block - 1) / p.rows_per_block);
        if (a.x_dtype == EMBER_F32) launch_quantize<float>(p, grid, s);
        else launch_quantize<uint16_t>(p, grid, s);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_rows4(const Rows4Args& a, hipStream_t s) {
    RowsParams p;
    p.a = a;
    p.nblk = (int)((a.D + kBlockCols - 1) / kBlockCols);
    p.magic = magic_of(p.nblk);
    p.rows_per_block = rows_per_block(p.nblk);
    const int es = a.y_dtype == EMBER_F32 ? 4 : 2;
    const bool past = a.n * a.D * es >= kPastBytes;
    const int64_t part = kMaxGridBlocks * p.rows_per_block;
    for (int64_t row = 0; row < a.n; row += part) {
        p.a.Y = static_cast<char*>(a.Y) + row * a.ldy * es;
        if (a.tok) p.a.tok = a.tok + row;
        p.first = row;
        p.a.n = std::min(part, a.n - row);
        const unsigned grid = (unsigned)((p.a.n + p.rows_per_block - 1) / p.rows_per_block);
        if (a.y_dtype == EMBER_F32) past ? launch_rows<float, true>(p, grid, s) : launch_rows<float, false>(p, grid, s);
        else past ? launch_rows<uint16_t, true>(p, grid, s) : launch_rows<uint16_t, false>(p, grid, s);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_logits4(const Logits4Args& a, hipStream_t s) {
    if (a.group == 32) return launch_group<32>(a, s);
    if (a.group == 64) return launch_group<64>(a, s);
    return launch_group<128>(a, s);
}

} // namespace ember
