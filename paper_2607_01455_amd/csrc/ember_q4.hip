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

#include "ember_device.h"
#include "ember_interface_launch.h"
#include "ember_tile.h"

namespace ember {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
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
constexpr int kUnitLanes = 16;                            // lanes a block of codes, one dword each
constexpr int kUnitsPerPass = kRowThreads / kUnitLanes;   // blocks of codes side by side

// Columns [col, col + 4) of a row, zeros past D.
template <typename T>
__device__ __forceinline__ f32x4 load4(const T* row, int col, int D) {
    f32x4 v = {0, 0, 0, 0};
    if (col + 4 <= D) {
        if constexpr (sizeof(T) == 4) {
            v = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(row + col));
        } else {
            const u32x2_t w = __builtin_nontemporal_load(reinterpret_cast<const u32x2_t*>(row + col));
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[e] = __uint_as_float((e & 1) ? w[e >> 1] & 0xFFFF0000u : w[e >> 1] << 16);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (col + e < D) v[e] = load_elem(row, col + e, sizeof(T) == 2);
    }
    return v;
}

struct QuantParams {
    Quant4Args a;
    int nblk;            // blocks of codes a row
    int groups;          // groups a row
    uint32_t magic;      // of nblk
    int rows_per_block;
};

// A lane rounds the eight columns of one dword; a group is 4, 8 or 16 lanes.
template <typename T, int G>
__global__ __launch_bounds__(kRowThreads) void ember_quantize_q4(QuantParams p) {
    const Quant4Args& a = p.a;
    const int lane = threadIdx.x % kUnitLanes, w = lane / 4, q = lane % 4;
    const int64_t row0 = (int64_t)blockIdx.x * p.rows_per_block;
    const int rows = (int)min((int64_t)p.rows_per_block, a.rows - row0);
    const int units = rows * p.nblk, D = (int)a.D;
    for (int u = threadIdx.x / kUnitLanes; u < units; u += kUnitsPerPass) {
        const int r = (int)div_small(u, p.magic), s = u - r * p.nblk;
        const T* x = static_cast<const T*>(a.X) + (row0 + r) * a.ldx;
        const int col = s * kBlockCols + 32 * w + 4 * q;
        const f32x4 lo = load4(x, col, D), hi = load4(x, col + 16, D);
        float top = 0.0f;
        bool fine = true;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            top = fmaxf(top, fmaxf(fabsf(lo[e]), fabsf(hi[e])));
            fine = fine && isfinite(lo[e]) && isfinite(hi[e]);
        }
        top = fine ? top : __builtin_inff();      // a maximum passes over a NaN
#pragma unroll
        for (int m = 1; m < G / 8; m <<= 1) top = fmaxf(top, __shfl_xor(top, m));
        const uint32_t bits = pack_bf16(top / 7.0f, 0.0f) & 0xFFFFu;
        const float scale = bf16_bits_f32(bits);
        const bool some = top >= kTiny && top < __builtin_inff();
        uint32_t codes = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int cl = some ? (int)rintf(lo[e] / scale) : 0, ch = some ? (int)rintf(hi[e] / scale) : 0;
            codes |= (uint32_t)((cl & 15) | (ch & 15) << 4) << (8 * e);
        }
        uint8_t* out = a.Q + (row0 + r) * a.ldq + s * kBlockBytes + 16 * q + 4 * w;
        *reinterpret_cast<uint32_t*>(out) = codes;
        const int g = (s * kBlockCols + 32 * w) / G;
        if (lane % (G / 8) == 0 && g < p.groups)
            a.gscale[(row0 + r) * a.ldg + g] = (uint16_t)(some ? bits : top < kTiny ? 0u : 0x7FC0u);
    }
}

struct RowsParams {
    Rows4Args a;
    int nblk;
    uint32_t magic;
    int rows_per_block;
};

// Rows of the table, or those of given tokens: the exact product of a code (4 bits)
// and its scale (8), rounded once.  A token outside the table has NaN.
template <typename T, int G>
__global__ __launch_bounds__(kRowThreads) void ember_rows_q4(RowsParams p) {
    const Rows4Args& a = p.a;
    const int lane = threadIdx.x % kUnitLanes, w = lane / 4, q = lane % 4;
    const int64_t row0 = (int64_t)blockIdx.x * p.rows_per_block;
    const int rows = (int)min((int64_t)p.rows_per_block, a.n - row0);
    const int units = rows * p.nblk, D = (int)a.D;
    for (int u = threadIdx.x / kUnitLanes; u < units; u += kUnitsPerPass) {
        const int r = (int)div_small(u, p.magic), s = u - r * p.nblk;
        const int64_t v = a.tok ? a.tok[row0 + r] : row0 + r;
        const bool in = v >= 0 && v < a.V;
        const int col = s * kBlockCols + 32 * w + 4 * q;
        uint32_t codes = 0;
        float scale = __uint_as_float(0x7FC00000u);
        if (in && col < D) {
            codes = *reinterpret_cast<const uint32_t*>(a.Wq + v * a.ldw + s * kBlockBytes + 16 * q + 4 * w);
            scale = bf16_bits_f32(a.wscale[v * a.ldg + (s * kBlockCols + 32 * w) / G]);
        }
        float lo[4], hi[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            lo[e] = (float)((int)(codes << (28 - 8 * e)) >> 28) * scale;
            hi[e] = (float)((int)(codes << (24 - 8 * e)) >> 28) * scale;
        }
        T* y = static_cast<T*>(a.Y) + (row0 + r) * a.ldy;
        store_values<T, 4>(y, col, D, lo);
        store_values<T, 4>(y, col + 16, D, hi);
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
template <typename T>
void launch_rows(const RowsParams& p, unsigned grid, hipStream_t s) {
    if (p.a.group == 32) ember_rows_q4<T, 32><<<grid, kRowThreads, 0, s>>>(p);
    else if (p.a.group == 64) ember_rows_q4<T, 64><<<grid, kRowThreads, 0, s>>>(p);
    else ember_rows_q4<T, 128><<<grid, kRowThreads, 0, s>>>(p);
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
    static constexpr int kWaves = kWide ? 8 : 16;
    static constexpr int kThreads = kWaves * kWave;
    static constexpr int kDepth = kWide ? 2 : 3;            // units in registers
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
template <typename C, int G, typename YT>
__global__ __launch_bounds__(C::kThreads) void ember_logits_q4_few(Few4Params p) {
    const Logits4Args& a = p.a;
    constexpr int kPer = kBlockCols / G;                    // groups a block
    constexpr int kScaleBytes = kUnit * kPer * 2;           // of a unit: 8, 16 or 32
    constexpr int kScaleWords = kScaleBytes / 4;
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
    const int per_block = C::kWaves / p.share, mate = wave % p.share, place = wave / p.share;
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
    const uint32_t off_s = (uint32_t)row * (uint32_t)a.ldg * 2;
    auto buffer = [&](const void* base, int64_t bytes) {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0,
                                                 (int)(bytes < kBufferMax ? bytes : kBufferMax), kBufferWord3);
    };
    struct Unit {
        i32x4 w[C::kLoadsW];
        uint32_t s[kScaleWords];
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
        // (16 bytes at a time where there are as many; groups past the row's are not used)
        const uint32_t off = u * kUnit * kPer < p.groups ? off_s + u * kScaleBytes : kBufferMax;
        if constexpr (kScaleBytes == 8) {
            const u32x2_t d = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_raw_buffer_load_b64(rs, off, 0, 0));
            k.s[0] = d[0];
            k.s[1] = d[1];
        } else {
#pragma unroll
            for (int q = 0; q < kScaleWords; q += 4) {
                const u32x4_t d = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rs, off + 4 * q, 0, 0));
#pragma unroll
                for (int e = 0; e < 4; ++e) k.s[q + e] = d[e];
            }
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
                scale[j] = __uint_as_float((g & 1) ? k.s[g / 2] & 0xFFFF0000u : k.s[g / 2] << 16);
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
        for (int n = threadIdx.x; n < T * cols; n += C::kThreads) {
            const int t = n / cols, c = n - t * cols, k0 = (u0 * kUnit * 8 + c) * 16;
            i32x4 x = {0, 0, 0, 0};
            if (k0 < D) {   // the padding up to 16 columns is readable
                x = *reinterpret_cast<const i32x4*>(a.Xq + (t0 + t) * a.ldx + k0);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int left = D - k0 - 4 * j;
                    x[j] &= left >= 4 ? -1 : left <= 0 ? 0 : (int)((1u << (8 * left)) - 1);
                }
            }
            const int w = c % 8 / 2, h = c % 2;
            uint8_t* at = lds + t * p.pitch + c / 8 * kBlockCols;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int to = C::kWide ? w * 32 + (j >> 1) * 16 + ((j & 1) * 2 + h) * 4
                                        : (w >> 1) * 64 + j * 16 + ((w & 1) * 2 + h) * 4;
                *reinterpret_cast<int*>(at + to) = x[j];
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
    int64_t tile0, tile1, per_xcd;
    int group_m;
};

template <int BM_, int BN_, int WM_, int WN_, int STAGES_>
struct Tile4 {
    static constexpr int BM = BM_, BN = BN_;       // tokens, channels a block
    static constexpr int WM = WM_, WN = WN_;       // wavefronts over them
    static constexpr int kStages = STAGES_;
    static constexpr int kWavesB = WM * WN;
    static constexpr int kThreads = kWavesB * kWave;
    static constexpr int MT = BM / WM / 32, NT = BN / WN / 32;   // MFMA tiles a wave
    static constexpr int kX = BM * kBlockCols, kW = BN * kBlockBytes, kS = BN * 16;   // bytes of a stage
    static constexpr int kLoadsX = BM / 8 / kWavesB, kLoadsW = BN / 16 / kWavesB;     // a wave and step
    static constexpr int kLoads = kLoadsX + kLoadsW + 1;
    static constexpr int kStageBytes = kX + kW + kS;
    static constexpr int kLds = kStages * kStageBytes;
    static_assert(BM % (8 * kWavesB) == 0 && BN % (16 * kWavesB) == 0 && kWavesB % 2 == 0, "equal loads a wave");
    static_assert(BM <= kThreads, "a thread a token's row");
    static_assert(BN % 64 == 0 && kWavesB % (BN / 64) == 0, "loads of the scales");
    static_assert(kStages >= 2 && (kStages - 2) * kLoads < 64, "vmcnt range");
    static_assert((int64_t)std::max(BM, BN) * EMBER_Q8_MAX_LD < (int64_t)1 << 31, "32-bit load offsets");
    static_assert(kLds <= 160 * 1024, "LDS of one CU");
};

// BM tokens x BN channels a block, a block of 128 columns a step.  A ring of LDS
// stages holds the tokens' codes, the table's, and 16 bytes of scales a channel
// (eight groups, among them the step's).
template <typename C, int G, typename YT>
__global__ __launch_bounds__(C::kThreads) void ember_logits_q4(Tile4Params p) {
    __shared__ __attribute__((aligned(1024))) uint8_t lds[C::kLds];
    const Logits4Args& a = p.a;
    constexpr int kPer = kBlockCols / G;
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int wm = wave % C::WM, wn = wave / C::WM;
    const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
    const int64_t l = p.tile0 + (int64_t)(blockIdx.x % kXcds) * p.per_xcd + blockIdx.x / kXcds;
    if (l >= min(p.tile0 + (int64_t)(blockIdx.x % kXcds + 1) * p.per_xcd, p.tile1)) return;
    int tm;
    int64_t tn;
    tile_at(p.MT, p.NT, p.group_m, l, tm, tn);
    const int64_t t0 = (int64_t)tm * C::BM, v0 = tn * C::BN;
    const int D = (int)a.D;

    const int row_x = wave * 8 + lane / 8, row_w = wave * 16 + lane / 4;
    const int k_x = ((lane % 8) ^ swizzle<8>(row_x)) * 16, k_w = ((lane % 4) ^ swizzle<4>(row_w)) * 16;
    const int row_s = wave % (C::BN / 64) * 64 + lane;
    const uint32_t off_x = row_x * (uint32_t)a.ldx + k_x, off_w = row_w * (uint32_t)a.ldw + k_w;
    const uint32_t off_s = row_s * (uint32_t)(2 * a.ldg);
    auto issue = [&](int kt, uint32_t st) {
        const bool in = kt < p.nk;
        const int64_t kx = in ? (int64_t)kt * kBlockCols : 0, kw = in ? (int64_t)kt * kBlockBytes : 0;
        const int64_t ks = in ? (int64_t)kt * kPer / 8 * 8 : 0;
        const i32x4 rx = rsrc(a.Xq + t0 * a.ldx + kx, in ? (a.T - t0) * a.ldx - kx : 0);
        const i32x4 rw = rsrc(a.Wq + v0 * a.ldw + kw, in ? (a.V - v0) * a.ldw - kw : 0);
        const i32x4 rs = rsrc(a.wscale + v0 * a.ldg + ks, in ? ((a.V - v0) * a.ldg - ks) * 2 : 0);
        const uint32_t ox = k_x < D - (int)kx ? off_x : kBufferMax;
#pragma unroll
        for (int j = 0; j < C::kLoadsX; ++j)
            load_to_lds(rx, st + (wave + C::kWavesB * j) * 1024, ox + j * (C::kWavesB * 8 * (uint32_t)a.ldx));
#pragma unroll
        for (int j = 0; j < C::kLoadsW; ++j)
            load_to_lds(rw, st + C::kX + (wave + C::kWavesB * j) * 1024, off_w + j * (C::kWavesB * 16 * (uint32_t)a.ldw));
        load_to_lds(rs, st + C::kX + C::kW + wave % (C::BN / 64) * 1024, off_s);
    };
    const int half = lane >> 5, sh = half ? 0 : 4;
    const int rx0 = wm * (C::MT * 32) + (lane & 31), rw0 = wn * (C::NT * 32) + (lane & 31);
    auto lds_at = [](uint32_t at) { return *(const __attribute__((address_space(3))) i32x4*)(uintptr_t)at; };

    f32x16 f[C::MT][C::NT];
#pragma unroll
    for (int m = 0; m < C::MT; ++m)
#pragma unroll
        for (int n = 0; n < C::NT; ++n)
#pragma unroll
            for (int e = 0; e < 16; ++e) f[m][n][e] = 0.0f;

#pragma unroll
    for (int q = 0; q < C::kStages - 1; ++q) issue(q, lds_base + q * C::kStageBytes);
    uint32_t st = lds_base, fill = lds_base + (C::kStages - 1) * C::kStageBytes;
    for (int i = 0; i < p.nk; ++i) {
        // this wave's loads of step i have landed (those of later steps may be out), and past
        // the barrier everyone's have, and no one reads the stage of step i - 1 any more
        wait_step<(C::kStages - 2) * C::kLoads>();
        issue(i + C::kStages - 1, fill);
        if (D % 16 != 0 && i == p.nk - 1) {
            // the last chunk of a token's row holds columns that do not count
            const int c = D % kBlockCols / 16, r = threadIdx.x;
            if (r < C::BM) {
                auto* const x = (__attribute__((address_space(3))) i32x4*)(uintptr_t)(st + r * kBlockCols + (c ^ swizzle<8>(r)) * 16);
                i32x4 y = *x;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int b = D % 16 - 4 * e;
                    y[e] &= b >= 4 ? -1 : b <= 0 ? 0 : (int)((1u << (8 * b)) - 1);
                }
                *x = y;
            }
            wait_step<63>();
        }
        i32x4 wd[C::NT][4];
        float scale[C::NT][kPer];
#pragma unroll
        for (int n = 0; n < C::NT; ++n) {
            const int r = rw0 + 32 * n;
#pragma unroll
            for (int t = 0; t < 4; ++t) wd[n][t] = lds_at(st + C::kX + r * kBlockBytes + ((t ^ swizzle<4>(r)) * 16));
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                const uint32_t at = st + C::kX + C::kW + r * 16 + (i * kPer + j) % 8 * 2;
                const uint32_t h = *(const __attribute__((address_space(3))) uint16_t*)(uintptr_t)at;
                // no group: what stands in its place is not a scale
                scale[n][j] = kPer == 1 || i * kPer + j < p.groups ? bf16_bits_f32(h) : 0.0f;
            }
        }
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
#pragma unroll
            for (int m = 0; m < C::MT; ++m) {
                i32x16 sum[C::NT];
#pragma unroll
                for (int g = 0; g < 4 / kPer; ++g) {
                    const int w = j * (4 / kPer) + g;
                    const int r = rx0 + 32 * m;
                    const i32x4 x = lds_at(st + r * kBlockCols + (((2 * w + half) ^ swizzle<8>(r)) * 16));
#pragma unroll
                    for (int n = 0; n < C::NT; ++n) {
                        i32x4 op;
#pragma unroll
                        for (int t = 0; t < 4; ++t) op[t] = (int)(((uint32_t)wd[n][t][w] << sh) & 0xF0F0F0F0u);
                        i32x16 zero;
#pragma unroll
                        for (int e = 0; e < 16; ++e) zero[e] = 0;
                        sum[n] = __builtin_amdgcn_mfma_i32_32x32x32_i8(x, op, g == 0 ? zero : sum[n], 0, 0, 0);
                    }
                }
#pragma unroll
                for (int n = 0; n < C::NT; ++n)
#pragma unroll
                    for (int e = 0; e < 16; ++e) f[m][n][e] += (float)sum[n][e] * scale[n][j];
            }
        }
        st = st + C::kStageBytes == lds_base + C::kLds ? lds_base : st + C::kStageBytes;
        fill = fill + C::kStageBytes == lds_base + C::kLds ? lds_base : fill + C::kStageBytes;
    }
    wait_step<0>();    // the zero-filling loads past the end have landed

    // a lane holds 16 tokens of a channel
#pragma unroll
    for (int n = 0; n < C::NT; ++n) {
        const int64_t v = v0 + rw0 + 32 * n;
        if (v >= a.V) continue;
        const float bias = a.bias ? a.bias[v] : 0.0f;
#pragma unroll
        for (int m = 0; m < C::MT; ++m) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int64_t t = t0 + (wm * C::MT + m) * 32 + 8 * (e / 4) + 4 * half + e % 4;
                if (t >= a.T) continue;
                const float y = f[m][n][e] * (a.xscale[t] * 0.0625f) + bias;
                if constexpr (sizeof(YT) == 4) static_cast<float*>(a.Y)[t * a.ldy + v] = y;
                else static_cast<uint16_t*>(a.Y)[t * a.ldy + v] = (uint16_t)pack_bf16(y, 0.0f);
            }
        }
    }
}

// Bytes of a token's units in LDS.  They end 16 bytes past a multiple of the banks: the
// lanes of a part read different ones.
int64_t few_pitch(int64_t units) { return (units * kUnit * kBlockCols + 255) / 256 * 256 + 16; }
static_assert(16 * (4 * 3 * kUnit * kBlockCols + 16) <= kFewLds, "16 tokens: a window for four waves, three units deep");

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
    const int64_t per_block = C::kWaves / p.share;
    p.together = p.strips >= 4 * kCus ? 4 : 1;
    const int64_t all = p.several ? (p.strips + p.together - 1) / p.together : (p.strips + per_block - 1) / per_block;
    p.blocks = (int)(p.several ? std::min<int64_t>(all, std::max(1, kCus / p.tiles)) : all);
    const dim3 grid((unsigned)((p.blocks + kXcds - 1) / kXcds * kXcds * p.tiles));
    if (a.y_dtype == EMBER_F32) ember_logits_q4_few<C, G, float><<<grid, C::kThreads, 0, s>>>(p);
    else ember_logits_q4_few<C, G, uint16_t><<<grid, C::kThreads, 0, s>>>(p);
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
    const int64_t total = (int64_t)p.MT * p.NT;
    for (int64_t t0 = 0; t0 < total; t0 += kMaxGridBlocks) {
        p.tile0 = t0;
        p.tile1 = std::min(t0 + kMaxGridBlocks, total);
        p.per_xcd = (p.tile1 - t0 + kXcds - 1) / kXcds;
        const unsigned grid = (unsigned)(p.per_xcd * kXcds);
        if (a.y_dtype == EMBER_F32) launch_tile<C, G, float>(p, grid, s);
        else launch_tile<C, G, uint16_t>(p, grid, s);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

using T128x128 = Tile4<128, 128, 4, 2, 3>;
using T256x256 = Tile4<256, 256, 2, 4, 3>;

template <int G>
hipError_t launch_group(const Logits4Args& a, hipStream_t s) {
    if (a.T <= 64) {
        const int64_t pitch = few_pitch((a.D + 511) / 512);
        if (a.T <= 16 || a.V < 16384 || 32 * pitch > kFewLds) return launch_few<Stream<false, 1>, G>(a, s);
        if (a.T <= 32 || 64 * pitch > kFewLds) return launch_few<Stream<true, 1>, G>(a, s);
        return launch_few<Stream<true, 2>, G>(a, s);
    }
    if (a.T <= 512 || a.V <= 16384) return launch_tiles<T128x128, G>(a, s);
    return launch_tiles<T256x256, G>(a, s);
}

} // namespace

hipError_t launch_quantize4(const Quant4Args& a, hipStream_t s) {
    QuantParams p;
    p.a = a;
    p.nblk = (int)((a.D + kBlockCols - 1) / kBlockCols);
    p.groups = (int)((a.D + a.group - 1) / a.group);
    p.magic = magic_of(p.nblk);
    p.rows_per_block = rows_per_block(p.nblk);
    const unsigned grid = (unsigned)((a.rows + p.rows_per_block - 1) / p.rows_per_block);
    if (a.x_dtype == EMBER_F32) launch_quantize<float>(p, grid, s);
    else launch_quantize<uint16_t>(p, grid, s);
    return hipGetLastError();
}

hipError_t launch_rows4(const Rows4Args& a, hipStream_t s) {
    RowsParams p;
    p.a = a;
    p.nblk = (int)((a.D + kBlockCols - 1) / kBlockCols);
    p.magic = magic_of(p.nblk);
    p.rows_per_block = rows_per_block(p.nblk);
    const unsigned grid = (unsigned)((a.n + p.rows_per_block - 1) / p.rows_per_block);
    if (a.y_dtype == EMBER_F32) launch_rows<float>(p, grid, s);
    else launch_rows<uint16_t>(p, grid, s);
    return hipGetLastError();
}

hipError_t launch_logits4(const Logits4Args& a, hipStream_t s) {
    if (a.group == 32) return launch_group<32>(a, s);
    if (a.group == 64) return launch_group<64>(a, s);
    return launch_group<128>(a, s);
}

} // namespace ember
