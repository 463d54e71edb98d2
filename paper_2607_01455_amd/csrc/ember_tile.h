// Loads into LDS, barriers and orders that the 8-bit and 4-bit logits kernels share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ember_launch.h"

namespace ember {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

constexpr int kXcds = 8;
constexpr int kCus = 256;
constexpr int kBufferWord3 = 0x00020000;   // raw 32-bit data format, gfx9 family
// Bytes of a buffer at most; an offset past every buffer, also with what is added to it
// (unsigned: below 2^30 + 2^12).
constexpr uint32_t kBufferMax = 0x7FFFFFF0;

// Raw buffer resource of `bytes` bytes at a wave-uniform base.
__device__ __forceinline__ i32x4 rsrc(const void* base, int64_t bytes) {
    const uint64_t p = reinterpret_cast<uint64_t>(base);
    i32x4 r;
    r.x = __builtin_amdgcn_readfirstlane((int)p);
    r.y = __builtin_amdgcn_readfirstlane((int)(p >> 32) & 0xFFFF);
    r.z = __builtin_amdgcn_readfirstlane(bytes > kBufferMax ? (int)kBufferMax : bytes < 0 ? 0 : (int)bytes);
    r.w = kBufferWord3;
    return r;
}

// 16 bytes per lane from a buffer into LDS at lds_base + 16 lane; lanes outside
// the buffer's range write zeros.  Inline assembly, so that the compiler does
// not make every later LDS read wait for it; completion is awaited with
// wait_step before a stage is read.  M0 holds the (wave-uniform) LDS base.
__device__ __forceinline__ void load_to_lds(i32x4 rs, uint32_t lds_base, uint32_t voffset) {
    const uint32_t base = __builtin_amdgcn_readfirstlane(lds_base);
    uint32_t saved;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"
                 "buffer_load_dwordx4 %2, %3, 0 offen lds\n\ts_mov_b32 m0, %0"
                 : "=&s"(saved)
                 : "s"(base), "v"(voffset), "s"(rs)
                 : "memory");
}

// The step barrier: at most N of this wave's vector-memory loads outstanding and
// all of its LDS reads returned, then the block's waves meet.
template <int N>
__device__ __forceinline__ void wait_step() {
    static_assert(N >= 0 && N < 64, "vmcnt range");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4));
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Orders a wave's LDS accesses before and after it (they execute in order, so
// only the compiler has to be held).
__device__ __forceinline__ void wave_lds_order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Chunk c of a slice's row r sits at position c ^ swizzle(r): the reads of the
// same chunk of 8 (or 16) consecutive rows then cover 32 (or all 64) LDS banks
// once, and a wave-wide load still fills whole rows.
template <int kChunks>
__device__ __forceinline__ int swizzle(int r) {
    return kChunks == 16 ? r & 15 : ((kChunks == 8 ? r & 7 : (r >> 1) & 3) ^ ((r >> 3) & 1));
}

// Tile l of MT x NT -> (token tile, channel tile): groups of group_m token tiles,
// token tile fastest inside a group.
__device__ __forceinline__ void tile_at(int MT, int64_t NT, int group_m, int64_t l, int& tm, int64_t& tn) {
    const int64_t per_group = (int64_t)group_m * NT;
    const int64_t g = l / per_group;
    const int first = (int)(g * group_m);
    const int gm = min(MT - first, group_m);
    const int64_t q = l - g * per_group;
    tm = first + (int)(q % gm);
    tn = q / gm;
}

} // namespace ember
