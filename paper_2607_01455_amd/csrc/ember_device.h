// Element access and reductions shared by the norm, 8-bit and clipping kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ember_launch.h"

namespace ember {

typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float bf16_bits_f32(uint32_t h) { return __uint_as_float(h << 16); }

// Two fp32 -> bf16 (low, high half), round to nearest even: one v_cvt_pk_bf16_f32.
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const f32x2 f = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
}

template <typename T> constexpr int kChunkElems = 16 / (int)sizeof(T);   // elements of a 16-byte chunk

// Element e of a 16-byte chunk of T (float, or uint16_t for bf16).
template <typename T>
__device__ __forceinline__ float elem(const u32x4_t& w, int e) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
    else return (e & 1) ? __uint_as_float(w[e >> 1] & 0xFFFF0000u) : __uint_as_float(w[e >> 1] << 16);
}

__device__ __forceinline__ float load_elem(const void* p, int64_t i, bool bf16) {
    return bf16 ? bf16_bits_f32(static_cast<const uint16_t*>(p)[i]) : static_cast<const float*>(p)[i];
}

// The chunk at columns [col, col + chunk) of a row of D elements: one 16-byte
// load where it lies inside the row, and in the row's last partial chunk too if
// another row follows (what is loaded past the row is then its padding, see
// kept_words); element loads there in the last row; zeros past it.
template <typename T>
__device__ __forceinline__ u32x4_t load_chunk(const T* row, int col, int D, bool follows) {
    u32x4_t w = {0, 0, 0, 0};
    if (col + kChunkElems<T> <= D || (follows && col < D)) {
        w = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(row + col));
    } else {
#pragma unroll
        for (int e = 0; e < kChunkElems<T>; ++e) {
            if (col + e < D) {
                if constexpr (sizeof(T) == 4) w[e] = reinterpret_cast<const uint32_t*>(row)[col + e];
                else w[e >> 1] |= (uint32_t)reinterpret_cast<const uint16_t*>(row)[col + e] << (16 * (e & 1));
            }
        }
    }
    return w;
}

// The bits of a chunk from load_chunk that belong to its row.
template <typename T>
__device__ __forceinline__ u32x4_t kept_words(int col, int D) {
    constexpr int kPer = 4 / (int)sizeof(T);   // elements a word
    u32x4_t w;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int n = D - col - q * kPer;
        w[q] = n >= kPer ? 0xFFFFFFFFu : kPer == 2 && n == 1 ? 0xFFFFu : 0u;
    }
    return w;
}

template <bool kNT, typename V>
__device__ __forceinline__ void store_vec(void* p, V v) {
    if constexpr (kNT) __builtin_nontemporal_store(v, static_cast<V*>(p));
    else *static_cast<V*>(p) = v;
}

// N fp32 values into columns [col, col + N) of a row of T, rounded to nearest
// even for bf16: vector stores where they lie inside the row (col * sizeof(T) a
// multiple of the vector's size; kNT: non-temporal), element stores in its last
// partial chunk.
template <typename T, int N, bool kNT = false>
__device__ __forceinline__ void store_values(T* row, int col, int D, const float (&v)[N]) {
    constexpr int kWords = N * (int)sizeof(T) / 4;
    uint32_t w[kWords];
#pragma unroll
    for (int q = 0; q < kWords; ++q) {
        if constexpr (sizeof(T) == 4) w[q] = __float_as_uint(v[q]);
        else w[q] = pack_bf16(v[2 * q], v[2 * q + 1]);
    }
    if (col + N <= D) {
        if constexpr (kWords == 2) {
            store_vec<kNT>(row + col, u32x2_t{w[0], w[1]});
        } else {
#pragma unroll
            for (int q = 0; q < kWords; q += 4)
                store_vec<kNT>(reinterpret_cast<uint32_t*>(row + col) + q, u32x4_t{w[q], w[q + 1], w[q + 2], w[q + 3]});
        }
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            if (col + e < D) {
                if constexpr (sizeof(T) == 4) reinterpret_cast<uint32_t*>(row)[col + e] = w[e];
                else reinterpret_cast<uint16_t*>(row)[col + e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
            }
        }
    }
}

// Sum and maximum over the TPR threads that share a row, the same in all of
// them and in an order fixed by TPR: within a wave by exchanges, then over the
// waves in wave order through LDS (red: one slot a wave; the caller's next use
// of the same slots has to come after another barrier).
template <typename V, typename Op>
__device__ __forceinline__ V wave_all(V x, Op op) {
#pragma unroll
    for (int m = 1; m < kWave; m <<= 1) x = op(x, __shfl_xor(x, m));
    return x;
}
template <int TPR, typename V, typename Op>
__device__ __forceinline__ V row_all(V x, Op op, V* red) {
    x = wave_all(x, op);
    if constexpr (TPR > kWave) {
        const int wave = threadIdx.x / kWave;
        if ((threadIdx.x & (kWave - 1)) == 0) red[wave] = x;
        __syncthreads();
        x = red[0];
#pragma unroll
        for (int w = 1; w < TPR / kWave; ++w) x = op(x, red[w]);
    }
    return x;
}

} // namespace ember
