// Logits of an LM head held in 8 bits (gfx950):
//   Y_tv = (sum_k Xq_tk Wq_vk) xscale_t wscale_v + bias_v,
// with int8 matrix instructions.  The sum is exact in int32 (D is limited to
// EMBER_Q8_MAX_D), so neither tiling nor order changes a bit of it; it is rounded
// to fp32 once, scaled and rounded to the type of Y.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ember_device.h"
#include "ember_launch.h"

namespace ember {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

constexpr int kTile = 64;   // tokens and channels a block
constexpr int kStep = 64;   // columns a step

// 16 columns [k, k + 16) of a row: zeros past the row's D columns.
__device__ __forceinline__ i32x4 load16(const int8_t* row, int k, int D, bool valid) {
    i32x4 w = {0, 0, 0, 0};
    if (!valid) return w;
    if (k + 16 <= D) return *reinterpret_cast<const i32x4*>(row + k);
    for (int e = 0; e < 16; ++e)
        if (k + e < D) w[e >> 2] |= (int)(uint8_t)row[k + e] << (8 * (e & 3));
    return w;
}

__global__ __launch_bounds__(kBlock) void ember_logits_tile(LogitsArgs a) {
    __shared__ __attribute__((aligned(16))) int8_t lx[kTile][kStep + 16], lw[kTile][kStep + 16];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int64_t t0 = (int64_t)blockIdx.y * kTile, v0 = (int64_t)blockIdx.x * kTile;
    const int row = threadIdx.x / 4, chunk = threadIdx.x % 4;
    const int wt = (wave & 1) * 32, wv = (wave >> 1) * 32;
    i32x16 acc = {};
    const int D = (int)a.D;
    for (int k = 0; k < D; k += kStep) {
        const i32x4 x = load16(a.Xq + (t0 + row) * a.ldx, k + 16 * chunk, D, t0 + row < a.T);
        const i32x4 w = load16(a.Wq + (v0 + row) * a.ldw, k + 16 * chunk, D, v0 + row < a.V);
        __syncthreads();
        *reinterpret_cast<i32x4*>(&lx[row][16 * chunk]) = x;
        *reinterpret_cast<i32x4*>(&lw[row][16 * chunk]) = w;
        __syncthreads();
#pragma unroll
        for (int kk = 0; kk < kStep; kk += 32) {
            const i32x4 fa = *reinterpret_cast<const i32x4*>(&lx[wt + (lane & 31)][kk + 16 * (lane >> 5)]);
            const i32x4 fb = *reinterpret_cast<const i32x4*>(&lw[wv + (lane & 31)][kk + 16 * (lane >> 5)]);
            acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(fa, fb, acc, 0, 0, 0);
        }
    }
    const int64_t v = v0 + wv + (lane & 31);
    if (v >= a.V) return;
    const float ws = a.wscale[v], bias = a.bias ? a.bias[v] : 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int64_t t = t0 + wt + 8 * (i >> 2) + 4 * (lane >> 5) + (i & 3);
        if (t >= a.T) continue;
        const float y = (float)acc[i] * (a.xscale[t] * ws) + bias;
        if (a.y_dtype == EMBER_F32) static_cast<float*>(a.Y)[t * a.ldy + v] = y;
        else static_cast<uint16_t*>(a.Y)[t * a.ldy + v] = (uint16_t)pack_bf16(y, 0.0f);
    }
}

} // namespace

hipError_t launch_logits(const LogitsArgs& a, hipStream_t s) {
    const dim3 grid((unsigned)((a.V + kTile - 1) / kTile), (unsigned)((a.T + kTile - 1) / kTile));
    ember_logits_tile<<<grid, kBlock, 0, s>>>(a);
    return hipGetLastError();
}

} // namespace ember
