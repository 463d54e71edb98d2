// Launchers of the norm, the 8-bit and 4-bit tables, sampling and the clipping, for ember_api.cpp:
// arguments checked, all work enqueued on s.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "ember.h"

namespace ember {

// Norm with the residual's addition and its gradient, and rows to 8 bits
// (ember_norm.hip; gain null: no norm).
struct NormArgs {
    const void* X;
    int x_dtype;
    int64_t ldx;
    const void* R;
    int64_t ldr;
    const void* gain;
    int gain_dtype;
    float eps;
    int64_t T;
    int64_t D;
    void* S;
    int64_t lds;
    void* Y;
    int y_dtype;
    int64_t ldy;
    int8_t* Q;
    int64_t ldq;
    float* qscale;
    float* rstd;
};
hipError_t launch_rmsnorm(const NormArgs& a, hipStream_t s);
struct NormGradArgs {
    const void* dY;
    int64_t lddy;
    const void* S;
    int x_dtype;      // of dY, S, dS and dX
    int64_t lds;
    const void* gain;
    int gain_dtype;
    const float* rstd;
    const void* dS;
    int64_t ldds;
    int64_t T;
    int64_t D;
    void* dX;
    int64_t lddx;
    float* dgain;
    char* ws;
};
size_t norm_grad_ws_bytes(int64_t T, int64_t D);
hipError_t launch_rmsnorm_grad(const NormGradArgs& a, hipStream_t s);

// 8-bit logits (ember_q8.hip).
struct LogitsArgs {
    const int8_t* Xq;
    int64_t ldx;
    const float* xscale;
    const int8_t* Wq;
    int64_t ldw;
    const float* wscale;
    const float* bias;
    int64_t T;
    int64_t V;
    int64_t D;
    void* Y;
    int y_dtype;
    int64_t ldy;
};
hipError_t launch_logits(const LogitsArgs& a, hipStream_t s);

// Tables in 4 bits: rows to them and back, logits (ember_q4.hip).  Scales: bf16 bits.
struct Quant4Args {
    const void* X;
    int x_dtype;
    int64_t ldx;
    int64_t rows;
    int64_t D;
    int group;
    uint8_t* Q;
    int64_t ldq;      // bytes
    uint16_t* gscale;
    int64_t ldg;      // scales
};
hipError_t launch_quantize4(const Quant4Args& a, hipStream_t s);
struct Rows4Args {
    const uint8_t* Wq;
    int64_t ldw;
    const uint16_t* wscale;
    int64_t ldg;
    int group;
    int64_t V;
    int64_t D;
    const int64_t* tok;
    int64_t n;
    void* Y;
    int y_dtype;
    int64_t ldy;
};
hipError_t launch_rows4(const Rows4Args& a, hipStream_t s);
struct Logits4Args {
    const int8_t* Xq;
    int64_t ldx;
    const float* xscale;
    const uint8_t* Wq;
    int64_t ldw;
    const uint16_t* wscale;
    int64_t ldg;
    int group;
    const float* bias;
    int64_t T;
    int64_t V;
    int64_t D;
    void* Y;
    int y_dtype;
    int64_t ldy;
};
hipError_t launch_logits4(const Logits4Args& a, hipStream_t s);

// A token a row of logits (ember_sample.hip).
struct SampleArgs {
    const void* L;
    int l_dtype;
    int64_t ldl;
    int64_t T;
    int64_t V;
    const float* temperature;
    const int* top_k;
    const float* top_p;
    const float* min_p;
    const float* u;
    int64_t* ids;
    float* logp;
    int* kept;
    char* ws;
};
size_t sample_ws_bytes(int64_t T, int64_t V);
hipError_t launch_sample(const SampleArgs& a, hipStream_t s);

// Global gradient norm and clipping (ember_clip.hip).
size_t clip_ws_bytes(int64_t n);
hipError_t launch_clip(const ember_grad* g, int64_t n, float max_norm, float* out, char* ws, hipStream_t s);

} // namespace ember
