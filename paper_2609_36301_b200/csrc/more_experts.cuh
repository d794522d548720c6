// What the kernels of the experts' feed-forward blocks share (more_experts_sm100.cu, more_experts_pairs.cu): parameters and the
// activation.  Internal.
#pragma once

#include "sm100_common.cuh"

#include <cuda_fp16.h>

namespace more {

struct ExpertsArgs {
    const __nv_bfloat16* X;       // [T][h]
    const __nv_bfloat16* W1;      // [M][h][2s]
    const __nv_bfloat16* W2;      // [M][s][h]
    const int32_t* idx;           // [T][k]
    const int32_t* offsets;       // [M + 1]
    const int32_t* pairs;         // [T k]
    int T, h, s, M, k;
    // forward
    __nv_bfloat16* out_y;         // [T k][h]
    __nv_bfloat16* out_hidden;    // [T k][2s], nullable
    // backward
    const float* gate;            // [T][k]
    const __nv_bfloat16* hidden;  // [T k][2s]
    const __nv_bfloat16* dout;    // [T][h]
    __nv_bfloat16* out_dx;        // [T][h], nullable
    float* out_dgate;             // [T][k], nullable
    __nv_bfloat16* out_dw1;       // [M][h][2s], nullable
    __nv_bfloat16* out_dw2;       // [M][s][h], nullable
    void* workspace;
    cudaStream_t stream;
};

// Forward for few pairs: a cluster of CTAs per pair, no workspace.
int launch_experts_pairs(const ExpertsArgs& a, const DeviceCtx& ctx);

namespace {

// sigmoid(x) in fp32; e^-x overflows to infinity for x < -88, where the quotient is 0 as it should be.  Good to five units of 2^-23 at every x:
// it feeds the gate gradients, which leave in 32 bits.
__device__ __forceinline__ float sigmoidf(float x) { return __fdividef(1.f, 1.f + expf(-x)); }
// The same with an exponential whose error grows with x (30 units of 2^-23 at -25, 10^-5 at -80), far below the rounding to bf16 that what
// is computed from it in the forward pass ends in; sigmoidf there costs 3 % with few wide experts (324 us for 314, 32768 x 8 pairs of 256).
__device__ __forceinline__ float sigmoid_to_round(float x) { return __fdividef(1.f, 1.f + __expf(-x)); }

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float bf16_lo(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }

}  // namespace

}  // namespace more
