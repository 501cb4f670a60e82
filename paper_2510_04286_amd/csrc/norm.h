// Norm of the residual stream (norm.hip): launchers, and the conversion to e4m3 that the 8-bit operators share.
#pragma once
#include "common.h"

namespace slicemoe {

constexpr float kE4m3Max = 448.f;      // largest e4m3 value
constexpr float kE4m3Floor = 1e-30f;   // a group whose largest value is below this is scaled as if it were this

// Four values as e4m3, rounded to nearest even; beyond +-448 (a quotient by the scale may round up past it) the largest value, NaN stays NaN.
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d)
{
    const auto clamp = [](float v) { return v > kE4m3Max ? kE4m3Max : v < -kE4m3Max ? -kE4m3Max : v; };
    int p = __builtin_amdgcn_cvt_pk_fp8_f32(clamp(a), clamp(b), 0, false);
    p = __builtin_amdgcn_cvt_pk_fp8_f32(clamp(c), clamp(d), p, true);
    return (uint32_t)p;
}

constexpr int kNormMaxWidth = 16384;        // what sixteen wavefronts hold of an fp32 row (four of a bf16 one)
constexpr int kNormBackwardBlocks = 768;    // persistent blocks of the backward pass at most, three per CU (its registers): rows of partial weight gradients
int norm_backward_blocks(const slicemoe_norm_config &c);
hipError_t launch_add_rmsnorm(const slicemoe_norm_config &c, const void *x, const void *residual, const void *weight, void *sum, void *y,
                              uint8_t *yq, float *yscale, hipStream_t s);
hipError_t launch_add_rmsnorm_backward(const slicemoe_norm_config &c, const void *sum, const void *weight, const void *dy,
                                       const void *dsum, void *dx, float *dw, float *part, hipStream_t s);

}  // namespace slicemoe
