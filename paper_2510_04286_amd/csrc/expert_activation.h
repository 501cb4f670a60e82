// The experts' activation on the matrix-core path, on packed fp16 pairs (described in ffn_mfma.hip), and what else its kernels share.
#pragma once
#include "mfma.h"

namespace slicemoe {

typedef _Float16 half_t;
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// Packed fp16 constants of the activation stage, passed by value (uniform: they live in SGPRs).
struct EpiConst {
    uint32_t neg_w0;
    uint32_t q[kGeluM + 1];
    uint32_t half;
};

static uint32_t pack2_f16(float f)
{
    const _Float16 h = (_Float16)f;
    uint16_t u;
    __builtin_memcpy(&u, &h, 2);
    return (uint32_t)u | ((uint32_t)u << 16);
}

static EpiConst make_epi_const()
{
    EpiConst K;
    K.neg_w0 = pack2_f16(-kGeluW0);
    for (int i = 0; i <= kGeluM; ++i) K.q[i] = pack2_f16(kGeluQ[i]);
    K.half = pack2_f16(0.5f);
    return K;
}

__device__ __forceinline__ h2 as_h2(uint32_t u) { return __builtin_bit_cast(h2, u); }
__device__ __forceinline__ h2 pk_fma(h2 a, h2 b, h2 c) { return __builtin_elementwise_fma(a, b, c); }
// fused multiply-add with the instruction's output clamp to [0, 1]
__device__ __forceinline__ h2 pk_fma_clamp01(h2 a, h2 b, h2 c)
{
    h2 d;
    asm("v_pk_fma_f16 %0, %1, %2, %3 clamp" : "=v"(d) : "v"(a), "v"(b), "v"(c));
    return d;
}

// Two accumulators -> a packed fp16 pair of kappa * GELU(z): what activation_tile does eight times.
__device__ __forceinline__ uint32_t activation_pair(float a0, float a1, h2 p2, h2 bias, const EpiConst &K)
{
    const h2 s = pk_fma(__builtin_bit_cast(h2, __builtin_amdgcn_cvt_pkrtz(a0, a1)), p2, bias);
    const h2 v = pk_fma(s, s, as_h2(K.neg_w0));
    h2 Q = pk_fma(v, as_h2(K.q[kGeluM]), as_h2(K.q[kGeluM - 1]));
#pragma unroll
    for (int c = kGeluM - 2; c >= 0; --c) Q = pk_fma(Q, v, as_h2(K.q[c]));
    const h2 F = pk_fma_clamp01(s, Q, as_h2(K.half));
    return __builtin_bit_cast(uint32_t, s * F);
}

// 16 accumulators of one 32x32 tile -> 8 packed fp16 pairs of kappa * GELU(z); pair i holds the
// accumulator registers 2i and 2i+1, i.e. contraction slots of GEMM2 in register order.
__device__ __forceinline__ void activation_tile(const f32x16 &acc, h2 p2, const h2 (&bias)[8], const EpiConst &K, uint4 (&out)[2])
{
    uint32_t o[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const h2 A = __builtin_bit_cast(h2, __builtin_amdgcn_cvt_pkrtz(acc[2 * i], acc[2 * i + 1]));
        const h2 s = pk_fma(A, p2, bias[i]);
        const h2 v = pk_fma(s, s, as_h2(K.neg_w0));
        h2 Q = pk_fma(v, as_h2(K.q[kGeluM]), as_h2(K.q[kGeluM - 1]));
#pragma unroll
        for (int c = kGeluM - 2; c >= 0; --c) Q = pk_fma(Q, v, as_h2(K.q[c]));
        const h2 F = pk_fma_clamp01(s, Q, as_h2(K.half));
        o[i] = __builtin_bit_cast(uint32_t, s * F);
    }
    out[0] = make_uint4(o[0], o[1], o[2], o[3]);
    out[1] = make_uint4(o[4], o[5], o[6], o[7]);
}

// The 16 fp16 biases (already scaled by kappa) of hidden tile ht for lane group g, in accumulator order.
__device__ __forceinline__ void load_bias_tile(const uint4 *__restrict__ b1s, int ht, int g, h2 (&bias)[8])
{
    const uint4 b0 = b1s[(ht * 2 + g) * 2 + 0], b1 = b1s[(ht * 2 + g) * 2 + 1];
    bias[0] = as_h2(b0.x); bias[1] = as_h2(b0.y); bias[2] = as_h2(b0.z); bias[3] = as_h2(b0.w);
    bias[4] = as_h2(b1.x); bias[5] = as_h2(b1.y); bias[6] = as_h2(b1.z); bias[7] = as_h2(b1.w);
}

__device__ __forceinline__ uint32_t pack_half2(float a, float b)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(a, b));
}

}  // namespace slicemoe
