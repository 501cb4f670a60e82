// What the matrix-core routers share: the split of hidden activations, biases in accumulator order, and what follows the second layer (softmax,
// selection).
#pragma once
#include "mfma.h"

namespace slicemoe {

typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x2 __attribute__((ext_vector_type(2)));

// ReLU and the two-term fp16 split of a pair of hidden activations, four instructions: the round-toward-zero conversion
// of the pair; ReLU of both halves as a packed signed-integer max (negative halves are negative integers); and per
// activation one mixed-precision multiply-add a - u0 that rounds to fp16 and clamps to [0, 1].  The clamp is the ReLU of
// the small term (a < 0 has u0 = 0, so a - u0 = a < 0 becomes 0) and leaves a remainder untouched as long as it is
// below 1, i.e. for activations below 2048.
__device__ __forceinline__ void relu_split_pair(float a0, float a1, uint32_t &u0, uint32_t &u1)
{
    const s16x2 raw = __builtin_bit_cast(s16x2, __builtin_amdgcn_cvt_pkrtz(a0, a1));
    const uint32_t hi = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(raw, s16x2{0, 0}));
    uint32_t lo;
    asm("v_fma_mixlo_f16 %0, %1, -1.0, %2 op_sel_hi:[1,0,0] clamp" : "=v"(lo) : "v"(hi), "v"(a0));
    asm("v_fma_mixhi_f16 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0] clamp" : "+v"(lo) : "v"(hi), "v"(a1));
    u0 = hi;
    u1 = lo;
}

__device__ __forceinline__ f32x16 load_bias_tile(const float *__restrict__ b, int tile, int g)
{
    f32x16 r;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const f32x4 v = *(const f32x4 *)(b + tile * 32 + 8 * q + 4 * g);
#pragma unroll
        for (int c = 0; c < 4; ++c) r[4 * q + c] = v[c];
    }
    return r;
}

// What follows the second layer, for one slice per lane pair (j, j + 32) and v[16 et + r] the logit of expert
// 32 et + acc_feature(r, g): logit noise, softmax, top-k, and the selections added to the LDS table counts[64].  MODE:
// inference; with the noise; and with the cross-slice dropout of the selected probabilities (a launch of its own took 2 to 4 us of every
// training step).  Instances of their own, because the unused branches and arguments cost the inference router 0.6 us of 22, and those of
// the dropout the router with the noise 0.6 of a forward's 58 (width 64, 125 000 slices, E = 32).
enum { kRouteInference, kRouteNoise, kRouteDropout };
template <int ET, int MODE>
__device__ __forceinline__ void select_experts(float (&v)[ET * 16], long long n, bool valid, int g, int E, int k,
                                               const float *__restrict__ noise_, float sigma, float exp_scale,
                                               const float *__restrict__ drop_u_, float rate, int32_t *__restrict__ idx,
                                               float *pk, bool count, int *counts)
{
    const float *noise = MODE != kRouteInference ? noise_ : nullptr, *drop_u = MODE == kRouteDropout ? drop_u_ : nullptr;
    float u2[2] = {1.f, 1.f};   // the dropout's draws of a slice with two experts: requested ahead of the softmax
    if (drop_u != nullptr && k == 2 && valid && g == 0) {
        u2[0] = drop_u[n * 2];
        u2[1] = drop_u[n * 2 + 1];
    }
    if (noise != nullptr) {   // training-time logit noise: g += sigma * draw, before the selection and the softmax
        const float *nr = noise + (valid ? n : 0) * E;
        if ((E & 3) == 0) {   // rows of the table are 16-byte aligned: this lane's four consecutive experts at once
#pragma unroll
            for (int et = 0; et < ET; ++et)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int e0 = et * 32 + 8 * q + 4 * g;
                    if (e0 < E) {
                        const f32x4 z = *(const f32x4 *)(nr + e0);
#pragma unroll
                        for (int c = 0; c < 4; ++c) v[et * 16 + 4 * q + c] = fmaf(sigma, z[c], v[et * 16 + 4 * q + c]);
                    }
                }
        } else {
#pragma unroll
            for (int et = 0; et < ET; ++et)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int e = et * 32 + acc_feature(r, g);
                    if (e < E) v[et * 16 + r] = fmaf(sigma, nr[e], v[et * 16 + r]);
                }
        }
    }
    if (E != ET * 32) {   // padded experts never win
#pragma unroll
        for (int et = 0; et < ET; ++et)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (et * 32 + acc_feature(r, g) >= E) v[et * 16 + r] = -INFINITY;
    }
    // Largest and second-largest logit of the lane (the median of the running pair and a new value is the new
    // second), then of the slice: lanes j and j + 32 trade values with one swap instruction whose two results are
    // {own, other} in an order that max / min / + do not care about.
    // (the maximum as a median with +infinity: the median instruction takes its operands as they are, while a
    // floating-point maximum would first spend an instruction on quieting each of them)
    float kInf;   // (opaque to the compiler, which would otherwise turn the medians back into maxima)
    asm("v_mov_b32 %0, 0x7f800000" : "=v"(kInf));
    float m = v[0], second = -INFINITY;
#pragma unroll
    for (int i = 1; i < ET * 16; ++i) {
        second = __builtin_amdgcn_fmed3f(m, second, v[i]);
        m = __builtin_amdgcn_fmed3f(m, v[i], kInf);
    }
    {
        const auto sm = __builtin_amdgcn_permlane32_swap(__float_as_uint(m), __float_as_uint(m), false, false);
        const auto ss = __builtin_amdgcn_permlane32_swap(__float_as_uint(second), __float_as_uint(second), false, false);
        const float m0 = __uint_as_float(sm[0]), m1 = __uint_as_float(sm[1]);
        m = __builtin_amdgcn_fmed3f(m0, m1, kInf);
        const float lower = __builtin_amdgcn_fmed3f(m0, m1, -kInf);   // the smaller of the two maxima (the negation is an operand modifier)
        second = __builtin_amdgcn_fmed3f(__builtin_amdgcn_fmed3f(__uint_as_float(ss[0]), __uint_as_float(ss[1]), kInf), lower, kInf);
    }
    // softmax denominator: exp((v - m) / tau) = exp2(v * c - m * c) with c = log2(e) / tau, one multiply-add and
    // one exp2 per logit
    const float kLog2e = exp_scale;
    const float nm = -m * kLog2e;
    float den = 0.f;
#pragma unroll
    for (int i = 0; i < ET * 16; ++i) den += __builtin_amdgcn_exp2f(fmaf(v[i], kLog2e, nm));
    {
        const auto sd = __builtin_amdgcn_permlane32_swap(__float_as_uint(den), __float_as_uint(den), false, false);
        den = __uint_as_float(sd[0]) + __uint_as_float(sd[1]);
    }
    const float rden = __builtin_amdgcn_rcpf(den);   // within one unit in the last place, like the exp2 above

    // k = 2 with distinct top values (wavefront-wide; anything else takes the general selection below): the two
    // experts are where the two values sit, the lowest index among equals of the second value
    bool picked = false;
    if (k == 2 && __builtin_amdgcn_ballot_w64(!(m > second)) == 0) {
        constexpr int kNone = 1 << 20;
        int ia = kNone, ib = kNone;
#pragma unroll
        for (int i = ET * 16 - 1; i >= 0; --i) {
            const int e0 = (i >> 4) * 32 + acc_feature(i & 15, 0);   // + 4 g below: constants here
            ia = v[i] == m ? e0 : ia;
            ib = v[i] == second ? e0 : ib;
        }
        ia += 4 * g;
        ib += 4 * g;
        const auto sa = __builtin_amdgcn_permlane32_swap((uint32_t)ia, (uint32_t)ia, false, false);
        const auto sb = __builtin_amdgcn_permlane32_swap((uint32_t)ib, (uint32_t)ib, false, false);
        ia = min(min((int)sa[0], (int)sa[1]), E - 1);   // the bound only matters for logits that are not numbers
        ib = min(min((int)sb[0], (int)sb[1]), E - 1);
        if (valid && g == 0) {
            idx[n * 2] = ia;
            idx[n * 2 + 1] = ib;
            float p2[2] = {__builtin_amdgcn_exp2f(fmaf(m, kLog2e, nm)) * rden, __builtin_amdgcn_exp2f(fmaf(second, kLog2e, nm)) * rden};
            if (drop_u != nullptr) drop_assignments(p2, u2, 2, rate);
            pk[n * 2] = p2[0];
            pk[n * 2 + 1] = p2[1];
            if (count) {
                atomicAdd(&counts[ia], 1);
                atomicAdd(&counts[ib], 1);
            }
        }
        picked = true;
    }

    for (int jj = 0; jj < (picked ? 0 : k); ++jj) {
        float bv = v[0];
        int be = acc_feature(0, g);
#pragma unroll
        for (int i = 1; i < ET * 16; ++i) {
            const int e = (i >> 4) * 32 + acc_feature(i & 15, g);
            if (v[i] > bv) {
                bv = v[i];
                be = e;
            }
        }
        const float ov = __shfl_xor(bv, 32);
        const int oe = __shfl_xor(be, 32);
        if (ov > bv || (ov == bv && oe < be)) {
            bv = ov;
            be = oe;
        }
#pragma unroll
        for (int i = 0; i < ET * 16; ++i) {
            const int e = (i >> 4) * 32 + acc_feature(i & 15, g);
            if (e == be) v[i] = -INFINITY;
        }
        if (valid && g == 0) {
            idx[n * k + jj] = be;
            pk[n * k + jj] = __builtin_amdgcn_exp2f(fmaf(bv, kLog2e, nm)) * rden;
            if (count) atomicAdd(&counts[be], 1);
        }
    }
    if (drop_u != nullptr && !picked && valid && g == 0) drop_assignments(pk + n * k, drop_u + n * k, k, rate);   // (this lane has written them)
}

}  // namespace slicemoe
