// The whole layer for few tokens in one launch: a block takes a slice from its router to its sum.
//
// slicemoe_forward is four launches whose outputs are the next one's inputs, 18 to 26 us for any small batch, of which the work of 32 tokens
// is a few: what bounds it is launches and round trips.  Grouping by expert, which they are for, saves weight traffic only where an expert
// has several rows.  Here nothing crosses a block: the eight wavefronts share a slice's router (a hidden tile each), one of them adds up
// the logits and selects, then they share the k experts' hidden tiles and, behind a barrier, their output tiles; the k outputs meet in the LDS.
// A slice takes a whole column of the matrix instruction's 32, and all 32 columns hold it: the loads of the weights (48 KB for the router
// and 64 KB per expert at width 64, from the L2) and not the instructions set the pace, and a fragment is read by one lane each.
//
// Every sum has the order it has in the four launches (route_mfma.hip, ffn_mfma.hip, combine.hip), so the outputs are their bits.
#include "expert_activation.h"
#include "route_select.h"
#include "wavefront.h"

namespace slicemoe {

constexpr int kFewWaves = 8, kFewThreads = kFewWaves * 64;
constexpr int kFewGroup = 4;   // hidden tiles whose second-layer fragments a wavefront holds, twice: these and the next ones

struct FewArgs {
    const bf16_t *x;
    const char *packed;
    PackedLayout L;
    int k, HT;
    bool b2_first;
    EpiConst K;
    bf16_t *out;
    int32_t *idx;
    float *p;
};

// LDS: terms of the router's hidden layer, its second layer, activations [k][HT][2][2] pieces, outputs [k][ds] fp16.
constexpr int kFewTerms = 8 * 2 * 2 * 2 * 16;
__host__ __device__ constexpr size_t few_router2(int E) { return (size_t)((E + 31) / 32) * 8 * 2 * 64 * 16; }
__host__ __device__ constexpr size_t few_lds(int E, int k, int HT, int ds) { return kFewTerms + few_router2(E) + (size_t)k * HT * 64 + (size_t)k * ds * 2 + 64; }

// (Two blocks a CU where the registers allow it: 512 slices of width 64 are one round then.)
template <int DS, int ET>
__global__ __launch_bounds__(kFewThreads, DS <= 64 ? 4 : 2) void few_mfma_kernel(FewArgs A)
{
    constexpr int KS = SliceTiles<DS>::KS, OT = SliceTiles<DS>::OT, HTr = 8;
    constexpr bool AHEAD = KS <= 8;   // the next hidden tile's fragments are requested before this one's are used
    extern __shared__ __align__(16) char lds[];
    uint4 *us = (uint4 *)lds;                                    // [HTr][2 K-steps][2 terms][2 lane groups]
    uint4 *w2s = (uint4 *)(lds + kFewTerms);                     // [ET][HTr][2][64]
    char *rest = lds + kFewTerms + ET * HTr * 2 * 64 * 16;
    uint4 *hs = (uint4 *)rest;                                   // [k][HT][2][2]
    half_t *ys = (half_t *)(rest + (size_t)A.k * A.HT * 64);     // [k][DS]
    __shared__ int sel_idx[8];
    __shared__ float sel_p[8];
    const int tid = threadIdx.x, lane = tid & 63, j = lane & 31, g = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const long long n = blockIdx.x;
    const int k = A.k, HT = A.HT;

    const uint4 *xr = (const uint4 *)(A.x + n * DS);
    bf16x8 xb[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) xb[ks] = load_row_piece<DS>(xr, ks, g);
    {
        const uint4 *w1 = (const uint4 *)(A.packed + A.L.r_w1) + wave * KS * 64 + lane;
        uint4 w1r[KS], w2r[ET][2];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) w1r[ks] = w1[ks * 64];
        const uint4 *w2 = (const uint4 *)(A.packed + A.L.r_w2) + lane;   // [ET][HTr][2][64]
#pragma unroll
        for (int et = 0; et < ET; ++et)
#pragma unroll
            for (int s = 0; s < 2; ++s) w2r[et][s] = w2[((et * HTr + wave) * 2 + s) * 64];
        f32x16 acc = load_bias_tile((const float *)(A.packed + A.L.r_b1), wave, g), gacc[ET];
        if (wave == 0)
#pragma unroll
            for (int et = 0; et < ET; ++et) gacc[et] = load_bias_tile((const float *)(A.packed + A.L.r_b2), et, g);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) acc = mfma_bf16(__builtin_bit_cast(bf16x8, w1r[ks]), xb[ks], acc);
#pragma unroll
        for (int et = 0; et < ET; ++et)
#pragma unroll
            for (int s = 0; s < 2; ++s) w2s[((et * HTr + wave) * 2 + s) * 64 + lane] = w2r[et][s];
        uint32_t t0[8], t1[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) relu_split_pair(acc[2 * i], acc[2 * i + 1], t0[i], t1[i]);
        if (j == 0)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                us[((wave * 2 + s) * 2 + 0) * 2 + g] = make_uint4(t0[4 * s], t0[4 * s + 1], t0[4 * s + 2], t0[4 * s + 3]);
                us[((wave * 2 + s) * 2 + 1) * 2 + g] = make_uint4(t1[4 * s], t1[4 * s + 1], t1[4 * s + 2], t1[4 * s + 3]);
            }
        lds_barrier();
        if (wave == 0) {
#pragma unroll
            for (int h = 0; h < HTr; ++h)
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const f16x8 u0 = __builtin_bit_cast(f16x8, us[((h * 2 + s) * 2 + 0) * 2 + g]);
                    const f16x8 u1 = __builtin_bit_cast(f16x8, us[((h * 2 + s) * 2 + 1) * 2 + g]);
#pragma unroll
                    for (int et = 0; et < ET; ++et) {   // small term first
                        const f16x8 a2 = __builtin_bit_cast(f16x8, w2s[((et * HTr + h) * 2 + s) * 64 + lane]);
                        gacc[et] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a2, u1, gacc[et], 0, 0, 0);
                        gacc[et] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a2, u0, gacc[et], 0, 0, 0);
                    }
                }
            float v[ET * 16];
#pragma unroll
            for (int et = 0; et < ET; ++et)
#pragma unroll
                for (int r = 0; r < 16; ++r) v[et * 16 + r] = gacc[et][r];
            select_experts<ET, kRouteInference>(v, 0, j == 0, g, A.L.E, k, nullptr, 0.f, 1.4426950408889634f, nullptr, 0.f, sel_idx, sel_p, false, nullptr);
        }
        lds_barrier();
    }
    if (tid < k) {   // (the selection is in range whatever the logits are: see select_experts)
        if (A.idx) A.idx[n * k + tid] = sel_idx[tid];
        if (A.p) A.p[n * k + tid] = sel_p[tid];
    }
    const auto expert = [&](int jj) { return A.packed + A.L.experts + (size_t)__builtin_amdgcn_readfirstlane(sel_idx[jj]) * A.L.e_stride; };

    // Second layer: the k OT output tiles, each the sum over all hidden tiles in their order, kFewGroup of them at a time.
    const int jobs2 = k * OT;
    uint4 w2[2][kFewGroup][2];
    const auto load_w2 = [&](int set, int job, int ht0) {   // [HT][2][OT][64]
        const uint4 *p = (const uint4 *)(expert(job / OT) + A.L.e_w2) + (size_t)(job % OT) * 64 + lane;
#pragma unroll
        for (int i = 0; i < kFewGroup; ++i)
#pragma unroll
            for (int s = 0; s < 2; ++s) w2[set][i][s] = p[(size_t)(min(ht0 + i, HT - 1) * 2 + s) * OT * 64];
    };
    // First layer: the k HT hidden tiles in turn over the wavefronts.
    {
        const int jobs = k * HT;
        uint4 w1[AHEAD ? 2 : 1][KS];
        const auto load_w1 = [&](int set, int job) {
            const uint4 *p = (const uint4 *)(expert(job / HT) + A.L.e_w1) + (size_t)(job % HT) * KS * 64 + lane;
#pragma unroll
            for (int i = 0; i < KS; ++i) w1[set][i] = p[i * 64];
        };
        const auto tile = [&](int set, int job) {
            const int jj = job / HT, ht = job - jj * HT;
            h2 bias[8];
            load_bias_tile((const uint4 *)(expert(jj) + A.L.e_b1), ht, g, bias);
            const float pv = sel_p[jj];
            const h2 p2 = __builtin_bit_cast(h2, __builtin_amdgcn_cvt_pkrtz(pv, pv));
            f32x16 acc;
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[r] = 0.f;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) acc = mfma_bf16(__builtin_bit_cast(bf16x8, w1[set][ks]), xb[ks], acc);
            uint4 hb[2];
            activation_tile(acc, p2, bias, A.K, hb);
            if (j == 0)
#pragma unroll
                for (int s = 0; s < 2; ++s) hs[(job * 2 + s) * 2 + g] = hb[s];
        };
        load_w1(0, min(wave, jobs - 1));
        if (wave < jobs2) load_w2(0, wave, 0);
#pragma unroll 1
        for (int job = wave; job < jobs; job += AHEAD ? 2 * kFewWaves : kFewWaves) {
            if constexpr (AHEAD) {   // (past the end: the last one again)
                load_w1(1, min(job + kFewWaves, jobs - 1));
                tile(0, job);
                load_w1(0, min(job + 2 * kFewWaves, jobs - 1));
                if (job + kFewWaves < jobs) tile(1, job + kFewWaves);
            } else {
                tile(0, job);
                load_w1(0, min(job + kFewWaves, jobs - 1));
            }
        }
    }
    if (wave < jobs2 && HT > kFewGroup) load_w2(1, wave, kFewGroup);
    lds_barrier();
    for (int job = wave; job < jobs2; job += kFewWaves) {
        const int jj = job / OT, ot = job - jj * OT;
        const f32x16 bias = load_bias_tile((const float *)(expert(jj) + A.L.e_b2), ot, g);   // padded with zeros by the packer
        f32x16 acc;
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[r] = A.b2_first ? bias[r] : 0.f;
        if (job != wave) {
            load_w2(0, job, 0);
            if (HT > kFewGroup) load_w2(1, job, kFewGroup);
        }
        const auto group = [&](int set, int ht0) {
#pragma unroll
            for (int i = 0; i < kFewGroup; ++i) {
                if (ht0 + i >= HT) break;
#pragma unroll
                for (int s = 0; s < 2; ++s)
                    acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, w2[set][i][s]),
                                                                 __builtin_bit_cast(f16x8, hs[((jj * HT + ht0 + i) * 2 + s) * 2 + g]), acc, 0, 0, 0);
            }
            if (ht0 + 2 * kFewGroup < HT) load_w2(set, job, ht0 + 2 * kFewGroup);
        };
        for (int ht0 = 0; ht0 < HT; ht0 += 2 * kFewGroup) {
            group(0, ht0);
            if (ht0 + kFewGroup < HT) group(1, ht0 + kFewGroup);
        }
        if (j == 0)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int f = ot * 32 + 8 * q + 4 * g;
                if (f >= DS) continue;   // padding columns of the last tile
                float v[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) v[c] = A.b2_first ? acc[4 * q + c] : acc[4 * q + c] + bias[4 * q + c];
                *(uint2 *)(ys + jj * DS + f) = make_uint2(pack_half2(v[0], v[1]), pack_half2(v[2], v[3]));
            }
    }
    lds_barrier();
    for (int f = tid; f < DS; f += kFewThreads) {
        float s = 0.f;
        for (int jj = 0; jj < k; ++jj) s += (float)ys[jj * DS + f];
        A.out[n * DS + f] = f32_to_bf16(s);
    }
}

// Any shape, either storage type, fp32 arithmetic on the logical tensors: a thread per hidden unit, then per output.
struct FewGenericArgs {
    const void *x;
    slicemoe_weights w;
    int ds, Hr, E, He, k;
    void *out;
    int32_t *idx;
    float *p;
};
constexpr int kFewGenericThreads = 256;
static size_t few_generic_lds(int ds, int Hr, int He) { return (size_t)(ds + (Hr > He ? Hr : He) + kFewGenericThreads + ds) * 4; }

// out[o] = sum over i < in of v[i] W[i * ld + o] for o < n, by `parts` threads each (a power of two that divides 256 into columns): f(o, sum).
template <typename T, typename F>
__device__ __forceinline__ void few_columns(const float *v, int in, const T *__restrict__ W, int ld, int n, float *part, const F &f)
{
    int parts = 1;
    while (parts < 16 && parts * 2 * n <= kFewGenericThreads) parts *= 2;
    const int per = kFewGenericThreads / parts, tid = threadIdx.x, q = tid / per, lo = tid % per;
    for (int o0 = 0; o0 < n; o0 += per) {
        const int o = o0 + lo;
        float s = 0.f;
        if (o < n) {
            const T *w = W + o;
            int i = q;
            for (; i + 7 * parts < in; i += 8 * parts) {   // eight rows in flight
                float t[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) t[u] = Storage<T>::load(w + (size_t)(i + u * parts) * ld);
#pragma unroll
                for (int u = 0; u < 8; ++u) s = fmaf(v[i + u * parts], t[u], s);
            }
            for (; i < in; i += parts) s = fmaf(v[i], Storage<T>::load(w + (size_t)i * ld), s);
        }
        if (parts > 1) {
            part[tid] = s;
            __syncthreads();
            s = 0.f;
            if (q == 0)
                for (int u = 0; u < parts; ++u) s += part[u * per + lo];
        }
        if (q == 0 && o < n) f(o, s);
        if (parts > 1) __syncthreads();
    }
}

template <typename T> __global__ __launch_bounds__(kFewGenericThreads) void few_generic_kernel(FewGenericArgs A)
{
    extern __shared__ __align__(16) char lds[];
    float *xs = (float *)lds, *hid = xs + A.ds, *part = hid + (A.Hr > A.He ? A.Hr : A.He), *ys = part + kFewGenericThreads;
    __shared__ float logit[64], sel_p[8];
    __shared__ int sel_idx[8];
    const int tid = threadIdx.x, ds = A.ds, E = A.E, k = A.k;
    const long long n = blockIdx.x;
    for (int i = tid; i < ds; i += kFewGenericThreads) {
        xs[i] = Storage<T>::load((const T *)A.x + n * ds + i);
        ys[i] = 0.f;
    }
    __syncthreads();
    few_columns<T>(xs, ds, (const T *)A.w.Wr1, A.Hr, A.Hr, part, [&](int o, float s) { hid[o] = fmaxf(s + Storage<T>::load((const T *)A.w.br1 + o), 0.f); });
    __syncthreads();
    few_columns<T>(hid, A.Hr, (const T *)A.w.Wr2, E, E, part, [&](int o, float s) { logit[o] = s + Storage<T>::load((const T *)A.w.br2 + o); });
    __syncthreads();
    if (tid < 64) {   // lane e has expert e; equal logits go to the lower one
        float v = tid < E ? logit[tid] : -INFINITY;
        float m = v;
#pragma unroll
        for (int i = 32; i > 0; i >>= 1) m = fmaxf(m, __shfl_xor(m, i));
        const float ex = tid < E ? expf(v - m) : 0.f;
        const float den = wavefront_sum_f32(ex);
        bool free_ = tid < E;
        for (int jj = 0; jj < k; ++jj) {
            float bv = free_ ? v : -INFINITY;
            int be = free_ ? tid : 64 + tid;
#pragma unroll
            for (int i = 32; i > 0; i >>= 1) {
                const float ov = __shfl_xor(bv, i);
                const int oe = __shfl_xor(be, i);
                if (ov > bv || (!(bv > ov) && oe < be)) {
                    bv = ov;
                    be = oe;
                }
            }
            be = __builtin_amdgcn_readfirstlane(be);   // (the lanes agree but where logits are not numbers; nor does the bound matter elsewhere)
            be = be < E ? be : E - 1;
            if (tid == be) {
                free_ = false;
                sel_idx[jj] = be;
                sel_p[jj] = ex / den;
            }
        }
    }
    __syncthreads();
    if (tid < k) {
        if (A.idx) A.idx[n * k + tid] = sel_idx[tid];
        if (A.p) A.p[n * k + tid] = sel_p[tid];
    }
    for (int jj = 0; jj < k; ++jj) {
        const int e = sel_idx[jj];
        const float p = sel_p[jj];
        const T *b1 = (const T *)A.w.b1 + (size_t)e * A.He, *b2 = (const T *)A.w.b2 + (size_t)e * ds;
        few_columns<T>(xs, ds, (const T *)A.w.W1 + (size_t)e * ds * A.He, A.He, A.He, part, [&](int o, float s) {
            const float z = fmaf(p, s, Storage<T>::load(b1 + o));
            hid[o] = 0.5f * z * (1.f + erff(z * 0.70710678118654752f));
        });
        __syncthreads();
        few_columns<T>(hid, A.He, (const T *)A.w.W2 + (size_t)e * A.He * ds, ds, ds, part, [&](int o, float s) { ys[o] += s + Storage<T>::load(b2 + o); });
        __syncthreads();
    }
    for (int i = tid; i < ds; i += kFewGenericThreads) Storage<T>::store((T *)A.out + n * ds + i, ys[i]);
}

size_t few_lds_bytes(const slicemoe_config &c, bool mfma)
{
    const int ds = c.d / c.S;
    return mfma ? few_lds(c.E, c.k, c.He / 32, ds) : few_generic_lds(ds, c.Hr, c.He);
}

template <int DS> static hipError_t run_few(const slicemoe_config &c, const FewArgs &A, size_t lds, hipStream_t s)
{
    const auto kern = c.E <= 32 ? few_mfma_kernel<DS, 1> : few_mfma_kernel<DS, 2>;
    const hipError_t e = grant_dynamic_lds((const void *)kern, lds);
    if (e != hipSuccess) return e;
    kern<<<c.T * c.S, kFewThreads, lds, s>>>(A);
    return hipGetLastError();
}

hipError_t launch_forward_few(const slicemoe_config &c, const void *h, const slicemoe_weights &w, bool mfma, void *h_out, int32_t *idx, float *p,
                              hipStream_t s)
{
    if (c.T == 0) return hipSuccess;
    const int ds = c.d / c.S;
    const size_t lds = few_lds_bytes(c, mfma);
    if (!mfma) {
        const FewGenericArgs A{h, w, ds, c.Hr, c.E, c.He, c.k, h_out, idx, p};
        const auto kern = c.dtype == SLICEMOE_BF16 ? few_generic_kernel<bf16_t> : few_generic_kernel<float>;
        const hipError_t e = grant_dynamic_lds((const void *)kern, lds);
        if (e != hipSuccess) return e;
        kern<<<c.T * c.S, kFewGenericThreads, lds, s>>>(A);
        return hipGetLastError();
    }
    const FewArgs A{(const bf16_t *)h, (const char *)w.packed, packed_layout(c), c.k, c.He / 32, ffn_bias_first(c), make_epi_const(), (bf16_t *)h_out, idx, p};
    switch (ds) {
        case 24: return run_few<24>(c, A, lds, s);
        case 48: return run_few<48>(c, A, lds, s);
        case 64: return run_few<64>(c, A, lds, s);
        case 96: return run_few<96>(c, A, lds, s);
        case 128: return run_few<128>(c, A, lds, s);
        case 192: return run_few<192>(c, A, lds, s);
        default: return run_few<384>(c, A, lds, s);
    }
}

}  // namespace slicemoe
