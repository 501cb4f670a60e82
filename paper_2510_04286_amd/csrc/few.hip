// The whole layer for few tokens in one launch: a block takes a slice from its router to its sum.
//
// slicemoe_forward is four launches whose outputs are the next one's inputs, 16 to 26 us for any small batch, of which the work of 32 tokens
// is a few: what bounds it is launches and round trips.  Grouping by expert, which they are for, saves weight traffic only where an expert
// has several rows.  Here nothing crosses a block.  The eight wavefronts share a slice's router (a hidden tile each) and one of them adds up
// the logits and selects; then they share the k experts' hidden tiles, whose sums become activations a pair of hidden units per thread, and
// the output tiles, several wavefronts to a tile where there are fewer tiles; the k outputs meet in the LDS.
// A slice takes a whole column of the matrix instruction's 32, and all 32 columns hold it: the loads of the weights (48 KB for the router
// and 64 KB per expert at width 64, from the L2) and not the instructions set the pace, and a fragment is read by one lane each.  What
// remains is one chain of router, selection and two layers, each a trip to the L2 (requested ahead where the address is known) and, at width
// 128, two experts of 256 KB through one CU's 44 bytes a cycle.
//
// us in a graph, here / slicemoe_forward: d 1024 in 16 slices of 64 (32 experts, He 256): 1 token 7.1 / 16.0, 32 tokens 9.8 / 18.1; d 4096 in 32 slices
// of 128 (64 experts, He 512): 1 token 11.5 / 22, 8 tokens 16.3 / 24, 16 tokens 29.8 / 24.3 (two rounds of blocks: from 512 slices of 128 columns on
// the four launches are faster); d 768 in 8 slices of 96: 64 tokens 13.1 / 19.6; fp32, d 256 in 4 slices: 64 tokens 13.6 / 26.
//
// Every sum has the order it has in the four launches (route_mfma.hip, ffn_mfma.hip, combine.hip), so the outputs are their bits.
#include "expert_activation.h"
#include "gemm_tile.h"
#include "route_select.h"
#include "wavefront.h"

namespace slicemoe {

constexpr int kFewWaves = 8, kFewThreads = kFewWaves * 64;
constexpr int kFewGroup = 4;   // hidden tiles whose second-layer fragments are requested together

struct FewArgs {
    const bf16_t *x;
    const char *packed;
    PackedLayout L;
    int k, HT;
    uint32_t ht_magic;   // ceil(2^31 / HT): see `job_of`
    int parts_log2, run; // wavefronts that share an output tile, and hidden tiles of each
    bool b2_first;
    EpiConst K;
    bf16_t *out;
    int32_t *idx;
    float *p;
};

// LDS: terms of the router's hidden layer, its second layer, first-layer sums [k][HT][2][16], activations [k][HT][2][2] pieces, outputs [k][ds] fp16.
constexpr int kFewTerms = 8 * 2 * 2 * 2 * 16;
__host__ __device__ constexpr size_t few_router2(int E) { return (size_t)((E + 31) / 32) * 8 * 2 * 64 * 16; }
__host__ __device__ constexpr size_t few_lds(int E, int k, int HT, int ds) { return kFewTerms + few_router2(E) + (size_t)k * HT * 192 + (size_t)k * ds * 2; }

// Largest value over the wavefront.
__device__ __forceinline__ float wavefront_max(float v)
{
    v = fmaxf(v, __int_as_float(lane_move<0xB1>(__float_as_int(v))));
    v = fmaxf(v, __int_as_float(lane_move<0x4E>(__float_as_int(v))));
    v = fmaxf(v, __int_as_float(lane_move<0x141>(__float_as_int(v))));
    v = fmaxf(v, __int_as_float(lane_move<0x140>(__float_as_int(v))));
    const int b = __float_as_int(v);
    return fmaxf(fmaxf(__int_as_float(__builtin_amdgcn_readlane(b, 0)), __int_as_float(__builtin_amdgcn_readlane(b, 16))),
                 fmaxf(__int_as_float(__builtin_amdgcn_readlane(b, 32)), __int_as_float(__builtin_amdgcn_readlane(b, 48))));
}

// The lane with the largest v among the `open` ones, the lowest of equal ones (of values that are not numbers any open lane), which is then closed.
__device__ __forceinline__ int largest_open(float v, int lane, unsigned long long &open)
{
    const bool mine = open >> lane & 1;
    const float most = wavefront_max(mine ? v : -INFINITY);
    const unsigned long long at = __ballot(mine && v == most);
    const int e = __builtin_ctzll(at ? at : open);
    open &= ~(1ull << e);
    return e;
}

// (Two blocks a CU where the registers allow it: 512 slices of width 64 are one round then.)
template <int DS, int ET>
__global__ __launch_bounds__(kFewThreads, DS <= 96 ? 4 : 2) void few_mfma_kernel(FewArgs A)
{
    constexpr int KS = SliceTiles<DS>::KS, OT = SliceTiles<DS>::OT, HTr = 8;
    // First-layer fragments in registers, two sets of them: of two hidden tiles, or of the two halves of one
    constexpr int HALVES = KS == 6 || KS == 24 ? 2 : 1, CH = KS / HALVES;
    constexpr int SETS = DS <= 96 || DS == 384 ? 1 : 2;   // of second-layer fragments: one where two blocks a CU, or wide rows, leave no more registers
    constexpr float kLog2e = 1.4426950408889634f;
    extern __shared__ __align__(16) char lds[];
    u32x4 *us = (u32x4 *)lds;                                    // [HTr][2 K-steps][2 terms][2 lane groups]
    u32x4 *w2s = (u32x4 *)(lds + kFewTerms);                     // [ET][HTr][2][64]
    float *zs = (float *)(lds + kFewTerms + ET * HTr * 2 * 64 * 16);   // [k][HT][2 lane groups][16]
    uint32_t *hs = (uint32_t *)(zs + (size_t)A.k * A.HT * 32);   // [k][HT][2 K-steps][2 lane groups][4]
    half_t *ys = (half_t *)(hs + (size_t)A.k * A.HT * 16);       // [k][DS]
    __shared__ __align__(16) float logits[64];                   // then their exponentials
    __shared__ int sel_idx[8];
    __shared__ float sel_p[8];
    __shared__ f32x4 sums[kFewWaves / 2][4][2];                  // of output tiles that wavefronts share
    const int tid = threadIdx.x, lane = tid & 63, j = lane & 31, g = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const long long n = blockIdx.x;
    const int k = A.k, HT = A.HT;

    const uint4 *xr = (const uint4 *)(A.x + n * DS);
    bf16x8 xb[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) xb[ks] = load_row_piece<DS>(xr, ks, g);
    float v = -INFINITY;   // wavefront 0: the logit of expert `lane`
    {
        const u32x4 *w1 = (const u32x4 *)(A.packed + A.L.r_w1) + wave * KS * 64 + lane;
        u32x4 w1r[KS], w2r[ET][2];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) w1r[ks] = w1[ks * 64];
        f32x16 acc = load_bias_tile((const float *)(A.packed + A.L.r_b1), wave, g), gacc[ET];
        const u32x4 *w2 = (const u32x4 *)(A.packed + A.L.r_w2) + lane;   // [ET][HTr][2][64]
#pragma unroll
        for (int et = 0; et < ET; ++et)
#pragma unroll
            for (int s = 0; s < 2; ++s) w2r[et][s] = w2[((et * HTr + wave) * 2 + s) * 64];
        if (wave == 0)
#pragma unroll
            for (int et = 0; et < ET; ++et) gacc[et] = load_bias_tile((const float *)(A.packed + A.L.r_b2), et, g);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) acc = mfma_bf16(__builtin_bit_cast(bf16x8, w1r[ks]), xb[ks], acc);
        uint32_t t0[8], t1[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) relu_split_pair(acc[2 * i], acc[2 * i + 1], t0[i], t1[i]);
        if (j == 0)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                us[((wave * 2 + s) * 2 + 0) * 2 + g] = u32x4{t0[4 * s], t0[4 * s + 1], t0[4 * s + 2], t0[4 * s + 3]};
                us[((wave * 2 + s) * 2 + 1) * 2 + g] = u32x4{t1[4 * s], t1[4 * s + 1], t1[4 * s + 2], t1[4 * s + 3]};
            }
#pragma unroll
        for (int et = 0; et < ET; ++et)
#pragma unroll
            for (int s = 0; s < 2; ++s) w2s[((et * HTr + wave) * 2 + s) * 64 + lane] = w2r[et][s];
        lds_barrier();
        if (wave == 0) {
            // (the operands are read three K-steps ahead: a chain that waits for each read takes twice as long)
            constexpr int RING = 4, N = 2 * HTr;
            f16x8 u0[RING], u1[RING], a2[RING][ET];
            const auto fetch = [&](auto index) {
                constexpr int I = decltype(index)::value;
                u0[I % RING] = __builtin_bit_cast(f16x8, us[(I * 2 + 0) * 2 + g]);
                u1[I % RING] = __builtin_bit_cast(f16x8, us[(I * 2 + 1) * 2 + g]);
#pragma unroll
                for (int et = 0; et < ET; ++et) a2[I % RING][et] = __builtin_bit_cast(f16x8, w2s[(et * N + I) * 64 + lane]);
            };
            for_range<0, RING - 1>(fetch);
            for_range<0, N>([&](auto index) {
                constexpr int I = decltype(index)::value;
                if constexpr (I + RING - 1 < N) fetch(Int<I + RING - 1>());
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int et = 0; et < ET; ++et)   // small term first
                    gacc[et] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a2[I % RING][et], u1[I % RING], gacc[et], 0, 0, 0);
#pragma unroll
                for (int et = 0; et < ET; ++et) gacc[et] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a2[I % RING][et], u0[I % RING], gacc[et], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            });
            // an expert per lane
            if (j == 0)
#pragma unroll
                for (int et = 0; et < ET; ++et)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        *(f32x4 *)(logits + et * 32 + 8 * q + 4 * g) = f32x4{gacc[et][4 * q], gacc[et][4 * q + 1], gacc[et][4 * q + 2], gacc[et][4 * q + 3]};
            wave_lds_sync();
            if (lane < A.L.E) v = logits[lane];
            unsigned long long open = __ballot(lane < A.L.E);
            for (int jj = 0; jj < k; ++jj) {
                const int e = largest_open(v, lane, open);
                if (lane == 0) sel_idx[jj] = e;
            }
        }
        lds_barrier();
    }
    const int chosen = sel_idx[lane & 7];   // lane jj: the expert of selection jj
    const auto expert = [&](int jj) { return A.packed + A.L.experts + (size_t)__builtin_amdgcn_readlane(chosen, jj) * A.L.e_stride; };
    const uint32_t lane16 = 16 * lane;      // (addresses are a uniform base and this)

    // Second layer: the k OT output tiles, each the sum over all hidden tiles in their order.  With fewer tiles than wavefronts `parts` of these
    // share one: each has a run of the hidden tiles, whose fragments it requests as soon as the experts are known, and passes the sums on.
    const int jobs2 = k * OT, parts = 1 << A.parts_log2, part = wave & (parts - 1), job2 = wave >> A.parts_log2;
    const int first = part * A.run, last = min(HT, first + A.run);   // (the last runs may be empty)
    // job / HT without a division (2^31 / HT rounded up is off by less than HT / 2^31, and jobs are a few thousand)
    const auto job_of = [&](int job) { return (int)__umulhi(2u * (uint32_t)job, A.ht_magic); };
    u32x4 w2[SETS][kFewGroup][2];
    const auto load_w2 = [&](int set, int job, int ht0) {   // [HT][2][OT][64]
        const char *p = expert(job / OT) + A.L.e_w2 + (size_t)(job % OT) * 1024;
#pragma unroll
        for (int i = 0; i < kFewGroup; ++i) {
            const char *t = p + (size_t)min(ht0 + i, HT - 1) * (2 * OT * 1024);
#pragma unroll
            for (int s = 0; s < 2; ++s) w2[set][i][s] = *(const u32x4 *)(t + s * OT * 1024 + lane16);
        }
    };
    const auto bias2 = [&](int job) { return load_bias_tile((const float *)(expert(job / OT) + A.L.e_b2), job % OT, g); };   // padded with zeros by the packer
    // Activations: a pair of hidden units per thread and round (in the accumulators all 32 columns would be the same one).  b1: [HT][2 lane groups][8 pairs]
    const int pairs = k * HT * 16;
    const auto bias1 = [&](int q) {
        const int jj = job_of(q >> 4);
        return ((const uint32_t *)(A.packed + A.L.experts + (size_t)sel_idx[jj] * A.L.e_stride + A.L.e_b1))[q - jj * HT * 16];
    };
    uint32_t b1 = 0;
    f32x16 acc2;
    // First layer: the k HT hidden tiles in turn over the wavefronts.
    {
        const int jobs = k * HT;
        u32x4 w1[2][CH];
        f32x16 acc;
        const auto load_w1 = [&](int set, int job, int half) {
            const int jj = job_of(job);
            const char *p = expert(jj) + A.L.e_w1 + (size_t)(job - jj * HT) * (KS * 1024) + half * (CH * 1024);
#pragma unroll
            for (int i = 0; i < CH; ++i) w1[set][i] = *(const u32x4 *)(p + i * 1024 + lane16);
        };
        const auto multiply = [&](int set, auto which) {
            constexpr int HALF = decltype(which)::value;
            if constexpr (HALF == 0)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[r] = 0.f;
#pragma unroll
            for (int i = 0; i < CH; ++i) acc = mfma_bf16(__builtin_bit_cast(bf16x8, w1[set][i]), xb[HALF * CH + i], acc);
        };
        const auto leave = [&](int job) {
            if (j == 0)
#pragma unroll
                for (int q = 0; q < 4; ++q) *(f32x4 *)(zs + (job * 2 + g) * 16 + 4 * q) = f32x4{acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]};
        };
        load_w1(0, min(wave, jobs - 1), 0);
        if constexpr (HALVES == 2) load_w1(1, min(wave, jobs - 1), 1);
        else load_w1(1, min(wave + kFewWaves, jobs - 1), 0);
        if (job2 < jobs2) {
            load_w2(0, job2, first);
            acc2 = bias2(job2);
        }
        if (tid < pairs) b1 = bias1(tid);
        if (wave == 0) {   // the probabilities, while the weights are on their way; their sum in the order of select_experts
            const float nm = -wavefront_max(v) * kLog2e, ex = __builtin_amdgcn_exp2f(fmaf(v, kLog2e, nm));
            wave_lds_sync();
            logits[lane] = ex;
            wave_lds_sync();
            float den = 0.f;
#pragma unroll
            for (int et = 0; et < ET; ++et)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const f32x4 t = *(const f32x4 *)(logits + et * 32 + 8 * q + 4 * g);
#pragma unroll
                    for (int c = 0; c < 4; ++c) den += t[c];
                }
            const auto sd = __builtin_amdgcn_permlane32_swap(__float_as_uint(den), __float_as_uint(den), false, false);
            const float rden = __builtin_amdgcn_rcpf(__uint_as_float(sd[0]) + __uint_as_float(sd[1]));
            if (lane < k) {
                const int e = sel_idx[lane];
                const float p = logits[e] * rden;
                sel_p[lane] = p;
                if (A.idx) A.idx[n * k + lane] = e;
                if (A.p) A.p[n * k + lane] = p;
            }
        }
        // one hidden tile (two of them) and the requests of the next; the first time outside of the loop: in front of it the second layer's
        // fragments are on their way, and a loop would wait for them
        const auto some = [&](int job) {
            if constexpr (HALVES == 2) {
                multiply(0, Int<0>());
                if (job + kFewWaves < jobs) load_w1(0, job + kFewWaves, 0);
                multiply(1, Int<1>());
                if (job + kFewWaves < jobs) load_w1(1, job + kFewWaves, 1);
                leave(job);
            } else {
                multiply(0, Int<0>());
                leave(job);
                if (job + 2 * kFewWaves < jobs) load_w1(0, job + 2 * kFewWaves, 0);
                if (job + kFewWaves < jobs) {
                    multiply(1, Int<0>());
                    leave(job + kFewWaves);
                }
                if (job + 3 * kFewWaves < jobs) load_w1(1, job + 3 * kFewWaves, 0);
            }
        };
        constexpr int STEP = HALVES == 2 ? kFewWaves : 2 * kFewWaves;
        if (wave < jobs) some(wave);
#pragma unroll 1
        for (int job = wave + STEP; job < jobs; job += STEP) some(job);
    }
    if (SETS == 2 && job2 < jobs2 && first + kFewGroup < last) load_w2(SETS - 1, job2, first + kFewGroup);
    lds_barrier();
    for (int q = tid; q < pairs; q += kFewThreads) {
        const int job = q >> 4, i = q & 7;
        const float pv = sel_p[job_of(job)];
        const h2 p2 = __builtin_bit_cast(h2, __builtin_amdgcn_cvt_pkrtz(pv, pv));
        const float2 z = *(const float2 *)(zs + 2 * q);   // [job][g][pair]
        const uint32_t b = q == tid ? b1 : bias1(q);
        hs[((job * 2 + (i >> 2)) * 2 + (q >> 3 & 1)) * 4 + (i & 3)] = activation_pair(z.x, z.y, p2, as_h2(b), A.K);
    }
    lds_barrier();
    for (int stage = 0; stage < parts; ++stage) {
        if (part == stage)
            for (int job = job2; job < jobs2; job += kFewWaves) {   // (with parts one job at most)
                const int jj = job / OT, ot = job - jj * OT;
                if (job != job2) {
                    acc2 = bias2(job);
                    load_w2(0, job, first);
                    if (SETS == 2 && first + kFewGroup < last) load_w2(SETS - 1, job, first + kFewGroup);
                }
                const f32x16 bias = acc2;
                if (!A.b2_first)
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc2[r] = 0.f;
                if (stage > 0)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const f32x4 t = sums[job][q][g];
#pragma unroll
                        for (int c = 0; c < 4; ++c) acc2[4 * q + c] = t[c];
                    }
                const auto group = [&](int set, int ht0) {
                    f16x8 h[kFewGroup][2];   // (read together; past the end: the last one again)
#pragma unroll
                    for (int i = 0; i < kFewGroup; ++i)
#pragma unroll
                        for (int s = 0; s < 2; ++s)
                            h[i][s] = __builtin_bit_cast(f16x8, *(const u32x4 *)(hs + (((jj * HT + min(ht0 + i, HT - 1)) * 2 + s) * 2 + g) * 4));
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int i = 0; i < kFewGroup; ++i)
                        if (ht0 + i < last)
#pragma unroll
                            for (int s = 0; s < 2; ++s)
                                acc2 = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, w2[set][i][s]), h[i][s], acc2, 0, 0, 0);
                    if (ht0 + SETS * kFewGroup < last) load_w2(set, job, ht0 + SETS * kFewGroup);
                };
                for (int ht0 = first; ht0 < last; ht0 += SETS * kFewGroup) {
                    group(0, ht0);
                    if (SETS == 2 && ht0 + kFewGroup < last) group(SETS - 1, ht0 + kFewGroup);
                }
                if (stage + 1 < parts) {
                    if (j == 0)
#pragma unroll
                        for (int q = 0; q < 4; ++q) sums[job][q][g] = f32x4{acc2[4 * q], acc2[4 * q + 1], acc2[4 * q + 2], acc2[4 * q + 3]};
                } else if (j == 0)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int f = ot * 32 + 8 * q + 4 * g;
                        if (f >= DS) continue;   // padding columns of the last tile
                        float y[4];
#pragma unroll
                        for (int c = 0; c < 4; ++c) y[c] = A.b2_first ? acc2[4 * q + c] : acc2[4 * q + c] + bias[4 * q + c];
                        *(uint2 *)(ys + jj * DS + f) = make_uint2(pack_half2(y[0], y[1]), pack_half2(y[2], y[3]));
                    }
            }
        if (stage + 1 < parts) lds_barrier();
    }
    lds_barrier();
    for (int f = tid; f < DS; f += kFewThreads) {
        float s = 0.f;
        for (int jj = 0; jj < k; ++jj) s += (float)ys[jj * DS + f];
        A.out[n * DS + f] = f32_to_bf16(s);
    }
}

// Any shape, either storage type, fp32 arithmetic on the logical tensors: the columns of a layer by neighbouring threads, the rows of one by several
// where columns are few; the k experts together.  Bound by the L2's latency: sixteen rows in flight (16 tokens of d 256 in fp32: 12.7 us, 15.6 with
// four and one expert after the other).
struct FewGenericArgs {
    const void *x;
    slicemoe_weights w;
    int ds, Hr, E, He, k;
    void *out;
    int32_t *idx;
    float *p;
};
constexpr int kFewGenericThreads = 1024;
static size_t few_generic_lds(int ds, int Hr, int He, int k) { return (size_t)(ds + (Hr > k * He ? Hr : k * He) + kFewGenericThreads + k * ds) * 4; }

// f(o, sum over i < in of v(o)[i] col(o)[i * ld]) for the columns o < n, each by 2^p threads (neighbouring columns by neighbouring threads), sixteen
// rows in flight.
template <typename T, typename VEC, typename COL, typename F>
__device__ __forceinline__ void few_columns(int in, int ld, int n, float *part, const VEC &vec, const COL &col, const F &f)
{
    int p = 0;
    while (p < 5 && (n << (p + 1)) <= kFewGenericThreads && (8 << p) < in) ++p;
    constexpr int kLog2Threads = 10;
    static_assert(1 << kLog2Threads == kFewGenericThreads, "");
    const int parts = 1 << p, log2per = kLog2Threads - p, per = 1 << log2per, tid = threadIdx.x, q = tid >> log2per, lo = tid & (per - 1);
    for (int o0 = 0; o0 < n; o0 += per) {
        const int o = o0 + lo;
        float s = 0.f;
        if (o < n) {
            const T *w = col(o);
            const float *v = vec(o);
            int i = q;
            for (; i + 15 * parts < in; i += 16 * parts) {
                float t[16];
#pragma unroll
                for (int u = 0; u < 16; ++u) t[u] = Storage<T>::load(w + (size_t)(i + u * parts) * ld);
#pragma unroll
                for (int u = 0; u < 16; ++u) s = fmaf(v[i + u * parts], t[u], s);
            }
            for (; i + 3 * parts < in; i += 4 * parts) {
                float t[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) t[u] = Storage<T>::load(w + (size_t)(i + u * parts) * ld);
#pragma unroll
                for (int u = 0; u < 4; ++u) s = fmaf(v[i + u * parts], t[u], s);
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
        if (parts > 1 && o0 + per < n) __syncthreads();
    }
}

template <typename T> __global__ __launch_bounds__(kFewGenericThreads) void few_generic_kernel(FewGenericArgs A)
{
    extern __shared__ __align__(16) char lds[];
    float *xs = (float *)lds, *part = xs + A.ds, *ys = part + kFewGenericThreads, *hid = ys + A.k * A.ds;   // ys: [k][ds], hid: [k][He]
    __shared__ float logit[64], sel_p[8];
    __shared__ int sel_idx[8];
    const int tid = threadIdx.x, ds = A.ds, E = A.E, k = A.k;
    const long long n = blockIdx.x;
    for (int i = tid; i < ds; i += kFewGenericThreads) xs[i] = Storage<T>::load((const T *)A.x + n * ds + i);
    __syncthreads();
    const auto of_x = [&](int) { return xs; };
    const auto of_hidden = [&](int) { return hid; };
    few_columns<T>(ds, A.Hr, A.Hr, part, of_x, [&](int o) { return (const T *)A.w.Wr1 + o; },
                   [&](int o, float s) { hid[o] = fmaxf(s + Storage<T>::load((const T *)A.w.br1 + o), 0.f); });
    __syncthreads();
    few_columns<T>(A.Hr, E, E, part, of_hidden, [&](int o) { return (const T *)A.w.Wr2 + o; },
                   [&](int o, float s) { logit[o] = s + Storage<T>::load((const T *)A.w.br2 + o); });
    __syncthreads();
    if (tid < 64) {   // lane e has expert e
        const float v = tid < E ? logit[tid] : -INFINITY, ex = tid < E ? expf(v - wavefront_max(v)) : 0.f;
        const float den = wavefront_sum_f32(ex);
        unsigned long long open = __ballot(tid < E);
        for (int jj = 0; jj < k; ++jj) {
            const int e = largest_open(v, tid, open);
            if (tid == e) {
                const float p = ex / den;
                sel_idx[jj] = e;
                sel_p[jj] = p;
                if (A.idx) A.idx[n * k + jj] = e;
                if (A.p) A.p[n * k + jj] = p;
            }
        }
    }
    __syncthreads();
    // the k experts together: column o = jj He + hidden unit, then jj ds + output
    const int He = A.He;
    few_columns<T>(ds, He, k * He, part, of_x,
                   [&](int o) {
                       const int jj = o / He;
                       return (const T *)A.w.W1 + (size_t)sel_idx[jj] * ds * He + (o - jj * He);
                   },
                   [&](int o, float s) {
                       const int jj = o / He;
                       const float z = fmaf(sel_p[jj], s, Storage<T>::load((const T *)A.w.b1 + (size_t)sel_idx[jj] * He + (o - jj * He)));
                       hid[o] = 0.5f * z * (1.f + erff(z * 0.70710678118654752f));
                   });
    __syncthreads();
    few_columns<T>(He, ds, k * ds, part, [&](int o) { return hid + o / ds * He; },
                   [&](int o) {
                       const int jj = o / ds;
                       return (const T *)A.w.W2 + (size_t)sel_idx[jj] * He * ds + (o - jj * ds);
                   },
                   [&](int o, float s) {
                       const int jj = o / ds;
                       ys[o] = s + Storage<T>::load((const T *)A.w.b2 + (size_t)sel_idx[jj] * ds + (o - jj * ds));
                   });
    __syncthreads();
    for (int i = tid; i < ds; i += kFewGenericThreads) {
        float s = 0.f;
        for (int jj = 0; jj < k; ++jj) s += ys[jj * ds + i];
        Storage<T>::store((T *)A.out + n * ds + i, s);
    }
}

size_t few_lds_bytes(const slicemoe_config &c, bool mfma)
{
    const int ds = c.d / c.S;
    return mfma ? few_lds(c.E, c.k, c.He / 32, ds) : few_generic_lds(ds, c.Hr, c.He, c.k);
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
    const int HT = c.He / 32, tiles = c.k * ((ds + 31) / 32);
    int parts_log2 = 0;   // output tiles times parts: at most the wavefronts
    while (tiles << (parts_log2 + 1) <= kFewWaves) ++parts_log2;
    const int run = (HT + (1 << parts_log2) - 1) >> parts_log2;
    const FewArgs A{(const bf16_t *)h, (const char *)w.packed, packed_layout(c), c.k, HT, (uint32_t)(((1ull << 31) + HT - 1) / HT), parts_log2, run,
                    ffn_bias_first(c), make_epi_const(), (bf16_t *)h_out, idx, p};
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
