// Gated feed-forward network that every token takes, forward and backward:
//
//   g = x Wg,  u = x Wu,  a = silu(g) u,  y = addend + a Wd                      (silu(g) = g sg,  sg = 1 / (1 + exp(-g)))
//   da = dy Wd^T,  dg = da u (sg + g sg (1 - sg)),  du = da g sg
//   dx = addend + dg Wg^T + du Wu^T,  dWg = x^T dg,  dWu = x^T du,  dWd = a^T dy
//
// A product is a tile of gemm_tile.h on the bf16 matrix cores with fp32 accumulation (few fp32 rows: on the fp32 matrix instruction); no
// transposed copy of anything is made (K-major operands are read transposed from the LDS).  Both projections share a tile, so that the
// gate is applied to the accumulators; the backward pass computes them again beside da, and the three weight gradients are one launch.  g, u
// and da stay on the chip, but where few tiles share out a long contraction: then their sums pass through memory in fp32.  a, dg and du are
// rounded to bf16 once (bf16 storage), so an output holds that rounding and its own: 1.4 times the error of one.
//
// Bound by the matrix cores and, where they are busy, by power: at T 8192, d 4096, H 11008 (bf16) up 1118 us = 1.32 PFLOP/s, down 562 =
// 1.31, gate backward 1866 = 1.19, weight gradients 1779 = 1.25, dx 1074 = 1.38, with the matrix pipes 63 to 81% busy at 1.65 to
// 1.8 GHz (a large library product: 1.0 to 1.5 on the same card); 8-bit projections of 4096 rows 374 us = 1.98 PFLOP/s.  Cards differ by
// 8% (up: 1063 to 1148 us).  Short contractions pay their rounds' first trip and epilogue: 16 steps (d = 1024) 31 us a round, 23 of them
// steps.
#include <algorithm>

#include "gated_ffn.h"
#include "gemm_tile.h"
#include "norm.h"

namespace slicemoe {

// ---- fp32 values as bf16 terms -------------------------------------------------------------------------------------------
// fp32 storage: an operand is the sum of three bf16 values, cut off rather than rounded, so that the remainders are exact and all 24 bits
// are kept (of a value below some 2^-108 those above 2^-133, bf16's smallest number).  A product is the six products of terms whose orders add up to at most two, largest first (the matrix instruction cuts its
// accumulator when the products outweigh it); what is left out is below 2^-21 of the product and has its sign (for normal random operands
// 2^-25 in the mean).  (A forward pass of few rows is bound by the weights and takes the fp32 instruction instead: see
// gated_few_f32_kernel.)
// An infinity is infinite in all three terms, and no term of a nonzero value is zero, since 2^-40 of the value is added to either
// remainder: the six products then are infinities of the product's sign, as in fp32 arithmetic, where infinity times a zero term would be
// NaN.  A NaN is one at least in the last term, whatever its payload.
// Six bf16 products run at 2.6 times the rate of the fp32 matrix instruction; errors against 64 bits 4e-7 (the library's fp32
// product: 7e-7).
constexpr int kPairs = 6;
constexpr int kPairR[kPairs] = {0, 0, 1, 1, 0, 2}, kPairF[kPairs] = {0, 1, 0, 1, 2, 0};

__device__ __forceinline__ void split_terms(float v, bf16_t (&t)[3])
{
    const uint32_t b = __float_as_uint(v);
    const bool finite = (b & 0x7f800000u) != 0x7f800000u;
    const float r1 = finite ? fmaf(v, 0x1p-40f, v - __uint_as_float(b & 0xffff0000u)) : v;
    const uint32_t b1 = __float_as_uint(r1);
    const float r2 = finite ? fmaf(v, 0x1p-40f, r1 - __uint_as_float(b1 & 0xffff0000u)) : v;
    t[0] = (bf16_t)(b >> 16);
    t[1] = (bf16_t)(b1 >> 16);
    t[2] = f32_to_bf16(r2);
}

// Eight values of a row as bf16 terms, zeros past the row's end (up to a whole 16-byte piece).
template <int TERMS> __device__ __forceinline__ void store_terms(bf16_t *p, size_t term, int col, int cols, const float *v)
{
    union {
        bf16_t h[8];
        uint4 q;
    } o[TERMS];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float x = col + i < cols ? v[i] : 0.f;
        if constexpr (TERMS == 3) {
            bf16_t t[3];
            split_terms(x, t);
#pragma unroll
            for (int k = 0; k < 3; ++k) o[k].h[i] = t[k];
        } else
            o[0].h[i] = f32_to_bf16(x);
    }
#pragma unroll
    for (int k = 0; k < TERMS; ++k) *(uint4 *)(p + k * term + col) = o[k].q;
}

typedef u32x4 __attribute__((aligned(2))) loose;   // 16 bytes at any element

struct CopyJob {
    const void *src;
    bf16_t *dst;
    int rows, cols, ld;
};
struct CopyJobs {
    CopyJob j[5];
    int f32;
};
// One 16-byte piece of the copy per thread.  Memory-bound: three terms of 3405 x 2705 and three weight matrices of 2705 x 244 23 us.
__global__ __launch_bounds__(256) void gated_copy_kernel(CopyJobs jobs)
{
    const CopyJob j = jobs.j[blockIdx.y];
    const int per_row = j.ld / 8;
    const long long n = (long long)j.rows * per_row;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) {
        const long long row = i / per_row;
        const int col = (int)(i - row * per_row) * 8;
        float v[8];
        const size_t at = (size_t)row * j.cols + col;
        if (col + 8 <= j.cols) {   // (a row may start at any element)
            if (jobs.f32) {
                const u32x4 a = *(const loose *)((const float *)j.src + at), b = *(const loose *)((const float *)j.src + at + 4);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    v[k] = __uint_as_float(a[k]);
                    v[4 + k] = __uint_as_float(b[k]);
                }
            } else {
                const u32x4 a = *(const loose *)((const bf16_t *)j.src + at);
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = __uint_as_float(k & 1 ? a[k >> 1] & 0xffff0000u : a[k >> 1] << 16);
            }
        } else
#pragma unroll
            for (int k = 0; k < 8; ++k)
                v[k] = col + k < j.cols ? (jobs.f32 ? ((const float *)j.src)[at + k] : bf16_to_f32(((const bf16_t *)j.src)[at + k])) : 0.f;
        bf16_t *d = j.dst + (size_t)row * j.ld;
        if (jobs.f32) store_terms<3>(d, (size_t)j.rows * j.ld, col, j.cols, v);
        else store_terms<1>(d, 0, col, j.cols, v);
    }
}

// ---- epilogues -----------------------------------------------------------------------------------------------------------
// 32 rows of a wavefront's accumulators (of NT feature tiles) leave through its own part of the LDS, so that eight consecutive
// features of a row come to one lane: put(row of the 32, feature of the tiles, eight values, which of the lane's pieces).
template <int NT, typename GET, typename PUT> __device__ __forceinline__ void store_rows(char *lds, const GET &get, const PUT &put)
{
    constexpr int W = 32 * NT, STRIDE = W + 4, PIECES = W / 8;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, j = lane & 31, g = lane >> 5;
    float *st = (float *)lds + wave * 32 * STRIDE;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const f32x16 v = get(t);
#pragma unroll
        for (int q = 0; q < 4; ++q) *(f32x4 *)(st + j * STRIDE + 32 * t + 8 * q + 4 * g) = f32x4{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
    }
    wave_lds_sync();
#pragma unroll
    for (int i = 0; i < PIECES / 2; ++i) {
        const int k = i * 64 + lane, r = k / PIECES, c = k % PIECES;
        const f32x4 lo = *(const f32x4 *)(st + r * STRIDE + 8 * c), hi = *(const f32x4 *)(st + r * STRIDE + 8 * c + 4);
        const float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        put(r, 8 * c, v, i);
    }
    wave_lds_sync();
    __builtin_amdgcn_sched_barrier(0);   // (the next rows' accumulators stay where they are until then)
}
constexpr int stage_bytes(int nt) { return 4 * 32 * (32 * nt + 4) * 4; }

struct Out {
    void *p;              // [rows][cols], bf16 or fp32
    const void *addend;   // the same layout, or none
    int rows, cols;
    int f32;
};
// The addend of eight columns of a row, where they are whole (zeros elsewhere and without one); 16-byte accesses at any element.
struct Addend {
    u32x4 lo, hi;   // hi: fp32 only
};
__device__ __forceinline__ Addend fetch_addend(const Out &o, int row, int col)
{
    Addend a = {{0, 0, 0, 0}, {0, 0, 0, 0}};
    if (o.addend && row < o.rows && col + 8 <= o.cols) {
        const size_t at = (size_t)row * o.cols + col;
        a.lo = *(const loose *)((const char *)o.addend + at * (o.f32 ? 4 : 2));
        if (o.f32) a.hi = *(const loose *)((const float *)o.addend + at + 4);
    }
    return a;
}
// out = addend + v for eight columns of a row; past the row's end value by value.
__device__ __forceinline__ void put_out(const Out &o, int row, int col, const float *v, const Addend &d)
{
    if (row >= o.rows || col >= o.cols) return;
    const size_t at = (size_t)row * o.cols + col;
    if (col + 8 <= o.cols) {
        if (o.f32) {
            const f32x4 a = f32x4{v[0], v[1], v[2], v[3]} + __builtin_bit_cast(f32x4, d.lo), b = f32x4{v[4], v[5], v[6], v[7]} + __builtin_bit_cast(f32x4, d.hi);
            *(loose *)((float *)o.p + at) = __builtin_bit_cast(u32x4, a);
            *(loose *)((float *)o.p + at + 4) = __builtin_bit_cast(u32x4, b);
        } else {
            u32x4 r;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                r[i] = (uint32_t)f32_to_bf16(v[2 * i] + __uint_as_float(d.lo[i] << 16)) |
                       (uint32_t)f32_to_bf16(v[2 * i + 1] + __uint_as_float(d.lo[i] & 0xffff0000u)) << 16;
            *(loose *)((bf16_t *)o.p + at) = r;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (col + i >= o.cols) break;
        if (o.f32) ((float *)o.p)[at + i] = v[i] + (o.addend ? ((const float *)o.addend)[at + i] : 0.f);
        else ((bf16_t *)o.p)[at + i] = f32_to_bf16(v[i] + (o.addend ? bf16_to_f32(((const bf16_t *)o.addend)[at + i]) : 0.f));
    }
}
__device__ __forceinline__ void put_out(const Out &o, int row, int col, const float *v) { put_out(o, row, col, v, fetch_addend(o, row, col)); }

template <bool PRECISE> __device__ __forceinline__ float sigmoid(float g)
{
    if constexpr (PRECISE) return 1.f / (1.f + expf(-g));
    return __builtin_amdgcn_rcpf(1.f + __expf(-g));
}

struct Hidden {
    bf16_t *p[3];         // a, dg, du: [terms][rows][ld]
    int rows, cols, ld;
};
constexpr int kAsF32 = 4;   // in place of a number of terms: rows of fp32 values
template <int TERMS> __device__ __forceinline__ void put_hidden(const Hidden &h, int which, int row, int col, const float *v)
{
    if (row >= h.rows || col >= h.cols) return;
    if constexpr (TERMS == kAsF32) {   // (past the row's end, in its padding, is not read)
        float *q = (float *)h.p[which] + (size_t)row * h.ld + col;
        *(f32x4 *)q = f32x4{v[0], v[1], v[2], v[3]};
        *(f32x4 *)(q + 4) = f32x4{v[4], v[5], v[6], v[7]};
    } else
        store_terms<TERMS>(h.p[which] + (size_t)row * h.ld, (size_t)h.rows * h.ld, col, h.cols, v);
}

struct Scales {
    const float *x, *g, *u;   // per row of x, per hidden unit of Wg and Wu (e4m3 operands)
};

// ---- kernels -------------------------------------------------------------------------------------------------------------
template <typename S> __device__ __forceinline__ void clear(f32x16 (&acc)[S::TF][S::TR])
{
#pragma unroll
    for (int t = 0; t < S::TF; ++t)
#pragma unroll
        for (int u = 0; u < S::TR; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[t][u][i] = 0.f;
}

__device__ __forceinline__ void share_of(const GemmProblem &p, int split, int &s0, int &s1)
{
    const int steps = p.segments * ((p.K + 127) >> 7), each = (steps + p.splits - 1) / p.splits;
    s0 = split * each;
    s1 = s0 + each < steps ? s0 + each : steps;
}

// Both projections and the gate (big tiles, T 16384, d 1024, H 2816: 184 to 215 us; the gate's exponential and reciprocal are 4 us
// of vector work per tile, the rows leave in whole 128-byte lines).
template <typename S, int TERMS>
__global__ __launch_bounds__(256) void gated_up_kernel(GemmProblem p, Hidden h, Scales sc)
{
    extern __shared__ __align__(1024) char lds[];
    const TilePlace at = tile_of(blockIdx.x, p.tiles_r, p.tiles_f, p.splits);
    const int row0 = at.r * S::BR, f0 = at.f * S::BF, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    f32x16 acc[S::TF][S::TR];
    clear<S>(acc);
    mma_steps<S>(acc, p, row0, f0, 0, p.segments * ((p.K + 127) >> 7), lds);
    const int row = row0 + wave / S::WF * 32 * S::TR, col = f0 + wave % S::WF * 32 * S::FT;
#pragma unroll
    for (int u = 0; u < S::TR; ++u) {
        float sx = 1.f;
        if constexpr (S::E4M3) {
            const int r = row + 32 * u + (lane & 31);
            sx = sc.x[r < h.rows ? r : h.rows - 1];
        }
        const auto gated = [&](int t) {
            f32x16 a;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float g = acc[t][u][i], v = acc[S::FT + t][u][i];
                if constexpr (S::E4M3) {
                    int c = col + 32 * t + acc_feature(i, lane >> 5);
                    c = c < h.cols ? c : h.cols - 1;
                    g *= sx * sc.g[c];
                    v *= sx * sc.u[c];
                }
                a[i] = g * sigmoid<TERMS == 3>(g) * v;
            }
            return a;
        };
        store_rows<S::FT>(lds, gated, [&](int r, int c, const float *v, int) { put_hidden<TERMS>(h, 0, row + 32 * u + r, col + c, v); });
    }
}

// A share of both projections (and, with D, of dy Wd^T): its raw sums, part[split][image][rows][ld] in fp32.
template <typename S, typename D>
__global__ __launch_bounds__(256) void gated_up_share_kernel(GemmProblem p, GemmProblem q, Hidden h, float *__restrict__ part)
{
    extern __shared__ __align__(1024) char lds[];
    constexpr int IMAGES = std::is_void<D>::value ? 2 : 3;
    const TilePlace at = tile_of(blockIdx.x, p.tiles_r, p.tiles_f, p.splits);
    const int row0 = at.r * S::BR, f0 = at.f * S::BF, wave = threadIdx.x >> 6;
    const int row = row0 + wave / S::WF * 32 * S::TR, col = f0 + wave % S::WF * 32 * S::FT;
    const auto put = [&](int image) {
        const Out o = {part + (size_t)(IMAGES * at.split + image) * h.rows * h.ld, nullptr, h.rows, h.ld, 1};
        return [=](int u) { return [=](int r, int c, const float *v, int) { put_out(o, row + 32 * u + r, col + c, v); }; };
    };
    int s0, s1;
    {
        f32x16 acc[S::TF][S::TR];
        clear<S>(acc);
        share_of(p, at.split, s0, s1);
        mma_steps<S>(acc, p, row0, f0, s0, s1, lds);
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int u = 0; u < S::TR; ++u) store_rows<S::FT>(lds, [&](int t) { return acc[m * S::FT + t][u]; }, put(m)(u));
    }
    if constexpr (IMAGES == 3) {
        lds_barrier();   // the sums have left the LDS
        f32x16 acc[D::TF][D::TR];
        clear<D>(acc);
        share_of(q, at.split, s0, s1);
        mma_steps<D>(acc, q, row0, f0, s0, s1, lds);
#pragma unroll
        for (int u = 0; u < D::TR; ++u) store_rows<D::TF>(lds, [&](int t) { return acc[t][u]; }, put(2)(u));
    }
}

// a (and dg, du) from the shares' sums.
template <int TERMS, bool E4M3, int IMAGES>
__global__ __launch_bounds__(256) void gated_up_sum_kernel(const float *__restrict__ part, Hidden h, Scales sc, int splits)
{
    const int per_row = (h.cols + 7) / 8;
    const long long n = (long long)h.rows * per_row;
    const size_t one = (size_t)h.rows * h.ld;
    for (long long k = (long long)blockIdx.x * 256 + threadIdx.x; k < n; k += (long long)gridDim.x * 256) {
        const int row = (int)(k / per_row), col = (int)(k - (long long)row * per_row) * 8;
        float v[IMAGES][8];
#pragma unroll
        for (int m = 0; m < IMAGES; ++m)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[m][i] = 0.f;
        const float *q = part + (size_t)row * h.ld + col;
        for (int s = 0; s < splits; ++s, q += IMAGES * one)
#pragma unroll
            for (int m = 0; m < IMAGES; ++m) {
                const f32x4 a = *(const f32x4 *)(q + m * one), b = *(const f32x4 *)(q + m * one + 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[m][e] += a[e];
                    v[m][4 + e] += b[e];
                }
            }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float g = v[0][i], u = v[1][i];
            if constexpr (E4M3) {
                const int c = col + i < h.cols ? col + i : h.cols - 1;
                g *= sc.x[row] * sc.g[c];
                u *= sc.x[row] * sc.u[c];
            }
            const float sg = sigmoid<TERMS >= 3>(g), s = g * sg;
            v[0][i] = s * u;
            if constexpr (IMAGES == 3) {
                const float d = v[2][i];
                v[1][i] = d * u * (sg + s * (1.f - sg));
                v[2][i] = d * s;
            }
        }
#pragma unroll
        for (int m = 0; m < (IMAGES == 3 ? 3 : 1); ++m) put_hidden<TERMS>(h, m, row, col, v[m]);
    }
}

// The same for few rows: bound by the weights' arrival (T 16, d 4096, H 11008 in 8 bits: 90 MB in 23 us; T 32, d 1024, H 2816 in bf16: 8 us,
// two round trips and the launch).  Against 128-feature tiles whose contraction was shared out over blocks and added up by a second kernel:
// 24 and 12 us.
template <typename S> __global__ __launch_bounds__(256) void gated_up_few_kernel(GemmProblem p, Hidden h, Scales sc)
{
    extern __shared__ __align__(1024) char lds[];
    const TilePlace at = tile_of(blockIdx.x, p.tiles_r, p.tiles_f, 1);
    const int row0 = at.r * S::BR, f0 = at.f * S::BF;
    few_rows<S>(p, row0, f0, 0, p.segments * ((p.K + 127) >> 7), lds, [&](int r, int c, const float (&v)[2][8]) {
        const int row = row0 + r, col = f0 + c;
        if (row >= h.rows) return;
        float a[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float g = v[0][i], u = v[1][i];
            if constexpr (S::E4M3) {
                const int k = col + i < h.cols ? col + i : h.cols - 1;
                g *= sc.x[row] * sc.g[k];
                u *= sc.x[row] * sc.u[k];
            }
            a[i] = g * sigmoid<false>(g) * u;
        }
        put_hidden<1>(h, 0, row, col, a);
    });
}

// Up to three products in one launch (the weight gradients: together they fill the chip where each alone would not), into their
// outputs or, with a split contraction, into fp32 shares.
struct Products {
    GemmProblem p[3];
    Out out[3];
    float *part[3];      // [split][rows][ld], ld = cols rounded up to 8; none without a split
    int first[4];        // first block of each
};
template <typename S> __global__ __launch_bounds__(256) void gated_product_kernel(Products ps)
{
    extern __shared__ __align__(1024) char lds[];
    int k = 0;
    while (k < 2 && (int)blockIdx.x >= ps.first[k + 1]) ++k;
    const GemmProblem &p = ps.p[k];
    const TilePlace at = tile_of(blockIdx.x - ps.first[k], p.tiles_r, p.tiles_f, p.splits);
    const int row0 = at.r * S::BR, f0 = at.f * S::BF, wave = threadIdx.x >> 6;
    const int row = row0 + wave / S::WF * 32 * S::TR, col = f0 + wave % S::WF * 32 * S::TF, lane = threadIdx.x & 63;
    Out o = ps.out[k];
    if (ps.part[k]) {
        const int ld = (o.cols + 7) & ~7;
        o = {ps.part[k] + (size_t)at.split * o.rows * ld, nullptr, o.rows, ld, 1};
    }
    f32x16 acc[S::TF][S::TR];
    clear<S>(acc);
    int s0, s1;
    share_of(p, at.split, s0, s1);
    mma_steps<S>(acc, p, row0, f0, s0, s1, lds);
    // the addend of 32 rows is requested while those before them are stored (piece by piece each would wait for its own: 32 waits)
    constexpr int PIECES = 4 * S::TF, MINE = PIECES / 2;
    Addend next[MINE], now[MINE];
    const auto fetch = [&](int u) {
#pragma unroll
        for (int i = 0; i < MINE; ++i) next[i] = fetch_addend(o, row + 32 * u + (i * 64 + lane) / PIECES, col + (i * 64 + lane) % PIECES * 8);
    };
    fetch(0);
#pragma unroll
    for (int u = 0; u < S::TR; ++u) {
#pragma unroll
        for (int i = 0; i < MINE; ++i) now[i] = next[i];
        if (u + 1 < S::TR) fetch(u + 1);
        store_rows<S::TF>(lds, [&](int t) { return acc[t][u]; }, [&](int r, int c, const float *v, int i) { put_out(o, row + 32 * u + r, col + c, v, now[i]); });
    }
}

template <typename S> __global__ __launch_bounds__(256) void gated_product_few_kernel(Products ps)
{
    extern __shared__ __align__(1024) char lds[];
    const GemmProblem &p = ps.p[0];
    const TilePlace at = tile_of(blockIdx.x, p.tiles_r, p.tiles_f, p.splits);
    const int row0 = at.r * S::BR, f0 = at.f * S::BF;
    int s0, s1;
    share_of(p, at.split, s0, s1);
    Out o = ps.out[0];
    if (ps.part[0]) {
        const int ld = (o.cols + 7) & ~7;
        o = {ps.part[0] + (size_t)at.split * o.rows * ld, nullptr, o.rows, ld, 1};
    }
    few_rows<S>(p, row0, f0, s0, s1, lds, [&](int r, int c, const float (&v)[1][8]) { put_out(o, row0 + r, f0 + c, v[0]); });
}

// fp32 with few rows: part[split][image][rows][ldp] = x W for one or two matrices [K][N] (K-major) or [N][K] (K-contiguous), on the fp32
// matrix instruction, which reads the weights where they are (laid out as terms first they cross memory twice more).  It takes one value
// of k per lane, so a lane's 16 bytes of a row of K-major W are four feature tiles (tile t has the features 4 i + t of the block's 128; of
// K-contiguous W 32 t + i, from four rows) and its 16 bytes of a row of x four instructions: nothing passes through the LDS but the four wavefronts' sums.  A wavefront takes 32 values of k in turn with the
// others (a cache line of x), eight at a time, the next three eights on their way.
//
// Bound by memory up to 32 rows: d 4096, H 11008 (541 MB of weights), the whole forward 123 us for one row, 128 for 22 (4.2 TB/s); as terms
// 574 and 587.  Above by the fp32 matrix instruction, where the terms' copies still cost more: 64 rows 200 against 615, 128 357 against
// 652, 256 674 against 675; d 1024, H 2816: 22 rows 25 against 53, 128 44 against 62, 256 66 against 73.  Tiles of 64 rows read the
// weights half as often and fill the chip worse: 22 rows 183, 64 202, 256 622.  The backward's K-contiguous products run at 2.1 TB/s, the
// K-major ones at 4.6 (one row: 172 us for 360 MB against 78); the 128 bytes of a row requested at once instead of eight by eight: 3%
// worse at d 4096, 2% better at d 1024.
struct FewF32 {
    const float *x[2];
    const float *w[2];
    float *part;
    int rows, K, N, ldx, ldp;
    int images, first, of;   // images here, which of part's `of` images the first of them is
    int splits, tiles_r, tiles_f;
};
template <int FL> __global__ __launch_bounds__(256) void gated_few_f32_kernel(FewF32 a)
{
    constexpr int SLOTS = 4;
    __shared__ __align__(16) float sums[4][32][128];   // piece p of row r (four features) at place p ^ r: no bank conflicts
    const TilePlace at = tile_of(blockIdx.x, a.tiles_r, a.tiles_f * a.images, a.splits);
    const int image = at.f / a.tiles_f, f0 = (at.f - image * a.tiles_f) * 128, row0 = at.r * 32;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 31, half = lane >> 5, col = f0 + 4 * i;
    const float *w = image ? a.w[1] : a.w[0];
    const float *x = (image ? a.x[1] : a.x[0]) + (size_t)(row0 + i < a.rows ? row0 + i : a.rows - 1) * a.ldx;
    f32x16 acc[4];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[t][r] = 0.f;

    // whole eights of k, those of the share [g0, g1); the wavefront's n-th is eight_of(n)
    const int eights = a.K >> 3, each = (eights + a.splits - 1) / a.splits, g0 = at.split * each, g1 = g0 + each < eights ? g0 + each : eights;
    const int share = g1 > g0 ? g1 - g0 : 0, rest = (share & 15) - 4 * wave;
    const int n = (share >> 4) * 4 + (rest < 0 ? 0 : rest > 4 ? 4 : rest);
    const auto eight_of = [&](int k) { return g0 + (k >> 2) * 16 + wave * 4 + (k & 3); };
    const auto run = [&](auto edge) {
        const float *wr[4];   // K-contiguous: the lane's rows
        if constexpr (FL == kKContiguous)
#pragma unroll
            for (int t = 0; t < 4; ++t) wr[t] = w + (size_t)(f0 + 32 * t + i < a.N ? f0 + 32 * t + i : a.N - 1) * a.K;
        const auto load_w = [&](int k) -> f32x4 {   // K-major, k < K
            const float *q = w + (size_t)k * a.N;
            if (!decltype(edge)::value || col + 4 <= a.N) return __builtin_bit_cast(f32x4, *(const loose *)(q + col));
            f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (col + e < a.N) v[e] = q[col + e];
            return v;
        };
        f32x4 wv[SLOTS][4], xv[SLOTS];
        const auto request = [&](int slot, int k) {
            const int k0 = 8 * eight_of(k) + 4 * half;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (FL == kKMajor) wv[slot][j] = load_w(k0 + j);
                else wv[slot][j] = __builtin_bit_cast(f32x4, *(const loose *)(wr[j] + k0));
            }
            xv[slot] = __builtin_bit_cast(f32x4, *(const loose *)(x + k0));
        };
        const auto multiply = [&](int slot) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int t = 0; t < 4; ++t)
                    acc[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(FL == kKMajor ? wv[slot][j][t] : wv[slot][t][j], xv[slot][j], acc[t], 0, 0, 0);
        };
#pragma unroll
        for (int k = 0; k < SLOTS; ++k)
            if (k < n) request(k, k);
        int k = 0;
        for (; k + 2 * SLOTS <= n; k += SLOTS)
#pragma unroll
            for (int c = 0; c < SLOTS; ++c) {
                multiply(c);
                request(c, k + SLOTS + c);
            }
#pragma unroll
        for (int c = 0; c < 2 * SLOTS - 1; ++c)
            if (k + c < n) {
                multiply(c % SLOTS);
                if (c < SLOTS && k + SLOTS + c < n) request(c % SLOTS, k + SLOTS + c);
            }
        // what is left of k: the last share's first wavefront, zeros past the end in both operands
        if ((a.K & 7) && at.split == a.splits - 1 && wave == 0) {
            const int k0 = 8 * eights + 4 * half;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool there = k0 + j < a.K;
                if constexpr (FL == kKMajor) wv[0][j] = there ? load_w(k0 + j) : f32x4{0.f, 0.f, 0.f, 0.f};
                else
#pragma unroll
                    for (int t = 0; t < 4; ++t) wv[0][t][j] = there ? wr[t][k0 + j] : 0.f;
                xv[0][j] = there ? x[k0 + j] : 0.f;
            }
            multiply(0);
        }
    };
    if (FL == kKContiguous || f0 + 128 <= a.N) run(std::false_type());
    else run(std::true_type());

    float *out = a.part + (size_t)(at.split * a.of + a.first + image) * a.rows * a.ldp;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        if constexpr (FL == kKMajor) *(f32x4 *)&sums[wave][i][4 * (acc_feature(r, half) ^ i)] = f32x4{acc[0][r], acc[1][r], acc[2][r], acc[3][r]};
        else {
            const f32x16 &v = acc[r >> 2];   // quarter r % 4 of its tile
            const int q = r & 3;
            *(f32x4 *)&sums[wave][i][4 * ((8 * (r >> 2) + 2 * q + half) ^ i)] = f32x4{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
        }
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const int piece = c * 256 + (int)threadIdx.x, r = piece >> 5, f = 4 * (piece & 31), place = f ^ 4 * r, row = row0 + r;
        f32x4 v = *(const f32x4 *)&sums[0][r][place];
#pragma unroll
        for (int k = 1; k < 4; ++k) v += *(const f32x4 *)&sums[k][r][place];
        if (row < a.rows && f0 + f < a.ldp) *(f32x4 *)(out + (size_t)row * a.ldp + f0 + f) = v;
    }
}

// Weight gradients of few fp32 rows (d 4096, H 11008: 541 MB in 84 us for one row, 234 for 64): out[r][f] = sum over t of l[t][r] m[t][f], three of them.  A wavefront has 32 of r and 128 of f: the
// features are the matrix instruction's second operand, so a lane holds four neighbours of a row and stores go out as rows.  Bound
// by the outputs' way to memory, from some 64 rows on by the instruction; l and m are small and come from the caches.
struct FewF32Weights {
    const float *l[3], *m[3];
    float *out[3];
    int nr[3], nf[3], ldl[3], ldm[3];
    int rows;
};
__global__ __launch_bounds__(256) void gated_few_f32_weights_kernel(FewF32Weights a)
{
    const int k = blockIdx.y, nr = a.nr[k], nf = a.nf[k], tiles_f = (nf + 127) / 128, tile = blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 31, half = lane >> 5;
    const int row0 = (tile / tiles_f * 4 + wave) * 32, col = tile % tiles_f * 128 + 4 * i;
    if (row0 >= nr) return;   // (a whole wavefront; there is no barrier)
    const float *l = a.l[k] + (row0 + i < nr ? row0 + i : nr - 1), *m = a.m[k];
    const size_t ldl = a.ldl[k], ldm = a.ldm[k];
    f32x16 acc[4];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[t][r] = 0.f;
    for (int t0 = 4 * half; t0 - 4 * half < a.rows; t0 += 8) {
        float lv[4];
        f32x4 mv[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int t = t0 + j;
            lv[j] = 0.f;
            mv[j] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (t >= a.rows) continue;
            lv[j] = l[t * ldl];
            if (col + 4 <= nf) mv[j] = __builtin_bit_cast(f32x4, *(const loose *)(m + t * ldm + col));
            else
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (col + e < nf) mv[j][e] = m[t * ldm + col + e];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int t = 0; t < 4; ++t) acc[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(lv[j], mv[j][t], acc[t], 0, 0, 0);
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int row = row0 + acc_feature(r, half);
        if (row >= nr) continue;
        float *q = a.out[k] + (size_t)row * nf + col;
        const f32x4 v = {acc[0][r], acc[1][r], acc[2][r], acc[3][r]};
        if (col + 4 <= nf) *(loose *)q = __builtin_bit_cast(u32x4, v);
        else
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (col + e < nf) q[e] = v[e];
    }
}

// The shares' sums, in their order within each of GROUPS groups (neighbours in a block; more of them where there are many shares of few
// outputs), then the groups'.
template <int GROUPS> __global__ __launch_bounds__(256) void gated_sum_kernel(Products ps)
{
    constexpr int PIECES = 256 / GROUPS;
    __shared__ float sums[GROUPS > 1 ? GROUPS : 1][GROUPS > 1 ? PIECES : 1][8];
    const int k = blockIdx.y, group = threadIdx.x / PIECES, lane = threadIdx.x % PIECES;
    if (!ps.part[k]) return;
    const Out o = ps.out[k];
    const int per_row = (o.cols + 7) / 8, ld = per_row * 8, splits = ps.p[k].splits;
    const long long n = (long long)o.rows * per_row;
    const size_t one = (size_t)o.rows * ld;
    for (long long base = (long long)blockIdx.x * PIECES; base < n; base += (long long)gridDim.x * PIECES) {
        const long long i = base + lane;
        const bool there = i < n;
        const int row = there ? (int)(i / per_row) : 0, col = there ? (int)(i - (long long)row * per_row) * 8 : 0;
        const float *q = ps.part[k] + (size_t)row * ld + col + group * one;
        f32x4 a = {0.f, 0.f, 0.f, 0.f}, b = a;
        for (int s = group; s < splits; s += GROUPS, q += GROUPS * one) {
            a += *(const f32x4 *)q;
            b += *(const f32x4 *)(q + 4);
        }
        if constexpr (GROUPS > 1) {
            __syncthreads();   // the last round's sums have been read
            *(f32x4 *)&sums[group][lane][0] = a;
            *(f32x4 *)&sums[group][lane][4] = b;
            __syncthreads();
            if (group > 0) continue;
#pragma unroll
            for (int g = 1; g < GROUPS; ++g) {
                a += *(const f32x4 *)&sums[g][lane][0];
                b += *(const f32x4 *)&sums[g][lane][4];
            }
        }
        const float v[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
        if (there) put_out(o, row, col, v);
    }
}

// Backward of the gate: both projections again, da beside them, and a, dg, du.  S: as gated_up_kernel; D: the same rows and features
// of dy Wd^T.  Half of its time at small d is the epilogue, three outputs at once (T 8191, d 768, H 2048: 54 us a round, 30 of them steps).
template <typename S, typename D, int TERMS>
__global__ __launch_bounds__(256) void gated_up_backward_kernel(GemmProblem p, GemmProblem q, Hidden h)
{
    static_assert(S::BR == D::BR && S::BF == D::BF && S::FT == D::TF && S::WF == D::WF, "one tile");
    extern __shared__ __align__(1024) char lds[];
    const TilePlace at = tile_of(blockIdx.x, p.tiles_r, p.tiles_f, 1);
    const int row0 = at.r * S::BR, f0 = at.f * S::BF, wave = threadIdx.x >> 6;
    f32x16 acc[S::TF][S::TR], da[D::TF][D::TR];
    clear<S>(acc);
    clear<D>(da);
    mma_steps<S>(acc, p, row0, f0, 0, p.segments * ((p.K + 127) >> 7), lds);
    mma_steps<D>(da, q, row0, f0, 0, q.segments * ((q.K + 127) >> 7), lds);
    const int row = row0 + wave / S::WF * 32 * S::TR, col = f0 + wave % S::WF * 32 * S::FT;
#pragma unroll
    for (int u = 0; u < S::TR; ++u) {
        const auto put = [&](int which) { return [&, which](int r, int c, const float *v, int) { put_hidden<TERMS>(h, which, row + 32 * u + r, col + c, v); }; };
        const auto first = [&](int t) {   // a; acc and da become dg and du
            f32x16 a;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float g = acc[t][u][i], v = acc[S::FT + t][u][i], d = da[t][u][i], sg = sigmoid<TERMS == 3>(g), s = g * sg;
                a[i] = s * v;
                acc[t][u][i] = d * v * (sg + s * (1.f - sg));
                da[t][u][i] = d * s;
            }
            return a;
        };
        store_rows<S::FT>(lds, first, put(0));
        store_rows<S::FT>(lds, [&](int t) { return acc[t][u]; }, put(1));
        store_rows<S::FT>(lds, [&](int t) { return da[t][u]; }, put(2));
    }
}

// ---- weights in e4m3 -----------------------------------------------------------------------------------------------------
// Column h of W [d][H] becomes row h of the copy, with the scale of its largest value.  A block takes 32 columns: once for the
// largest values, once more (from the cache) for the values, which turn in the LDS.  Done once for a set of weights: d 4096, H 11008 344 us,
// d 1024, H 2816 38 us; 64-byte pieces of W's rows and few blocks keep it at 0.2 to 1.6 TB/s.
__global__ __launch_bounds__(256) void gated_quantize_kernel(const bf16_t *__restrict__ Wg, const bf16_t *__restrict__ Wu, uint8_t *__restrict__ Qg,
                                                             uint8_t *__restrict__ Qu, float *__restrict__ sg, float *__restrict__ su, int d, int H)
{
    const bf16_t *W = blockIdx.y ? Wu : Wg;
    uint8_t *Q = blockIdx.y ? Qu : Qg;
    float *scales = blockIdx.y ? su : sg;
    __shared__ uint32_t top[8][32];
    __shared__ float tile[64][33];
    const int c = threadIdx.x & 31, y = threadIdx.x >> 5, col = blockIdx.x * 32 + c;
    uint32_t most = 0;
    if (col < H)
        for (int k = y; k < d; k += 8) {
            const uint32_t a = (uint32_t)(W[(size_t)k * H + col] & 0x7fff) << 16;
            most = a > most ? a : most;
        }
    top[y][c] = most;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) most = top[i][c] > most ? top[i][c] : most;
    const float t = __uint_as_float(most);
    float scale = (t < kE4m3Floor ? kE4m3Floor : t) / kE4m3Max;
    if (most >= 0x7f800000u) scale = __uint_as_float(0x7fc00000u);
    if (y == 0 && col < H) scales[col] = scale;
    const float inv = 1.f / scale;
    for (int k0 = 0; k0 < d; k0 += 64) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int k = k0 + y + 8 * i;
            tile[y + 8 * i][c] = k < d && col < H ? bf16_to_f32(W[(size_t)k * H + col]) * inv : 0.f;
        }
        __syncthreads();
        // 32 rows of 64 values: 16 threads of four values per row
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int r = i * 16 + (threadIdx.x >> 4), k = (threadIdx.x & 15) * 4, h = blockIdx.x * 32 + r;
            if (h < H && k0 + k < d)   // (d is a multiple of 16)
                *(uint32_t *)(Q + (size_t)h * d + k0 + k) = pack_e4m3(tile[k][r], tile[k + 1][r], tile[k + 2][r], tile[k + 3][r]);
        }
    }
}

// ---- host ----------------------------------------------------------------------------------------------------------------
// Tile shapes.  Big: 256 rows x 256 features (gate and up: 128 of each) and Wide: 256 x 128, one block per CU.  Middle: 128 x 128,
// two blocks per CU.  For the few rows of a decoding step: see FewShape.
template <int RL, int FL, bool DUAL, bool E4M3> struct Shapes {
    typedef TileShape<4, 4, 2, 2, RL, FL, DUAL, E4M3, 3, 2> Big;
    typedef TileShape<4, 2, 2, 2, RL, FL, DUAL, E4M3, 3, 2> Wide;
    typedef TileShape<2, 2, 2, 2, RL, FL, DUAL, E4M3, 3, 2> Middle;
};
template <typename S> constexpr int lds_of(int staged_tiles) { return S::LDS > stage_bytes(staged_tiles) ? S::LDS : stage_bytes(staged_tiles); }

static int ceil_div(long long a, long long b) { return (int)((a + b - 1) / b); }
static int steps_of(const GemmProblem &p) { return p.segments * ((p.K + 127) >> 7); }

enum TileSize { kBig, kWide, kMiddle, kFew };
constexpr int kFewRows = 64;   // up to these many rows of x take the kernels for few rows
constexpr int kFewRowsF32 = 256;   // the forward pass of up to these many fp32 rows multiplies fp32 values as they are (gated_few_f32_kernel),
// the backward pass up to these (both passes together, as they are against terms: d 4096, H 11008, 64 rows 892 against 1322, 128 rows 1487
// against 1620; d 1024, H 2816, 64 rows 114 against 136, 128 rows 165 against 159; d 1001, H 3001, 100 rows 211 against 192)
constexpr int kFewRowsF32Backward = 64;
struct TileChoice {
    TileSize size;
    int splits;   // shares of the contraction, so that few tiles fill the chip
};
// The fewest steps of a share: the ring's first round trip and the sums' way through memory do not pay for less.
constexpr int kLeastShare = 4;
static int most_shares(long long tiles, long long slots, int steps)
{
    return (int)std::max<long long>(1, std::min<long long>(slots / std::max(1ll, tiles), steps / kLeastShare));
}
static int whole_shares(int steps, int n) { return steps == 0 ? 1 : ceil_div(steps, ceil_div(steps, n)); }   // no empty ones

// What the choice goes by, in us, fitted to kernel traces of the three sizes on the same products: a step of a tile that has its CU to
// itself and of one that shares it, the rest of a round of tiles (launch, first round trip, epilogue), and for shares the launch of
// their addition and their way through memory.  (T 8191, d 768, H 2048, big / wide / middle: up 61 / 71 / 70, down in two shares
// 75 / 48 / 44, dx 86 / 71 / 67, weights in three shares 101 / 105 / 108; T 8192, d 4096, H 11008: up 1070 / 1276 / 1383, weights
// 1712 / 1889 / 2759, dx 1040 / 1313 / 1514; fp32, T 1000, d 256, H 683: up 45 / 27 / 18.)  Batches of 65 to some 2000 bf16 rows were not
// among them.
struct TileCost {
    int rows, features, slots;   // slots: tiles per CU
    double alone, shared, rest;
};
constexpr TileCost kCosts[3] = {{256, 256, 1, 1.5, 1.5, 10}, {256, 128, 1, 0.95, 0.95, 8}, {128, 128, 2, 0.6, 1.0, 6}};
constexpr double kSumLaunch = 6, kSumPerMB = 0.15;
// n products of nr x nf outputs and `steps` steps each.  dual: both projections in a tile (2), and dy Wd^T after them (3).
static TileChoice choose_tiles(long long nr, long long nf, int steps, int dual, bool may_split, int n = 1)
{
    const int cus = num_compute_units();
    if (nr <= kFewRows && n == 1) return {kFew, may_split ? whole_shares(steps, most_shares(ceil_div(nf, 64), cus, steps)) : 1};
    TileChoice best = {kBig, 1};
    double least = 0;
    for (int k = 0; k < 3; ++k) {
        const TileCost &c = kCosts[k];
        const long long slots = (long long)c.slots * cus, tiles = (long long)n * ceil_div(nr, c.rows) * ceil_div(dual ? 2 * nf : nf, c.features), sums = n * nr * nf * (dual ? dual : 1);
        const int most = may_split ? most_shares(tiles, slots, steps) : 1;
        for (int m = 1; m <= most; ++m) {
            const int splits = whole_shares(steps, m);
            double cost = ceil_div(tiles * splits, slots) * (ceil_div(steps, splits) * (tiles * splits <= cus ? c.alone : c.shared) + c.rest);
            if (splits > 1) cost += kSumLaunch + kSumPerMB * 4e-6 * splits * sums;
            if (least == 0 || cost < least) {
                least = cost;
                best = {(TileSize)k, splits};
            }
        }
    }
    return best;
}
// Bytes of the shares' sums, at most: shares fill the chip at most once (slots x a tile), and none is shorter than its least.  Neither
// bound falls as T grows, so a workspace made for the largest batch takes every smaller one.
static size_t share_bytes(long long slots, long long tile, int steps, size_t rows, size_t ld)
{
    return (size_t)std::min<long long>(slots * tile * 4, (long long)(steps / kLeastShare) * rows * ld * 4);
}
template <typename S> static void set_tiles(GemmProblem &p, int splits)
{
    p.tiles_r = ceil_div(p.nr, S::BR);
    p.tiles_f = ceil_div(p.nf, S::BF);
    p.splits = splits;
}

static size_t padded(int n) { return ((size_t)n + 63) / 64 * 64; }

// Contractions of a call's products that may be shared out, in steps.
struct CallSteps {
    int up, down, dx, dw;
};
static CallSteps call_steps(const slicemoe_gated_config &c, int terms, bool e4m3)
{
    const int pairs = terms == 3 ? kPairs : 1;
    const auto steps = [](long long bytes) { return (int)((bytes + 127) / 128); };
    CallSteps s;
    s.up = pairs * steps(e4m3 ? c.d : 2ll * c.d);
    s.down = pairs * steps(2ll * c.H);
    s.dx = 2 * s.down;
    s.dw = pairs * steps(2ll * c.T);
    return s;
}

// fp32 with few rows: shares of each product.  In us: 0.027 per value of k of a block's 128 features (512 bytes of its CU's part of the
// memory's rate), the rest of a block, and the way of the sums through memory.
constexpr double kF32PerK = 0.027, kF32Rest = 2;   // (a rest of 4: 64 rows of d 1024 31 instead of 33, 33 rows of d 1001, H 3001 58 instead of 51)
constexpr int kF32Tile = 32, kF32Most = 4;         // rows of a tile; tiles per CU at most
static int few_f32_splits(int rows, int images, int K, int N)
{
    const int cus = num_compute_units();
    const long long tiles = (long long)images * ceil_div(rows, kF32Tile) * ceil_div(N, 128);
    const int most = (int)std::max<long long>(1, std::min<long long>(kF32Most * cus / tiles, K / 128));
    int best = 1;
    double least = 0;
    for (int n = 1; n <= most; ++n) {
        const double cost = ceil_div(tiles * n, cus) * (kF32PerK * K / n + kF32Rest) + kSumPerMB * 4e-6 * n * images * rows * N;
        if (n == 1 || cost < least) {
            least = cost;
            best = n;
        }
    }
    return best;
}

GatedPlan gated_plan(const slicemoe_gated_config &c, bool backward, bool quantized)
{
    GatedPlan p = {};
    if (c.dtype != SLICEMOE_BF16 && c.T <= (backward ? kFewRowsF32Backward : kFewRowsF32)) {   // the hidden rows as fp32, and the shares
        p.few_f32 = true;
        p.ldh = (int)padded(c.H);
        const size_t hidden = align_up((size_t)c.T * p.ldh * 4, 256);
        p.dg = hidden;   // (after a, at the beginning)
        p.du = 2 * hidden;
        p.part = (backward ? 3 : 1) * hidden;
        // at most; neither bound falls as T grows
        const auto shares = [&](int images, int K, int N, int ld) {
            const size_t room = (size_t)c.T * images * ld * 4, least = std::max(1, K / 128);
            return std::max(room, std::min<size_t>((size_t)kF32Most * num_compute_units() * kF32Tile * 128 * 4, least * room));
        };
        const int d8 = (c.d + 7) / 8 * 8;
        const size_t part = backward ? std::max(shares(3, c.d, c.H, p.ldh), shares(2, c.H, c.d, d8)) : std::max(shares(2, c.d, c.H, p.ldh), shares(1, c.H, c.d, d8));
        p.total = std::max<size_t>(256, align_up(p.part + part, 256));
        return p;
    }
    const size_t T = c.T, d = c.d, H = c.H;
    p.terms = c.dtype == SLICEMOE_BF16 ? 1 : 3;
    p.copy_x = c.dtype != SLICEMOE_BF16 || c.d % 8 != 0;
    p.copy_h = c.dtype != SLICEMOE_BF16 || c.H % 8 != 0;
    p.ldd = (int)(p.copy_x ? padded(c.d) : d);
    p.ldh = (int)padded(c.H);
    size_t at = 0;
    const auto take = [&](size_t bytes) {
        const size_t was = at;
        at = align_up(at + bytes, 256);
        return was;
    };
    const size_t t2 = 2 * (size_t)p.terms;
    p.x = take(p.copy_x && !quantized ? t2 * T * p.ldd : 0);
    p.dy = take(p.copy_x && backward ? t2 * T * p.ldd : 0);
    p.Wg = take(p.copy_h && !quantized ? t2 * d * p.ldh : 0);
    p.Wu = take(p.copy_h && !quantized ? t2 * d * p.ldh : 0);
    p.Wd = take(p.copy_x ? t2 * H * p.ldd : 0);
    p.a = take(t2 * T * p.ldh);
    p.dg = take(backward ? t2 * T * p.ldh : 0);
    p.du = take(backward ? t2 * T * p.ldh : 0);
    const CallSteps st = call_steps(c, p.terms, quantized);
    const size_t d8 = (d + 7) / 8 * 8, h8 = (H + 7) / 8 * 8, few = std::min<size_t>(T, kFewRows);
    const long long cus = num_compute_units();
    // (tiles reach past the outputs' edges; what is stored ends there, so the outputs bound the bytes of the first kind too)
    const auto rows_shares = [&](int steps) {
        return std::max(share_bytes(cus, kFewRows * 64, steps, few, d8), T > few ? share_bytes(cus, 256 * 256, steps, T, d8) : 0);
    };
    size_t part = 0;
    const auto up_shares = [&](int steps, int images) { return share_bytes(cus, images * 256 * 128, steps, T, images * (size_t)p.ldh); };
    if (!backward) part = std::max(rows_shares(st.down), up_shares(st.up, 2));
    else
        part = std::max(std::max(rows_shares(st.dx), up_shares(st.up + st.up / 2, 3)), 3 * 256 + 2 * share_bytes(cus, 256 * 256, st.dw, d, h8) + share_bytes(cus, 256 * 256, st.dw, H, d8));
    p.part = take(part);
    p.total = std::max<size_t>(at, 256);
    if (p.terms == 3) {   // not below what the longest batch of few rows takes
        slicemoe_gated_config few_rows = c;
        few_rows.T = backward ? kFewRowsF32Backward : kFewRowsF32;
        p.total = std::max(p.total, gated_plan(few_rows, backward, false).total);
    }
    return p;
}

// The arrays that the tiles read: the caller's, or the copies.
struct Operands {
    const char *x, *dy, *Wg, *Wu, *Wd;
    size_t tx, tw, twd, th;       // bytes from one term to the next: rows of x and dy, of Wg and Wu, of Wd, of the hidden arrays
    long long ldx, ldw, ldwd, ldh;   // bytes per row
};
static hipError_t make_operands(const slicemoe_gated_config &c, const GatedPlan &p, const void *x, const void *dy, const slicemoe_gated_weights &w,
                                char *ws, Operands *o, hipStream_t s)
{
    o->ldx = o->ldwd = 2ll * (p.copy_x ? p.ldd : c.d);
    o->ldw = 2ll * (p.copy_h ? p.ldh : c.H);
    o->ldh = 2ll * p.ldh;
    o->tx = (size_t)c.T * o->ldx;
    o->tw = (size_t)c.d * o->ldw;
    o->twd = (size_t)c.H * o->ldwd;
    o->th = (size_t)c.T * o->ldh;
    CopyJobs jobs = {};
    jobs.f32 = c.dtype != SLICEMOE_BF16;
    int n = 0;
    const auto operand = [&](const void *src, bool copy, size_t at, int rows, int cols, int ld) -> const char * {
        if (!src || !copy) return (const char *)src;
        jobs.j[n++] = {src, (bf16_t *)(ws + at), rows, cols, ld};
        return ws + at;
    };
    o->x = operand(x, p.copy_x, p.x, c.T, c.d, p.ldd);
    o->dy = operand(dy, p.copy_x, p.dy, c.T, c.d, p.ldd);
    o->Wg = operand(w.Wg, p.copy_h, p.Wg, c.d, c.H, p.ldh);
    o->Wu = operand(w.Wu, p.copy_h, p.Wu, c.d, c.H, p.ldh);
    o->Wd = operand(w.Wd, p.copy_x, p.Wd, c.H, c.d, p.ldd);
    if (n == 0) return hipSuccess;
    long long most = 0;
    for (int i = 0; i < n; ++i) most = std::max(most, (long long)jobs.j[i].rows * (jobs.j[i].ld / 8));
    const int blocks = (int)std::min<long long>((most + 255) / 256, 8ll * num_compute_units());
    gated_copy_kernel<<<dim3(blocks, n), 256, 0, s>>>(jobs);
    return hipGetLastError();
}

// Fills the segments of r f^T: every pair of terms that counts.
static void add_segments(GemmProblem &p, int terms, const char *r, size_t tr, const char *f, size_t tf, const char *f2 = nullptr)
{
    const int pairs = terms == 3 ? kPairs : 1;
    for (int i = 0; i < pairs; ++i) {
        const int k = p.segments++;
        p.r[k] = r + kPairR[i] * tr;
        p.f[k] = f + kPairF[i] * tf;
        p.f2[k] = f2 ? f2 + kPairF[i] * tf : nullptr;
    }
}
static GemmProblem problem(int nr, int nf, long long K, long long ldr, long long ldf)
{
    GemmProblem p = {};
    p.nr = nr;
    p.nf = nf;
    p.K = (int)K;
    p.ldr = ldr;
    p.ldf = ldf;
    return p;
}

template <typename K> static hipError_t ready(K kernel, int lds) { return grant_dynamic_lds((const void *)kernel, lds); }

template <typename S, typename KERNEL> static hipError_t run_up(KERNEL kernel, int lds, GemmProblem p, const Hidden &h, const Scales &sc, hipStream_t s)
{
    set_tiles<S>(p, 1);
    const hipError_t e = ready(kernel, lds);
    if (e != hipSuccess) return e;
    kernel<<<p.tiles_r * p.tiles_f, 256, lds, s>>>(p, h, sc);
    return hipGetLastError();
}
template <typename S, typename D>
static hipError_t run_up_shares(GemmProblem p, GemmProblem q, const Hidden &h, int splits, float *part, hipStream_t s)
{
    set_tiles<S>(p, splits);
    q.splits = splits;
    constexpr int lds = lds_of<S>(S::FT);
    const auto kernel = gated_up_share_kernel<S, D>;
    const hipError_t e = ready(kernel, lds);
    if (e != hipSuccess) return e;
    kernel<<<p.tiles_r * p.tiles_f * splits, 256, lds, s>>>(p, q, h, part);
    return hipGetLastError();
}
template <int TERMS, bool E4M3, int IMAGES>
static hipError_t launch_up_sum(const float *part, const Hidden &h, const Scales &sc, int splits, hipStream_t s)
{
    const long long n = (long long)h.rows * ((h.cols + 7) / 8);
    gated_up_sum_kernel<TERMS, E4M3, IMAGES><<<(int)std::min<long long>((n + 255) / 256, 8ll * num_compute_units()), 256, 0, s>>>(part, h, sc, splits);
    return hipGetLastError();
}
template <int FL, bool E4M3, int TERMS> static hipError_t launch_up(const GemmProblem &p, const Hidden &h, const Scales &sc, float *part, hipStream_t s)
{
    typedef typename Shapes<kKContiguous, FL, true, E4M3>::Big Big;
    typedef typename Shapes<kKContiguous, FL, true, E4M3>::Wide Wide;
    typedef typename Shapes<kKContiguous, FL, true, E4M3>::Middle Middle;
    const TileChoice t = choose_tiles(p.nr, p.nf, steps_of(p), 2, p.nr > kFewRows);
    if (t.splits > 1) {
        const hipError_t e = t.size == kBig    ? run_up_shares<Big, void>(p, p, h, t.splits, part, s)
                             : t.size == kWide ? run_up_shares<Wide, void>(p, p, h, t.splits, part, s)
                                               : run_up_shares<Middle, void>(p, p, h, t.splits, part, s);
        return e == hipSuccess ? launch_up_sum<TERMS, E4M3, 2>(part, h, sc, t.splits, s) : e;
    }
    switch (t.size) {
        case kBig: return run_up<Big>(gated_up_kernel<Big, TERMS>, lds_of<Big>(Big::FT), p, h, sc, s);
        case kWide: return run_up<Wide>(gated_up_kernel<Wide, TERMS>, lds_of<Wide>(Wide::FT), p, h, sc, s);
        case kMiddle: return run_up<Middle>(gated_up_kernel<Middle, TERMS>, lds_of<Middle>(Middle::FT), p, h, sc, s);
        default: break;
    }
    if constexpr (TERMS == 3) return hipErrorInvalidValue;   // (fp32 with few rows: see launch_few_f32)
    else {
        const auto few = [&](auto shape) {
            typedef decltype(shape) S;
            return run_up<S>(gated_up_few_kernel<S>, S::LDS, p, h, sc, s);
        };
        // 64 features a block in bf16, two blocks per CU in 8 bits, where tiles of 32 features are more than the CUs; else the other form, on
        // more of them.  (The call, T 8, d 4096, H 8192, then 8256, this form / the other, us: bf16 58.7 / 55.6, 49.6 / 57.3; 8 bits 32.2 / 32.0,
        // 34.2 / 38.3; T 64: bf16 67.9 / 62.5, 60.3 / 68.3; H 2816 and 16384 of bf16: 43.0 / 39.9, 89.2 / 104.8.)
        const bool many = ceil_div(p.nf, 32) > num_compute_units();
        if constexpr (E4M3) {
            if (p.nr <= 32) return many ? few(FewShape<1, 1, FL, true, true, 2>()) : few(FewShape<1, 1, FL, true, true, 1>());
            return many ? few(FewShape<2, 1, FL, true, true, 2>()) : few(FewShape<2, 1, FL, true, true, 1>());
        } else {
            if (p.nr <= 32) return many ? few(FewShape<1, 2, FL, true, false, 1>()) : few(FewShape<1, 1, FL, true, false, 1>());
            return many ? few(FewShape<2, 2, FL, true, false, 1>()) : few(FewShape<2, 1, FL, true, false, 1>());
        }
    }
}

template <typename S, typename KERNEL> static hipError_t run_products(KERNEL kernel, int lds, Products &ps, int n, hipStream_t s)
{
    ps.first[0] = 0;
    for (int i = 0; i < 3; ++i) {
        if (i < n) set_tiles<S>(ps.p[i], ps.p[i].splits);
        ps.first[i + 1] = ps.first[i] + (i < n ? ps.p[i].tiles_r * ps.p[i].tiles_f * ps.p[i].splits : 0);
    }
    const hipError_t e = ready(kernel, lds);
    if (e != hipSuccess) return e;
    kernel<<<ps.first[n], 256, lds, s>>>(ps);
    return hipGetLastError();
}
// The sums of n products' shares; pieces: eight outputs each, of the largest.
static hipError_t launch_sum(const Products &ps, int n, long long pieces, int splits, hipStream_t s)
{
    if (splits >= 4) gated_sum_kernel<8><<<dim3((int)std::min<long long>((pieces + 31) / 32, 16ll * num_compute_units()), n), 256, 0, s>>>(ps);
    else gated_sum_kernel<1><<<dim3((int)std::min<long long>((pieces + 255) / 256, 8ll * num_compute_units()), n), 256, 0, s>>>(ps);
    return hipGetLastError();
}
// n products of one tile size (few rows: one product, R K-contiguous); part: room for the shares.
template <int RL, int FL> static hipError_t launch_products(Products &ps, int n, TileChoice t, char *part, hipStream_t s)
{
    typedef typename Shapes<RL, FL, false, false>::Big Big;
    typedef typename Shapes<RL, FL, false, false>::Wide Wide;
    typedef typename Shapes<RL, FL, false, false>::Middle Middle;
    long long most = 0;
    size_t at = 0;
    for (int i = 0; i < n; ++i) {
        ps.p[i].splits = t.splits;
        ps.part[i] = nullptr;
        if (t.splits == 1) continue;
        const long long pieces = (long long)ps.out[i].rows * ((ps.out[i].cols + 7) / 8);
        ps.part[i] = (float *)(part + at);
        at = align_up(at + (size_t)t.splits * pieces * 32, 256);
        most = std::max(most, pieces);
    }
    for (int i = n; i < 3; ++i) ps.part[i] = nullptr;
    hipError_t e;
    if (t.size == kBig) e = run_products<Big>(gated_product_kernel<Big>, lds_of<Big>(Big::TF), ps, n, s);
    else if (t.size == kWide) e = run_products<Wide>(gated_product_kernel<Wide>, lds_of<Wide>(Wide::TF), ps, n, s);
    else if (t.size == kMiddle) e = run_products<Middle>(gated_product_kernel<Middle>, lds_of<Middle>(Middle::TF), ps, n, s);
    else if constexpr (RL == kKContiguous) {
        typedef FewShape<1, 2, FL, false, false, 1> One;
        typedef FewShape<2, 2, FL, false, false, 1> Two;
        e = ps.p[0].nr <= 32 ? run_products<One>(gated_product_few_kernel<One>, One::LDS, ps, n, s)
                             : run_products<Two>(gated_product_few_kernel<Two>, Two::LDS, ps, n, s);
    } else
        e = hipErrorInvalidValue;
    return e != hipSuccess || t.splits == 1 ? e : launch_sum(ps, n, most, t.splits, s);
}

static hipError_t launch_down(const slicemoe_gated_config &c, const GatedPlan &plan, const char *Wd, size_t twd, long long ldwd, const void *addend,
                              void *y, char *ws, hipStream_t s)
{
    Products ps = {};
    ps.p[0] = problem(c.T, c.d, 2ll * c.H, 2ll * plan.ldh, ldwd);
    add_segments(ps.p[0], plan.terms, ws + plan.a, (size_t)c.T * 2 * plan.ldh, Wd, twd);
    ps.out[0] = {y, addend, c.T, c.d, c.dtype != SLICEMOE_BF16};
    return launch_products<kKContiguous, kKMajor>(ps, 1, choose_tiles(c.T, c.d, steps_of(ps.p[0]), false, true), ws + plan.part, s);
}

static Hidden hidden_of(const slicemoe_gated_config &c, const GatedPlan &p, char *ws)
{
    return {{(bf16_t *)(ws + p.a), (bf16_t *)(ws + p.dg), (bf16_t *)(ws + p.du)}, c.T, c.H, p.ldh};
}

template <int FL> static hipError_t run_few_f32(FewF32 a, hipStream_t s)
{
    a.tiles_r = ceil_div(a.rows, kF32Tile);
    a.tiles_f = ceil_div(a.N, 128);
    gated_few_f32_kernel<FL><<<a.tiles_r * a.tiles_f * a.images * a.splits, 256, 0, s>>>(a);
    return hipGetLastError();
}
// out = addend + the shares' sums, [T][d].
static hipError_t sum_few_f32(const slicemoe_gated_config &c, float *part, int shares, const void *addend, void *out, hipStream_t s)
{
    Products ps = {};
    ps.out[0] = {out, addend, c.T, c.d, 1};
    ps.part[0] = part;
    ps.p[0].splits = shares;
    return launch_sum(ps, 1, (long long)c.T * ((c.d + 7) / 8), shares, s);
}
static hipError_t launch_few_f32(const slicemoe_gated_config &c, const GatedPlan &plan, const float *x, const slicemoe_gated_weights &w,
                                 const void *addend, void *y, char *ws, hipStream_t s)
{
    float *part = (float *)(ws + plan.part), *a = (float *)ws;
    const int up_splits = few_f32_splits(c.T, 2, c.d, c.H), down_splits = few_f32_splits(c.T, 1, c.H, c.d);
    hipError_t e = run_few_f32<kKMajor>({{x, x}, {(const float *)w.Wg, (const float *)w.Wu}, part, c.T, c.d, c.H, c.d, plan.ldh, 2, 0, 2, up_splits}, s);
    if (e != hipSuccess) return e;
    const Hidden h = {{(bf16_t *)a}, c.T, c.H, plan.ldh};
    e = launch_up_sum<kAsF32, false, 2>(part, h, Scales(), up_splits, s);
    if (e != hipSuccess) return e;
    e = run_few_f32<kKMajor>({{a}, {(const float *)w.Wd}, part, c.T, c.H, c.d, plan.ldh, (c.d + 7) & ~7, 1, 0, 1, down_splits}, s);
    return e == hipSuccess ? sum_few_f32(c, part, down_splits, addend, y, s) : e;
}
static hipError_t launch_few_f32_backward(const slicemoe_gated_config &c, const GatedPlan &plan, const float *x, const slicemoe_gated_weights &w,
                                          const float *dy, const void *addend, void *dx, const slicemoe_gated_weight_grads &g, char *ws,
                                          hipStream_t s)
{
    float *part = (float *)(ws + plan.part), *a = (float *)(ws + plan.a), *dg = (float *)(ws + plan.dg), *du = (float *)(ws + plan.du);
    const float *Wg = (const float *)w.Wg, *Wu = (const float *)w.Wu, *Wd = (const float *)w.Wd;
    hipError_t e;
    if (c.T > 0) {
        const int splits = few_f32_splits(c.T, 3, c.d, c.H);
        e = run_few_f32<kKMajor>({{x, x}, {Wg, Wu}, part, c.T, c.d, c.H, c.d, plan.ldh, 2, 0, 3, splits}, s);
        if (e != hipSuccess) return e;
        e = run_few_f32<kKContiguous>({{dy}, {Wd}, part, c.T, c.d, c.H, c.d, plan.ldh, 1, 2, 3, splits}, s);
        if (e != hipSuccess) return e;
        e = launch_up_sum<kAsF32, false, 3>(part, hidden_of(c, plan, ws), Scales(), splits, s);
        if (e != hipSuccess) return e;
    }
    // before dx, which may take the place of dy
    const FewF32Weights p = {{x, x, a}, {dg, du, dy}, {(float *)g.Wg, (float *)g.Wu, (float *)g.Wd}, {c.d, c.d, c.H}, {c.H, c.H, c.d},
                             {c.d, c.d, plan.ldh}, {plan.ldh, plan.ldh, c.d}, c.T};
    const int tiles = std::max(ceil_div(c.d, 128) * ceil_div(c.H, 128), 1);   // of all three: 128 x 128 either way round
    gated_few_f32_weights_kernel<<<dim3(tiles, 3), 256, 0, s>>>(p);
    e = hipGetLastError();
    if (e != hipSuccess || c.T == 0) return e;
    const int splits = few_f32_splits(c.T, 2, c.H, c.d);
    e = run_few_f32<kKContiguous>({{dg, du}, {Wg, Wu}, part, c.T, c.H, c.d, plan.ldh, (c.d + 7) & ~7, 2, 0, 2, splits}, s);
    return e == hipSuccess ? sum_few_f32(c, part, 2 * splits, addend, dx, s) : e;
}

hipError_t launch_gated_ffn(const slicemoe_gated_config &c, const GatedPlan &plan, const void *x, const slicemoe_gated_weights &w,
                            const void *addend, void *y, char *ws, hipStream_t s)
{
    if (c.T == 0) return hipSuccess;
    if (plan.few_f32) return launch_few_f32(c, plan, (const float *)x, w, addend, y, ws, s);
    Operands o;
    hipError_t e = make_operands(c, plan, x, nullptr, w, ws, &o, s);
    if (e != hipSuccess) return e;
    GemmProblem p = problem(c.T, c.H, 2ll * c.d, o.ldx, o.ldw);
    add_segments(p, plan.terms, o.x, o.tx, o.Wg, o.tw, o.Wu);
    const Hidden h = hidden_of(c, plan, ws);
    float *part = (float *)(ws + plan.part);
    e = plan.terms == 1 ? launch_up<kKMajor, false, 1>(p, h, Scales(), part, s) : launch_up<kKMajor, false, 3>(p, h, Scales(), part, s);
    if (e != hipSuccess) return e;
    return launch_down(c, plan, o.Wd, o.twd, o.ldwd, addend, y, ws, s);
}

hipError_t launch_gated_ffn_quantized(const slicemoe_gated_config &c, const GatedPlan &plan, const uint8_t *x, const float *x_scale,
                                      const slicemoe_gated_weights_quantized &w, const void *addend, void *y, char *ws, hipStream_t s)
{
    if (c.T == 0) return hipSuccess;
    const slicemoe_gated_weights logical = {nullptr, nullptr, w.Wd};
    Operands o;
    hipError_t e = make_operands(c, plan, nullptr, nullptr, logical, ws, &o, s);
    if (e != hipSuccess) return e;
    GemmProblem p = problem(c.T, c.H, c.d, c.d, c.d);
    add_segments(p, 1, (const char *)x, 0, (const char *)w.Wg, 0, (const char *)w.Wu);
    e = launch_up<kKContiguous, true, 1>(p, hidden_of(c, plan, ws), Scales{x_scale, w.Wg_scale, w.Wu_scale}, (float *)(ws + plan.part), s);
    if (e != hipSuccess) return e;
    return launch_down(c, plan, o.Wd, o.twd, o.ldwd, addend, y, ws, s);
}

template <typename S, typename D, int TERMS> static hipError_t run_up_backward(GemmProblem p, GemmProblem q, const Hidden &h, hipStream_t s)
{
    set_tiles<S>(p, 1);
    set_tiles<D>(q, 1);
    constexpr int a = lds_of<S>(S::FT), b = lds_of<D>(S::FT), lds = a > b ? a : b;
    const auto kernel = gated_up_backward_kernel<S, D, TERMS>;
    const hipError_t e = ready(kernel, lds);
    if (e != hipSuccess) return e;
    kernel<<<p.tiles_r * p.tiles_f, 256, lds, s>>>(p, q, h);
    return hipGetLastError();
}
template <int TERMS> static hipError_t launch_up_backward(const GemmProblem &p, const GemmProblem &q, const Hidden &h, float *part, hipStream_t s)
{
    typedef Shapes<kKContiguous, kKMajor, true, false> Sh;
    typedef TileShape<4, 2, 2, 2, kKContiguous, kKContiguous, false, false, 3, 2> BigD;
    typedef TileShape<4, 1, 2, 2, kKContiguous, kKContiguous, false, false, 3, 2> WideD;
    typedef TileShape<2, 1, 2, 2, kKContiguous, kKContiguous, false, false, 3, 2> MiddleD;
    // (the products of a tile come one after the other: the sum of their steps; few rows take the middle tiles)
    const TileChoice t = choose_tiles(std::max(p.nr, kFewRows + 1), p.nf, steps_of(p) + steps_of(q) / 2, 3, true);
    if (t.splits > 1) {
        const hipError_t e = t.size == kBig    ? run_up_shares<typename Sh::Big, BigD>(p, q, h, t.splits, part, s)
                             : t.size == kWide ? run_up_shares<typename Sh::Wide, WideD>(p, q, h, t.splits, part, s)
                                               : run_up_shares<typename Sh::Middle, MiddleD>(p, q, h, t.splits, part, s);
        return e == hipSuccess ? launch_up_sum<TERMS, false, 3>(part, h, Scales(), t.splits, s) : e;
    }
    if (t.size == kBig) return run_up_backward<typename Sh::Big, BigD, TERMS>(p, q, h, s);
    if (t.size == kWide) return run_up_backward<typename Sh::Wide, WideD, TERMS>(p, q, h, s);
    return run_up_backward<typename Sh::Middle, MiddleD, TERMS>(p, q, h, s);
}

hipError_t launch_gated_ffn_backward(const slicemoe_gated_config &c, const GatedPlan &plan, const void *x, const slicemoe_gated_weights &w,
                                     const void *dy, const void *addend, void *dx, const slicemoe_gated_weight_grads &g, char *ws,
                                     hipStream_t s)
{
    if (plan.few_f32) return launch_few_f32_backward(c, plan, (const float *)x, w, (const float *)dy, addend, dx, g, ws, s);
    Operands o;
    hipError_t e = make_operands(c, plan, x, dy, w, ws, &o, s);
    if (e != hipSuccess) return e;
    const int terms = plan.terms, f32 = c.dtype != SLICEMOE_BF16;
    const char *a = ws + plan.a, *dg = ws + plan.dg, *du = ws + plan.du;
    char *part = ws + plan.part;
    if (c.T > 0) {
        GemmProblem p = problem(c.T, c.H, 2ll * c.d, o.ldx, o.ldw), q = problem(c.T, c.H, 2ll * c.d, o.ldx, o.ldwd);
        add_segments(p, terms, o.x, o.tx, o.Wg, o.tw, o.Wu);
        add_segments(q, terms, o.dy, o.tx, o.Wd, o.twd);
        const Hidden h = hidden_of(c, plan, ws);
        e = terms == 1 ? launch_up_backward<1>(p, q, h, (float *)part, s) : launch_up_backward<3>(p, q, h, (float *)part, s);
        if (e != hipSuccess) return e;
    }
    // The weight gradients, before dx: dx may then take the place of dy.  (T = 0: contractions of no steps, zeros.)
    {
        Products ps = {};
        ps.p[0] = problem(c.d, c.H, 2ll * c.T, o.ldx, o.ldh);
        ps.p[1] = ps.p[0];
        ps.p[2] = problem(c.H, c.d, 2ll * c.T, o.ldh, o.ldx);
        add_segments(ps.p[0], terms, o.x, o.tx, dg, o.th);
        add_segments(ps.p[1], terms, o.x, o.tx, du, o.th);
        add_segments(ps.p[2], terms, a, o.th, o.dy, o.tx);
        ps.out[0] = {g.Wg, nullptr, c.d, c.H, f32};
        ps.out[1] = {g.Wu, nullptr, c.d, c.H, f32};
        ps.out[2] = {g.Wd, nullptr, c.H, c.d, f32};
        const TileChoice t = choose_tiles(c.d, c.H, steps_of(ps.p[0]), false, true, 3);
        e = launch_products<kKMajor, kKMajor>(ps, 3, t, part, s);
        if (e != hipSuccess || c.T == 0) return e;
    }
    Products ps = {};
    ps.p[0] = problem(c.T, c.d, 2ll * c.H, o.ldh, o.ldw);
    add_segments(ps.p[0], terms, dg, o.th, o.Wg, o.tw);
    add_segments(ps.p[0], terms, du, o.th, o.Wu, o.tw);
    ps.out[0] = {dx, addend, c.T, c.d, f32};
    return launch_products<kKContiguous, kKContiguous>(ps, 1, choose_tiles(c.T, c.d, steps_of(ps.p[0]), false, true), part, s);
}

hipError_t launch_gated_quantize_weights(const slicemoe_gated_config &c, const slicemoe_gated_weights &w, uint8_t *Wg, float *Wg_scale,
                                         uint8_t *Wu, float *Wu_scale, hipStream_t s)
{
    gated_quantize_kernel<<<dim3((c.H + 31) / 32, 2), 256, 0, s>>>((const bf16_t *)w.Wg, (const bf16_t *)w.Wu, Wg, Wu, Wg_scale, Wu_scale, c.d, c.H);
    return hipGetLastError();
}

}  // namespace slicemoe
