// Root-mean-square norm of the residual stream in front of the layer, with the residual's addition, and its backward pass.
//
//   forward    s = x + residual,  r = 1 / sqrt(mean(s^2) + eps),  y = s r w
//   backward   n = s r,  m = dy w:   d_s = d_sum + r (m - n mean(m n)),   d_w = sum over the rows of dy n
//
// Both are one pass over memory: a row stays in the registers of the wavefronts that own it (one, four or sixteen of them) between
// its sums and its outputs, all of its pieces are requested before any is used, and the statistics are fp32.  The norm is taken of
// the fp32 sum, not of the stored one: y then carries one rounding.  The backward pass starts from the stored sum and computes r
// again, so the forward keeps nothing for it.  d_w: persistent blocks, a column sum per lane in registers over the block's rows, one
// row of partial sums per block, added in block order by a second kernel (bit-reproducible).
//
// Range: squares and their mean are fp32, so a row is squared as it is only where mean + eps lies in [2^-60, 2^60).  Any other row (values
// of 1e9 and more, or of 1e-9 and less with an eps as small) is multiplied by the power of two k that brings the larger of its largest
// value and sqrt(eps) to 1, summed again, and r is taken of k s and k^2 eps: n = (k s) r holds for every finite row.  All lanes of a row
// decide alike, by s and eps; k is 1 elsewhere and changes no bit.
//
// The e4m3 row: scale = max|y| / 448 (448: the largest e4m3 value), values y (1 / scale) rounded to nearest even.  A largest value below
// 1e-30 counts as 1e-30, so a row of zeros has a scale and no division by zero; a row that holds a NaN or an infinity has a NaN scale.
//
// HBM-bound.  65536 rows of 4096 bf16 values: forward 363 us = 5.9 TB/s, backward 430 + 6 = 4.9 (a copy of the same size: 5.2); 12289 rows
// of 768 with e4m3 output 13.8 us.  A decoding step's rows are their launch (32 x 1024: 3 us).  Rows that are not whole 16-byte pieces (d
// not a multiple of 8 for bf16, 4 for fp32) start at any element: their pieces are 16-byte accesses at element alignment, the last
// piece element by element.
#include "common.h"
#include "norm.h"
#include "wavefront.h"

namespace slicemoe {

template <typename T> struct RowPiece;   // 16 bytes of a row
template <> struct RowPiece<bf16_t> {
    static constexpr int V = 8;
    static __device__ __forceinline__ float get(const u32x4 &p, int i) { return __uint_as_float(i & 1 ? p[i >> 1] & 0xffff0000u : p[i >> 1] << 16); }
    static __device__ __forceinline__ u32x4 make(const float *v)
    {
        u32x4 p;
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = (uint32_t)f32_to_bf16(v[2 * i]) | (uint32_t)f32_to_bf16(v[2 * i + 1]) << 16;
        return p;
    }
};
template <> struct RowPiece<float> {
    static constexpr int V = 4;
    static __device__ __forceinline__ float get(const u32x4 &p, int i) { return __uint_as_float(p[i]); }
    static __device__ __forceinline__ u32x4 make(const float *v)
    {
        return u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    }
};

typedef u32x4 __attribute__((aligned(2))) loose;   // a row may start at any element
// Piece `at` (an element index, a multiple of V) of a row of d elements, zeros past its end.  ALIGNED: rows are whole aligned pieces.
template <typename T, bool ALIGNED> __device__ __forceinline__ u32x4 load_piece(const T *row, int at, int d)
{
    constexpr int V = RowPiece<T>::V;
    if constexpr (ALIGNED) {   // (no branch: the pieces of a row are requested together)
        u32x4 p = *(const u32x4 *)(row + (at < d ? at : 0));
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = at < d ? p[i] : 0;
        return p;
    }
    if (at >= d) return u32x4{0, 0, 0, 0};
    if (at + V <= d) return *(const loose *)(row + at);
    float v[V];
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = at + i < d ? Storage<T>::load(row + at + i) : 0.f;
    return RowPiece<T>::make(v);
}
template <typename T, bool ALIGNED> __device__ __forceinline__ void store_piece(T *row, int at, int d, const float *v)
{
    constexpr int V = RowPiece<T>::V;
    if constexpr (ALIGNED) *(u32x4 *)(row + at) = RowPiece<T>::make(v);
    else if (at + V <= d) *(loose *)(row + at) = RowPiece<T>::make(v);
    else
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (at + i < d) Storage<T>::store(row + at + i, v[i]);
}

// Sum (largest, as unsigned: absolute values in their bit order, a NaN above all) over the W wavefronts that own a row.
template <int W> __device__ __forceinline__ float row_sum(float v, float *lds)
{
    v = wavefront_sum_f32(v);
    if constexpr (W == 1) return v;
    __syncthreads();   // the values of the row's last sum have been read
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) s += lds[i];
    return s;
}
template <int W> __device__ __forceinline__ uint32_t row_max(uint32_t v, float *lds)
{
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) {
        const uint32_t o = (uint32_t)__shfl_xor((int)v, m);
        v = o > v ? o : v;
    }
    if constexpr (W == 1) return v;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = __uint_as_float(v);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < W; ++i) {
        const uint32_t o = __float_as_uint(lds[i]);
        v = o > v ? o : v;
    }
    return v;
}

// Below, squares lose bits that count for the mean; above, they or dy w s may overflow.
__device__ __forceinline__ bool in_range(float mean) { return mean >= 0x1p-60f && mean < 0x1p60f; }
// The power of two for a row whose largest magnitude has the bits `most`.  (An infinity or a NaN: any; 2^127 and 2^-126 are the ends.)
__device__ __forceinline__ float range_factor(uint32_t most, float eps)
{
    const uint32_t root = __float_as_uint(sqrtf(eps)), e = (most > root ? most : root) >> 23;
    return __uint_as_float((e < 253 ? 254 - e : 1) << 23);
}

// W wavefronts per row (W = 1: four rows per block of 256 threads), NP pieces per lane.  sum and y may be x or residual: a row's
// owners have all of it in registers before the first of them stores, and nothing tells the compiler that the arrays are apart.
template <typename T, bool ALIGNED, int W, int NP, bool QUANT>
__global__ __launch_bounds__(W == 16 ? 1024 : 256) void add_rmsnorm_kernel(const T *x, const T *residual, const T *__restrict__ w, T *sum, T *y,
                                                                         uint8_t *__restrict__ yq, float *__restrict__ yscale, int rows,
                                                                         int d, float eps)
{
    constexpr int V = RowPiece<T>::V, LANES = 64 * W;
    __shared__ float lds[W];
    const int lane = W == 1 ? threadIdx.x & 63 : threadIdx.x;
    const long long row = W == 1 ? (long long)blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x;
    if (row >= rows) return;   // (a whole wavefront; with W > 1 every block has its row)
    const size_t at0 = (size_t)row * d;
    u32x4 px[NP], pr[NP], pw[NP];
#pragma unroll
    for (int c = 0; c < NP; ++c) {
        const int at = (lane + c * LANES) * V;
        px[c] = load_piece<T, ALIGNED>(x + at0, at, d);
        pw[c] = load_piece<T, ALIGNED>(w, at, d);
    }
    if (residual)
#pragma unroll
        for (int c = 0; c < NP; ++c) pr[c] = load_piece<T, ALIGNED>(residual + at0, (lane + c * LANES) * V, d);
    float s[NP][V], ss = 0.f;
#pragma unroll
    for (int c = 0; c < NP; ++c)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            s[c][i] = RowPiece<T>::get(px[c], i);
            if (residual) s[c][i] += RowPiece<T>::get(pr[c], i);   // (without one, -0 stays -0)
            ss += s[c][i] * s[c][i];
        }
    float mean = row_sum<W>(ss, lds) / d + eps, k = 1.f;
    if (!in_range(mean)) {
        uint32_t top = 0;
#pragma unroll
        for (int c = 0; c < NP; ++c)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const uint32_t a = __float_as_uint(s[c][i]) & 0x7fffffffu;
                top = a > top ? a : top;
            }
        k = range_factor(row_max<W>(top, lds), eps);
        ss = 0.f;
#pragma unroll
        for (int c = 0; c < NP; ++c)
#pragma unroll
            for (int i = 0; i < V; ++i) ss += s[c][i] * k * (s[c][i] * k);
        mean = row_sum<W>(ss, lds) / d + eps * k * k;
    }
    const float r = 1.f / sqrtf(mean);
    uint32_t most = 0;
#pragma unroll
    for (int c = 0; c < NP; ++c) {
        const int at = (lane + c * LANES) * V;
        if (at < d && sum) store_piece<T, ALIGNED>(sum + at0, at, d, s[c]);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            s[c][i] = s[c][i] * k * r * RowPiece<T>::get(pw[c], i);
            const uint32_t a = __float_as_uint(s[c][i]) & 0x7fffffffu;
            if (QUANT && at + i < d) most = a > most ? a : most;
        }
        if (at < d && y) store_piece<T, ALIGNED>(y + at0, at, d, s[c]);
    }
    if constexpr (QUANT) {
        most = row_max<W>(most, lds);
        const float top = __uint_as_float(most);
        float scale = (top < kE4m3Floor ? kE4m3Floor : top) / kE4m3Max;
        if (most >= 0x7f800000u) scale = __uint_as_float(0x7fc00000u);   // an infinity or a NaN in the row
        const float inv = 1.f / scale;
        if (lane == 0) yscale[row] = scale;
#pragma unroll
        for (int c = 0; c < NP; ++c) {
            const int at = (lane + c * LANES) * V;
            if (at >= d) continue;
            uint32_t q[V / 4];
#pragma unroll
            for (int i = 0; i < V / 4; ++i) q[i] = pack_e4m3(s[c][4 * i] * inv, s[c][4 * i + 1] * inv, s[c][4 * i + 2] * inv, s[c][4 * i + 3] * inv);
            uint8_t *o = yq + at0 + at;
            if (ALIGNED) {
                if constexpr (V == 8) *(uint2 *)o = make_uint2(q[0], q[1]);
                else *(uint32_t *)o = q[0];
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (at + i < d) o[i] = (uint8_t)(q[i >> 2] >> 8 * (i & 3));
            }
        }
    }
}

// Two sums over the W wavefronts that own a row, in one exchange.  flip: alternates from row to row, so that one barrier per row does.
template <int W> __device__ __forceinline__ void row_sums(float &a, float &b, float (*lds)[2 * W], int flip)
{
    a = wavefront_sum_f32(a);
    b = wavefront_sum_f32(b);
    if constexpr (W == 1) return;
    float *l = lds[flip];
    if ((threadIdx.x & 63) == 0) {
        l[threadIdx.x >> 6] = a;
        l[W + (threadIdx.x >> 6)] = b;
    }
    lds_barrier();   // (the next row's loads stay on their way)
    a = b = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) {
        a += l[i];
        b += l[W + i];
    }
}

// Largest value over the same wavefronts.  l: LDS that the row has not used yet.
template <int W> __device__ __forceinline__ uint32_t row_most(uint32_t v, float *l)
{
    v = row_max<1>(v, nullptr);
    if constexpr (W == 1) return v;
    if ((threadIdx.x & 63) == 0) l[threadIdx.x >> 6] = __uint_as_float(v);
    lds_barrier();
#pragma unroll
    for (int i = 0; i < W; ++i) {
        const uint32_t o = __float_as_uint(l[i]);
        v = o > v ? o : v;
    }
    return v;
}

// Hides where a piece comes from: its values are unpacked again from here on, not kept in registers.
__device__ __forceinline__ void keep_packed(u32x4 &p) { asm volatile("" : "+v"(p)); }

// Block b takes the rows b, b + gridDim.x, .. (W = 1: its four wavefronts the row groups), so that a block's share differs by
// at most one row (group).  A row's pieces are requested while the row before it is worked on.  part[b][d]: its column sums of dy n.
template <typename T, bool ALIGNED, int W, int NP>
__global__ __launch_bounds__(W == 16 ? 1024 : 256) void add_rmsnorm_backward_kernel(
    const T *__restrict__ sum, const T *__restrict__ w, const T *dy, const T *dsum, T *dx, float *__restrict__ part, int rows, int d, float eps)
{
    constexpr int V = RowPiece<T>::V, LANES = 64 * W, ROWS = W == 1 ? 4 : 1;
    __shared__ float lds[2][2 * W];
    __shared__ float cols[W == 1 ? 3 : 1][W == 1 ? 64 * V : 1];
    const int lane = W == 1 ? threadIdx.x & 63 : threadIdx.x, wave = threadIdx.x >> 6;
    u32x4 pw[NP], ps[NP], pg[NP], pd[NP];
    float acc[NP][V];
    const auto request = [&](long long row) {
        const size_t at0 = (size_t)row * d;
#pragma unroll
        for (int c = 0; c < NP; ++c) {
            const int at = (lane + c * LANES) * V;
            ps[c] = load_piece<T, ALIGNED>(sum + at0, at, d);
            pg[c] = load_piece<T, ALIGNED>(dy + at0, at, d);
        }
        if (dsum)
#pragma unroll
            for (int c = 0; c < NP; ++c) pd[c] = load_piece<T, ALIGNED>(dsum + at0, (lane + c * LANES) * V, d);
    };
#pragma unroll
    for (int c = 0; c < NP; ++c) {
        pw[c] = load_piece<T, ALIGNED>(w, (lane + c * LANES) * V, d);
        pd[c] = u32x4{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < V; ++i) acc[c][i] = 0.f;
    }
    const float inv_d = 1.f / d;
    const long long stride = (long long)gridDim.x * ROWS;
    long long row = (long long)blockIdx.x * ROWS + (W == 1 ? wave : 0);
    long long left = 0, left_last = -1;   // first and last row out of range, whose turn comes at the end
    constexpr bool AHEAD = W < 16 && NP < 8;   // (where the registers hold two rows)
    if (AHEAD && row < rows) request(row);
    int flip = 0;
    for (; row < rows; row += stride, flip ^= 1) {
        if (!AHEAD) request(row);
        u32x4 cs[NP], cg[NP], cd[NP];
        float ss = 0.f, along = 0.f;
#pragma unroll
        for (int c = 0; c < NP; ++c) {
            cs[c] = ps[c];
            cg[c] = pg[c];
            cd[c] = pd[c];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float s = RowPiece<T>::get(cs[c], i);
                ss = fmaf(s, s, ss);
                along += RowPiece<T>::get(cg[c], i) * RowPiece<T>::get(pw[c], i) * s;
            }
        }
        if (AHEAD && row + stride < rows) request(row + stride);
        row_sums<W>(ss, along, lds, flip);
        const float mean = fmaf(ss, inv_d, eps);
        if (!in_range(mean)) {
            left = left_last < 0 ? row : left;
            left_last = row;
            continue;
        }
        const float r = 1.f / sqrtf(mean);
        const float mn = along * r * inv_d;   // mean(m n)
#pragma unroll
        for (int c = 0; c < NP; ++c) {
            const int at = (lane + c * LANES) * V;
            float v[V];
            if constexpr (NP >= 4) {   // (bf16 rows of 8192: 235 registers, two blocks per CU; without it 280, one)
                keep_packed(cs[c]);
                keep_packed(cg[c]);
            }
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float n = RowPiece<T>::get(cs[c], i) * r, g = RowPiece<T>::get(cg[c], i);
                acc[c][i] += g * n;
                v[i] = RowPiece<T>::get(cd[c], i) + r * (g * RowPiece<T>::get(pw[c], i) - n * mn);
            }
            if (at < d) store_piece<T, ALIGNED>(dx + (size_t)row * d, at, d, v);
        }
    }
    // The rows out of range, if there were any, in a loop of their own: handled above they cost every row registers and instructions (16384 x
    // 8192: 221 us became 234 to 253).  For the same reason each of their passes loads the pieces again, from an address that hides where it
    // is from.  Which rows they are is told by s alone (dy of the others may be their d_x by now), in the very operations of the loop above.
    // (65536 x 4096 bf16: 425 us without such a row, 424 with one, 947 with nothing else.)
    if (left_last >= 0)
        for (row = left; row <= left_last; row += stride, flip ^= 1) {
            const auto each = [&](const auto &f) {   // f(piece, its first element, pieces of s, dy, w)
                size_t at0 = (size_t)row * d;
                asm volatile("" : "+v"(at0));
#pragma unroll
                for (int c = 0; c < NP; ++c) {
                    const int at = (lane + c * LANES) * V;
                    f(c, at, load_piece<T, ALIGNED>(sum + at0, at, d), load_piece<T, ALIGNED>(dy + at0, at, d), load_piece<T, ALIGNED>(w, at, d));
                    __builtin_amdgcn_sched_barrier(0);
                }
            };
            float ss, along, k = 1.f;
            uint32_t top = 0;
            const auto sums = [&]() {
                ss = along = 0.f;
                each([&](int, int, const u32x4 &a, const u32x4 &b, const u32x4 &e) {
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const float v = RowPiece<T>::get(a, i), s = v * k;
                        const uint32_t u = __float_as_uint(v) & 0x7fffffffu;
                        top = u > top ? u : top;
                        ss = fmaf(s, s, ss);
                        along += RowPiece<T>::get(b, i) * RowPiece<T>::get(e, i) * s;
                    }
                });
                row_sums<W>(ss, along, lds, flip);
            };
            sums();
            if (in_range(fmaf(ss, inv_d, eps))) continue;
            // (every wavefront has read the last row's sums, which `flip ^ 1` held, and behind the next barrier this row's)
            k = range_factor(row_most<W>(top, lds[flip ^ 1]), eps);
            sums();
            const float r = 1.f / sqrtf(ss * inv_d + eps * k * k), mn = along * r * inv_d;   // of the scaled row
            each([&](int c, int at, const u32x4 &a, const u32x4 &b, const u32x4 &e) {
                u32x4 old = {0, 0, 0, 0};
                if (dsum) old = load_piece<T, ALIGNED>(dsum + (size_t)row * d, at, d);
                float v[V];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float n = RowPiece<T>::get(a, i) * k * r, g = RowPiece<T>::get(b, i);
                    acc[c][i] += g * n;
                    v[i] = RowPiece<T>::get(old, i) + r * ((g * RowPiece<T>::get(e, i) - n * mn) * k);
                }
                if (at < d) store_piece<T, ALIGNED>(dx + (size_t)row * d, at, d, v);
            });
        }
    // the block's column sums; with a row per wavefront the four wavefronts' are added in their order
    float *out = part + (size_t)blockIdx.x * d;
#pragma unroll
    for (int c = 0; c < NP; ++c) {
        const int at = (lane + c * LANES) * V;
        if constexpr (W == 1) {
            __syncthreads();
            if (wave > 0)
#pragma unroll
                for (int i = 0; i < V; ++i) cols[wave - 1][i * 64 + lane] = acc[c][i];
            __syncthreads();
            if (wave == 0)
#pragma unroll
                for (int i = 0; i < V; ++i) acc[c][i] = ((acc[c][i] + cols[0][i * 64 + lane]) + cols[1][i * 64 + lane]) + cols[2][i * 64 + lane];
        }
        if (W > 1 || wave == 0)
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (at + i < d) out[at + i] = acc[c][i];
    }
}

// d_w[c] = sum over the blocks, in their order: 64 columns per block, its 16 wavefronts take the partial rows b, b + 16, ..
__global__ __launch_bounds__(1024) void norm_weight_sum_kernel(const float *__restrict__ part, float *__restrict__ dw, int blocks, int d)
{
    __shared__ float t[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = blockIdx.x * 64 + lane;
    float a = 0.f;
    if (col < d) {
        int b = wave;
        for (; b + 15 * 16 < blocks; b += 256) {   // sixteen rows in flight
            float v[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = part[(size_t)(b + 16 * i) * d + col];
#pragma unroll
            for (int i = 0; i < 16; ++i) a += v[i];
        }
        for (; b < blocks; b += 16) a += part[(size_t)b * d + col];
    }
    t[wave][lane] = a;
    __syncthreads();
    if (wave == 0 && col < d) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) s += t[i][lane];
        dw[col] = s;
    }
}

// Calls f.run<T, ALIGNED, W, NP>() for a row of d elements: one wavefront takes up to eight pieces per lane (4096 bf16 or 2048 fp32
// values), then four, then sixteen of them.  kWide: four from three pieces per lane on (the backward pass holds four rows and a column
// sum per element: at d = 4096 one wavefront per row has two wavefronts per SIMD to hide the memory behind, 556 us against 4 x 2).
template <typename T, typename F> static hipError_t pick_row(int d, const F &f)
{
    constexpr int V = RowPiece<T>::V;
    const int pieces = (d + V - 1) / V;
    const auto go = [&](auto al) {
        constexpr bool A = decltype(al)::value;
        if (pieces <= 64) return f.template run<T, A, 1, 1>();
        if (pieces <= 128) return f.template run<T, A, 1, 2>();
        if constexpr (F::kWide) {
            if (pieces <= 256) return f.template run<T, A, 4, 1>();
            if (pieces <= 512) return f.template run<T, A, 4, 2>();
        } else {
            if (pieces <= 256) return f.template run<T, A, 1, 4>();
            if (pieces <= 512) return f.template run<T, A, 1, 8>();
        }
        if (pieces <= 1024) return f.template run<T, A, 4, 4>();
        if constexpr (V == 4)   // (bf16 rows end at 2048 pieces)
            if (pieces > 2048) return f.template run<T, A, 16, 4>();
        return f.template run<T, A, 4, 8>();
    };
    return d % V == 0 ? go(std::true_type()) : go(std::false_type());
}

constexpr int kNormLaunchBlocks = 1 << 21;   // a launch ends below 2^32 threads: more rows than these blocks hold are several launches
struct ForwardCall {
    static constexpr bool kWide = false;
    const void *x, *residual, *w;
    void *sum, *y;
    uint8_t *yq;
    float *yscale;
    int rows, d;
    float eps;
    hipStream_t s;
    template <typename T, bool A, int W, int NP> hipError_t run() const
    {
        constexpr int threads = W == 16 ? 1024 : 256, per_block = W == 1 ? 4 : 1, most = kNormLaunchBlocks * per_block;
        for (int first = 0;;) {
            const int n = rows - first < most ? rows - first : most;
            const unsigned blocks = (unsigned)((n + per_block - 1) / per_block);
            const size_t at = (size_t)first * d;
            const T *r = residual ? (const T *)residual + at : nullptr;
            T *so = sum ? (T *)sum + at : nullptr, *yo = y ? (T *)y + at : nullptr;
            if (yq)
                add_rmsnorm_kernel<T, A, W, NP, true><<<blocks, threads, 0, s>>>((const T *)x + at, r, (const T *)w, so, yo, yq + at, yscale + first, n,
                                                                               d, eps);
            else
                add_rmsnorm_kernel<T, A, W, NP, false><<<blocks, threads, 0, s>>>((const T *)x + at, r, (const T *)w, so, yo, nullptr, nullptr, n, d, eps);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess || rows - first <= most) return e;
            first += most;
        }
    }
};

struct BackwardCall {
    static constexpr bool kWide = true;
    const void *sum, *w, *dy, *dsum;
    void *dx;
    float *dw, *part;
    int rows, d, blocks;
    float eps;
    hipStream_t s;
    // Blocks at most, those that are resident together: with more the last ones run beside half a chip (16384 x 8192 bf16, 512 / 768: 206 / 233
    // us; 16384 x 4096 fp32 196 / 216; 8192 x 16384 bf16, 256 / 512 / 768: 312 / 327 / 344; 16384 x 8192 fp32 393 to 407 with any).
    template <typename T, int W, int NP> static constexpr int most()
    {
        return W == 16 || (NP == 8 && RowPiece<T>::V == 8) ? kNormBackwardBlocks / 3 : NP >= 4 ? kNormBackwardBlocks * 2 / 3 : kNormBackwardBlocks;
    }
    template <typename T, bool A, int W, int NP> hipError_t run() const
    {
        const int n = blocks < most<T, W, NP>() ? blocks : most<T, W, NP>();
        add_rmsnorm_backward_kernel<T, A, W, NP><<<n, W == 16 ? 1024 : 256, 0, s>>>((const T *)sum, (const T *)w, (const T *)dy, (const T *)dsum,
                                                                                  (T *)dx, part, rows, d, eps);   // (no rows: writes zeros to part)
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        norm_weight_sum_kernel<<<(d + 63) / 64, 1024, 0, s>>>(part, dw, n, d);
        return hipGetLastError();
    }
};

// Four rows per block: as many as it takes at once where a wavefront owns a row (up to 128 pieces: see pick_row).  Wider rows follow one
// another in a block, so there a row each as long as that makes no more than a block per CU (256 x 4096 bf16: 11.3 -> 10.3 us, 16 x 16384:
// 27 -> 16); with more blocks their partial rows cost more than they bring (1024 x 4096: 256 blocks 13.4, 768 20.0).
int norm_backward_blocks(const slicemoe_norm_config &c)
{
    const int pieces = c.dtype == SLICEMOE_BF16 ? (c.d + 7) / 8 : (c.d + 3) / 4, fours = c.T / 4 + (c.T % 4 != 0);
    const int each = pieces <= 128 ? 0 : c.T < kNormBackwardBlocks / 3 ? c.T : kNormBackwardBlocks / 3;
    const int blocks = fours > each ? fours : each;
    return blocks < 1 ? 1 : blocks < kNormBackwardBlocks ? blocks : kNormBackwardBlocks;
}

hipError_t launch_add_rmsnorm(const slicemoe_norm_config &c, const void *x, const void *residual, const void *weight, void *sum, void *y,
                              uint8_t *yq, float *yscale, hipStream_t s)
{
    if (c.T == 0) return hipSuccess;
    const ForwardCall f{x, residual, weight, sum, y, yq, yscale, c.T, c.d, c.eps, s};
    return c.dtype == SLICEMOE_BF16 ? pick_row<bf16_t>(c.d, f) : pick_row<float>(c.d, f);
}

hipError_t launch_add_rmsnorm_backward(const slicemoe_norm_config &c, const void *sum, const void *weight, const void *dy,
                                       const void *dsum, void *dx, float *dw, float *part, hipStream_t s)
{
    const BackwardCall f{sum, weight, dy, dsum, dx, dw, part, c.T, c.d, norm_backward_blocks(c), c.eps, s};
    return c.dtype == SLICEMOE_BF16 ? pick_row<bf16_t>(c.d, f) : pick_row<float>(c.d, f);
}

}  // namespace slicemoe
