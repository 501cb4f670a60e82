// Norms on both sides of a block's addition to the residual stream, with the block's gate and the stream's scale, and the backward pass.
//
//   forward    n = x r1 post,  r1 = 1 / sqrt(mean(x^2) + eps);   s = a residual + gate n;   y = s r2 pre,  r2 = 1 / sqrt(mean(s^2) + eps)
//   backward   m2 = dy pre, n2 = s r2:   ds = d_sum + r2 (m2 - n2 mean(m2 n2)),   d_residual = a ds
//              n1 = x r1, m1 = ds gate post:   d_x = r1 (m1 - n1 mean(m1 n1)),   d_gate = ds n1 post
//              d_pre = sum over the rows of dy n2,   d_post = sum of ds n1 gate   (and d_gate the sum of ds n1 post where the gate is one row)
//
// Both are one pass over memory with a row in the registers of the wavefronts that own it; the second norm's sum waits for the first's.  The
// norm is of the fp32 sum.  The forward leaves r1 and r2 of a row (8 bytes), so the backward has two sums per row (mean(m2 n2), then mean(m1 n1))
// and no squares to stay in range: n1 and n2 are formed before anything is multiplied.  Squares of the forward are in range as in norm.hip, by
// a power of two for the row.
// With one gate for all rows both d_post and d_gate are a column's sum of ds n1 times that column's gate and weight, so there are two column
// sums in either case; persistent blocks, a row of partial sums per block, added in block order (bit-reproducible).
#include "block_norm.h"
#include "mx.h"
#include "norm.h"
#include "norm_row.h"

namespace slicemoe {

// mean(v^2) + eps of a row in registers as r = 1 / sqrt of it and the power of two k that v was multiplied with: v / rms = (v k) r.
template <int W, int NP, int V> __device__ __forceinline__ float row_rsqrt(const float (&v)[NP][V], int d, float eps, float &k, float *lds)
{
    float ss = 0.f;
#pragma unroll
    for (int c = 0; c < NP; ++c)
#pragma unroll
        for (int i = 0; i < V; ++i) ss += v[c][i] * v[c][i];
    float mean = row_sum<W>(ss, lds) / d + eps;
    k = 1.f;
    if (!in_range(mean)) {
        uint32_t top = 0;
#pragma unroll
        for (int c = 0; c < NP; ++c)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const uint32_t a = __float_as_uint(v[c][i]) & 0x7fffffffu;
                top = a > top ? a : top;
            }
        k = range_factor(row_max<W>(top, lds), eps);
        ss = 0.f;
#pragma unroll
        for (int c = 0; c < NP; ++c)
#pragma unroll
            for (int i = 0; i < V; ++i) ss += v[c][i] * k * (v[c][i] * k);
        mean = row_sum<W>(ss, lds) / d + eps * k * k;
    }
    return 1.f / sqrtf(mean);
}

// A row's y as microscaled values: a block of 32 is in 32 / V neighbouring lanes.
template <int BITS, typename T, int W, int NP, int V>
__device__ __forceinline__ void store_mx(const float (&y)[NP][V], uint8_t *mx, uint8_t *scales, int row, int d, int lane)
{
    const int tiles_k = mx_tiles_k(d);
#pragma unroll
    for (int c = 0; c < NP; ++c) {
        const int at = (lane + c * 64 * W) * V;
        float v[V];
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            v[i] = at + i < d ? y[c][i] : 0.f;
            const uint32_t a = __float_as_uint(v[i]) & 0x7fffffffu;
            most = a > most ? a : most;
        }
        const auto larger = [&](int o) { most = (uint32_t)o > most ? (uint32_t)o : most; };
        larger(lane_move<0xB1>((int)most));              // quad_perm [1, 0, 3, 2]
        larger(lane_move<0x4E>((int)most));              // quad_perm [2, 3, 0, 1]
        if constexpr (V == 4) larger(lane_move<0x141>((int)most));   // row_half_mirror: the other four lanes
        if (at >= tiles_k * kMxCols) continue;           // (whole blocks)
        const uint32_t byte = mx_scale_byte<BITS>(most);
        const float inv = mx_inverse(byte);
        const int kb = at >> 5, m = at >> 2 & 7;
#pragma unroll
        for (int h = 0; h < V / 4; ++h) {
            const uint32_t q = mx_pack4<BITS>(v[4 * h] * inv, v[4 * h + 1] * inv, v[4 * h + 2] * inv, v[4 * h + 3] * inv);
            uint8_t *o = mx + mx_quad_offset<BITS>(row, kb, m + h, tiles_k);
            if constexpr (BITS == 4) *(uint16_t *)o = (uint16_t)q;
            else *(uint32_t *)o = q;
        }
        if (m == 0) scales[mx_scale_offset(row, kb, tiles_k)] = (uint8_t)byte;
    }
}

// A block takes the rows b, b + gridDim.x, .. (W = 1: each of its wavefronts one of four).  gate_ld: 0 for a gate of one row.  sum and y may
// be x or residual: a row's owners have all of it in registers before the first of them stores.
template <typename T, bool ALIGNED, int W, int NP, bool MX>
__global__ __launch_bounds__(W == 16 ? 1024 : 256) void block_norm_kernel(const T *x, const T *__restrict__ post, const T *__restrict__ gate, long long gate_ld,
                                                                        const T *residual, float a, const T *__restrict__ pre, T *sum, T *y,
                                                                        uint8_t *__restrict__ mx, uint8_t *__restrict__ mx_scales, int bits,
                                                                        float *__restrict__ stats, int rows, int d, float eps)
{
    constexpr int V = RowPiece<T>::V, LANES = 64 * W, ROWS = W == 1 ? 4 : 1;
    __shared__ float lds[W];
    const int lane = W == 1 ? threadIdx.x & 63 : threadIdx.x;
    for (long long row = (long long)blockIdx.x * ROWS + (W == 1 ? threadIdx.x >> 6 : 0); row < rows; row += (long long)gridDim.x * ROWS) {
        const size_t at0 = (size_t)row * d;
        u32x4 px[NP], pr[NP], pg[NP], po[NP], pw[NP];
#pragma unroll
        for (int c = 0; c < NP; ++c) {
            const int at = (lane + c * LANES) * V;
            px[c] = load_piece<T, ALIGNED>(x + at0, at, d);
            pr[c] = load_piece<T, ALIGNED>(residual + at0, at, d);
        }
        if (gate)
#pragma unroll
            for (int c = 0; c < NP; ++c) pg[c] = load_piece<T, ALIGNED>(gate + (size_t)row * gate_ld, (lane + c * LANES) * V, d);
        if (post)
#pragma unroll
            for (int c = 0; c < NP; ++c) po[c] = load_piece<T, ALIGNED>(post, (lane + c * LANES) * V, d);
        if (pre)
#pragma unroll
            for (int c = 0; c < NP; ++c) pw[c] = load_piece<T, ALIGNED>(pre, (lane + c * LANES) * V, d);
        float s[NP][V], k1 = 1.f, r1 = 1.f;
#pragma unroll
        for (int c = 0; c < NP; ++c)
#pragma unroll
            for (int i = 0; i < V; ++i) s[c][i] = RowPiece<T>::get(px[c], i);
        if (post) r1 = row_rsqrt<W, NP, V>(s, d, eps, k1, lds);
#pragma unroll
        for (int c = 0; c < NP; ++c) {
            const int at = (lane + c * LANES) * V;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float n = s[c][i] * k1 * r1;
                if (post) n *= RowPiece<T>::get(po[c], i);
                if (gate) n *= RowPiece<T>::get(pg[c], i);
                s[c][i] = fmaf(a, RowPiece<T>::get(pr[c], i), n);
            }
            if (at < d) store_piece<T, ALIGNED>(sum + at0, at, d, s[c]);
        }
        float k2, r2 = row_rsqrt<W, NP, V>(s, d, eps, k2, lds);
        if (stats && lane == 0) *(float2 *)(stats + 2 * row) = make_float2(k1 * r1, k2 * r2);
        if (!pre) continue;
#pragma unroll
        for (int c = 0; c < NP; ++c) {
            const int at = (lane + c * LANES) * V;
#pragma unroll
            for (int i = 0; i < V; ++i) s[c][i] = s[c][i] * k2 * r2 * RowPiece<T>::get(pw[c], i);
            if (at < d && y) store_piece<T, ALIGNED>(y + at0, at, d, s[c]);
        }
        if constexpr (MX) {
            if (bits == 4) store_mx<4, T, W, NP, V>(s, mx, mx_scales, (int)row, d, lane);
            else store_mx<8, T, W, NP, V>(s, mx, mx_scales, (int)row, d, lane);
        }
    }
}

// Sum over the W wavefronts of a row; two arrays in turn, so one barrier each does: who writes an array has passed the other's barrier,
// in front of which everybody had read it.
template <int W> __device__ __forceinline__ float row_sum_once(float v, float *l)
{
    v = wavefront_sum_f32(v);
    if constexpr (W == 1) return v;
    if ((threadIdx.x & 63) == 0) l[threadIdx.x >> 6] = v;
    lds_barrier();
    v = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) v += l[i];
    return v;
}

// part: [2][gridDim.x][d] column sums of dy n2 and of ds n1 (TOKEN: times the gate).  d_x may be d_y, d_residual may be d_sum (or d_y).
template <typename T, bool ALIGNED, int W, int NP, bool TOKEN>
__global__ __launch_bounds__(W == 16 ? 1024 : 256) void block_norm_backward_kernel(const T *__restrict__ x, const T *__restrict__ post, const T *__restrict__ gate,
                                                                                 const T *__restrict__ sum, const T *__restrict__ pre,
                                                                                 const float *__restrict__ stats, const T *dy, const T *dsum, float a, T *dx,
                                                                                 T *dres, T *dgate, float *__restrict__ part, int rows, int d)
{
    constexpr int V = RowPiece<T>::V, LANES = 64 * W, ROWS = W == 1 ? 4 : 1;
    __shared__ float lds[2][W];
    __shared__ float cols[W == 1 ? 3 : 1][W == 1 ? 64 * V : 1];
    const int lane = W == 1 ? threadIdx.x & 63 : threadIdx.x, wave = threadIdx.x >> 6;
    u32x4 pw[NP], po[NP], pc[NP], ps[NP], pg[NP], pd[NP], px[NP], pt[TOKEN ? NP : 1];
    float acc[2][NP][V];
    const auto request = [&](long long row) {
        const size_t at0 = (size_t)row * d;
#pragma unroll
        for (int c = 0; c < NP; ++c) {
            const int at = (lane + c * LANES) * V;
            ps[c] = load_piece<T, ALIGNED>(sum + at0, at, d);
            pg[c] = load_piece<T, ALIGNED>(dy + at0, at, d);
            px[c] = load_piece<T, ALIGNED>(x + at0, at, d);
            if constexpr (TOKEN) pt[c] = load_piece<T, ALIGNED>(gate + at0, at, d);
        }
        if (dsum)
#pragma unroll
            for (int c = 0; c < NP; ++c) pd[c] = load_piece<T, ALIGNED>(dsum + at0, (lane + c * LANES) * V, d);
    };
    float ones[V];
#pragma unroll
    for (int i = 0; i < V; ++i) ones[i] = 1.f;
#pragma unroll
    for (int c = 0; c < NP; ++c) {
        const int at = (lane + c * LANES) * V;
        pw[c] = load_piece<T, ALIGNED>(pre, at, d);
        po[c] = post ? load_piece<T, ALIGNED>(post, at, d) : RowPiece<T>::make(ones);
        if constexpr (!TOKEN) pc[c] = gate ? load_piece<T, ALIGNED>(gate, at, d) : RowPiece<T>::make(ones);
        pd[c] = u32x4{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < V; ++i) acc[0][c][i] = acc[1][c][i] = 0.f;
    }
    const float inv_d = 1.f / d, normed = post ? inv_d : 0.f;   // without a norm behind the block d_x is m1
    const long long stride = (long long)gridDim.x * ROWS;
    long long row = (long long)blockIdx.x * ROWS + (W == 1 ? wave : 0);
    constexpr bool AHEAD = W < 16 && NP < 4;   // (where the registers hold two rows)
    float2 r = make_float2(0.f, 0.f);
    if (AHEAD && row < rows) {
        request(row);
        r = *(const float2 *)(stats + 2 * row);
    }
    for (; row < rows; row += stride) {
        const size_t at0 = (size_t)row * d;
        if (!AHEAD) {
            request(row);
            r = *(const float2 *)(stats + 2 * row);
        }
        u32x4 cs[NP], cg[NP], cd[NP], cx[NP], ct[TOKEN ? NP : 1];
        float along = 0.f;
#pragma unroll
        for (int c = 0; c < NP; ++c) {
            cs[c] = ps[c];
            cg[c] = pg[c];
            cd[c] = pd[c];
            cx[c] = px[c];
            if constexpr (TOKEN) ct[c] = pt[c];
#pragma unroll
            for (int i = 0; i < V; ++i) along += RowPiece<T>::get(cg[c], i) * RowPiece<T>::get(pw[c], i) * (RowPiece<T>::get(cs[c], i) * r.y);
        }
        const float r1 = r.x, r2 = r.y;
        if (AHEAD && row + stride < rows) {
            request(row + stride);
            r = *(const float2 *)(stats + 2 * (row + stride));
        }
        const float mn2 = row_sum_once<W>(along, lds[0]) * inv_d;
        along = 0.f;
        float ds[NP][V];
#pragma unroll
        for (int c = 0; c < NP; ++c) {
            const int at = (lane + c * LANES) * V;
            float v[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float n2 = RowPiece<T>::get(cs[c], i) * r2, g = RowPiece<T>::get(cg[c], i), n1 = RowPiece<T>::get(cx[c], i) * r1;
                ds[c][i] = RowPiece<T>::get(cd[c], i) + r2 * (g * RowPiece<T>::get(pw[c], i) - n2 * mn2);
                const float gt = TOKEN ? RowPiece<T>::get(ct[TOKEN ? c : 0], i) : RowPiece<T>::get(pc[c], i), dn = ds[c][i] * n1;
                acc[0][c][i] += g * n2;
                acc[1][c][i] += TOKEN ? dn * gt : dn;
                along += dn * gt * RowPiece<T>::get(po[c], i);
                v[i] = a * ds[c][i];
            }
            if (at < d) store_piece<T, ALIGNED>(dres + at0, at, d, v);
            if constexpr (TOKEN) {
#pragma unroll
                for (int i = 0; i < V; ++i) v[i] = ds[c][i] * (RowPiece<T>::get(cx[c], i) * r1) * RowPiece<T>::get(po[c], i);
                if (at < d) store_piece<T, ALIGNED>(dgate + at0, at, d, v);
            }
        }
        const float mn1 = row_sum_once<W>(along, lds[1]) * normed;
#pragma unroll
        for (int c = 0; c < NP; ++c) {
            const int at = (lane + c * LANES) * V;
            float v[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float gt = TOKEN ? RowPiece<T>::get(ct[TOKEN ? c : 0], i) : RowPiece<T>::get(pc[c], i);
                v[i] = r1 * (ds[c][i] * gt * RowPiece<T>::get(po[c], i) - RowPiece<T>::get(cx[c], i) * r1 * mn1);
            }
            if (at < d) store_piece<T, ALIGNED>(dx + at0, at, d, v);
        }
    }
    // the block's column sums; with a row per wavefront the four wavefronts' are added in their order
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        float *out = part + ((size_t)q * gridDim.x + blockIdx.x) * d;
#pragma unroll
        for (int c = 0; c < NP; ++c) {
            const int at = (lane + c * LANES) * V;
            if constexpr (W == 1) {
                __syncthreads();
                if (wave > 0)
#pragma unroll
                    for (int i = 0; i < V; ++i) cols[wave - 1][i * 64 + lane] = acc[q][c][i];
                __syncthreads();
                if (wave == 0)
#pragma unroll
                    for (int i = 0; i < V; ++i) acc[q][c][i] = ((acc[q][c][i] + cols[0][i * 64 + lane]) + cols[1][i * 64 + lane]) + cols[2][i * 64 + lane];
            }
            if (W > 1 || wave == 0)
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (at + i < d) out[at + i] = acc[q][c][i];
        }
    }
}

// The sums over the blocks, in their order: 64 columns per block, its 16 wavefronts take the partial rows b, b + 16, ..  blockIdx.y = 0: d_pre; 1:
// d_post and, where the gate is one row, d_gate.
template <typename T>
__global__ __launch_bounds__(1024) void block_norm_weight_sum_kernel(const float *__restrict__ part, const T *__restrict__ post, const T *__restrict__ gate /* one row, or null */,
                                                                     float *__restrict__ dpre, float *__restrict__ dpost, float *__restrict__ dgate, int blocks, int d)
{
    __shared__ float t[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = blockIdx.x * 64 + lane;
    const float *p = part + (size_t)blockIdx.y * blocks * d;
    float a = 0.f;
    if (col < d) {
        int b = wave;
        for (; b + 15 * 16 < blocks; b += 256) {   // sixteen rows in flight
            float v[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = p[(size_t)(b + 16 * i) * d + col];
#pragma unroll
            for (int i = 0; i < 16; ++i) a += v[i];
        }
        for (; b < blocks; b += 16) a += p[(size_t)b * d + col];
    }
    t[wave][lane] = a;
    __syncthreads();
    if (wave == 0 && col < d) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) s += t[i][lane];
        if (blockIdx.y == 0) dpre[col] = s;
        else {
            if (dpost) dpost[col] = gate ? s * Storage<T>::load(gate + col) : s;
            if (dgate) dgate[col] = post ? s * Storage<T>::load(post + col) : s;
        }
    }
}

struct BlockNormForward {
    static constexpr bool kWide = true;
    const slicemoe_block_norm_config &c;
    const void *x, *post, *gate, *residual, *pre;
    void *sum, *y;
    uint8_t *mx;
    int bits;
    float *stats;
    hipStream_t s;
    template <typename T, bool A, int W, int NP> hipError_t run() const
    {
        constexpr int threads = W == 16 ? 1024 : 256, per_block = W == 1 ? 4 : 1;
        const int need = c.T / per_block + (c.T % per_block != 0), most = num_compute_units() * 8;
        const unsigned blocks = need < most ? need : most;
        uint8_t *scales = mx ? mx + mx_tiles(c.T, c.d) * mx_tile_bytes(bits) : nullptr;
        const auto kern = mx ? block_norm_kernel<T, A, W, NP, true> : block_norm_kernel<T, A, W, NP, false>;
        kern<<<blocks, threads, 0, s>>>((const T *)x, (const T *)post, (const T *)gate, c.gate == SLICEMOE_GATE_TOKEN ? c.d : 0, (const T *)residual,
                                        c.residual_scale, (const T *)pre, (T *)sum, (T *)y, mx, scales, bits, stats, c.T, c.d, c.eps);
        return hipGetLastError();
    }
};

struct BlockNormBackward {
    static constexpr bool kWide = true;
    const slicemoe_block_norm_config &c;
    const void *x, *post, *gate, *sum, *pre;
    const float *stats;
    const void *dy, *dsum;
    void *dx, *dres;
    float *dpost;
    void *dgate;
    float *dpre, *part;
    int blocks;
    hipStream_t s;
    template <typename T, bool A, int W, int NP> hipError_t run() const
    {
        constexpr int threads = W == 16 ? 1024 : 256;
        const bool token = c.gate == SLICEMOE_GATE_TOKEN;
        const auto kern = token ? block_norm_backward_kernel<T, A, W, NP, true> : block_norm_backward_kernel<T, A, W, NP, false>;
        kern<<<blocks, threads, 0, s>>>((const T *)x, (const T *)post, (const T *)gate, (const T *)sum, (const T *)pre, stats, (const T *)dy, (const T *)dsum,
                                        c.residual_scale, (T *)dx, (T *)dres, (T *)dgate, part, c.T, c.d);   // (no rows: writes zeros to part)
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        block_norm_weight_sum_kernel<T><<<dim3((c.d + 63) / 64, 2), 1024, 0, s>>>(part, (const T *)post, token ? nullptr : (const T *)gate, dpre, dpost,
                                                                                token || !gate ? nullptr : (float *)dgate, blocks, c.d);
        return hipGetLastError();
    }
};

int block_norm_backward_blocks(const slicemoe_block_norm_config &c)
{
    const slicemoe_norm_config n = {c.T, c.d, c.eps, c.dtype};
    return norm_backward_blocks(n);
}

hipError_t launch_block_norm(const slicemoe_block_norm_config &c, const void *x, const void *post, const void *gate, const void *residual,
                             const void *pre, void *sum, void *y, uint8_t *mx, int bits, float *stats, hipStream_t s)
{
    if (c.T == 0) return hipSuccess;
    const BlockNormForward f{c, x, post, gate, residual, pre, sum, y, mx, bits, stats, s};
    return c.dtype == SLICEMOE_BF16 ? pick_row<bf16_t>(c.d, f) : pick_row<float>(c.d, f);
}

hipError_t launch_block_norm_backward(const slicemoe_block_norm_config &c, const void *x, const void *post, const void *gate, const void *sum,
                                      const void *pre, const float *stats, const void *dy, const void *dsum, void *dx, void *dres,
                                      float *dpost, void *dgate, float *dpre, float *part, hipStream_t s)
{
    const BlockNormBackward f{c, x, post, gate, sum, pre, stats, dy, dsum, dx, dres, dpost, dgate, dpre, part, block_norm_backward_blocks(c), s};
    return c.dtype == SLICEMOE_BF16 ? pick_row<bf16_t>(c.d, f) : pick_row<float>(c.d, f);
}

}  // namespace slicemoe
