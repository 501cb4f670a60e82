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
//
// Bound by memory: 65536 x 4096 in bf16 with one gate row takes 440 us forward and 614 backward (its 2.1 and 3.2 GB: 418 and 627 us at the 5.14
// TB/s of a large copy), 12289 x 768 with a gate per token 20 and 33 (18.4 and 29.4); below some thousand rows by the launches, one forward and two
// backward (32 x 1024: 4 us in the kernel; 3001 x 513 in fp32 backward: 15 us of 9.6), and by a row's two sums one behind the other.
#include "block_norm.h"
#include "mx.h"
#include "norm.h"
#include "norm_row.h"

namespace slicemoe {

// How a row's pieces lie: whole and aligned; or each at any element, the last one the V elements in front of the row's end, of which the first
// `cut` are another lane's too (they count once in the sums, both lanes store them alike): no branch between the requests (12289 x 767 in bf16
// backward: 36.7 us, 81 with a branch for the last piece); kShared: the same, and these two lanes are in two wavefronts, so that in place the store of one may
// meet the load of the other, for which a barrier alone does not wait (a mode of its own: with the wait in both, rows of 8191 in bf16 need 68 registers for
// 62 and have one block a CU for two: 8192 of them 190 us for 161); or by element, for rows below a piece and where a lane's columns have to be its
// own (microscaled rows).
enum { kAligned, kOverlapped, kShared, kByElement };
// What this wavefront has requested has arrived.
__device__ __forceinline__ void wait_for_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
template <typename T, int MODE> struct Place {
    static constexpr bool OVERLAPS = MODE == kOverlapped || MODE == kShared;
    static constexpr int V = RowPiece<T>::V;
    int from, cut;
    bool mine;
    __device__ __forceinline__ Place(int at, int d) : from(OVERLAPS && at + V > d ? d - V : at), cut(at - from), mine(at < d) {}
    __device__ __forceinline__ uint32_t bytes() const { return (uint32_t)from * (uint32_t)sizeof(T); }   // (32 bits on a row's uniform start)
    __device__ __forceinline__ u32x4 load(const T *row, int d) const
    {
        if constexpr (MODE == kByElement) return load_piece<T, false>(row, from, d);
        else if constexpr (OVERLAPS) return *(const loose *)((const char *)row + bytes());
        else {   // (zeros past the row's end)
            u32x4 p = *(const u32x4 *)((const char *)row + (mine ? bytes() : 0u));
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] = mine ? p[i] : 0;
            return p;
        }
    }
    __device__ __forceinline__ void store(T *row, int d, const float *v) const
    {
        if (!mine) return;
        if constexpr (MODE == kByElement) store_piece<T, false>(row, from, d, v);
        else if constexpr (OVERLAPS) *(loose *)((char *)row + bytes()) = RowPiece<T>::make(v);
        else *(u32x4 *)((char *)row + bytes()) = RowPiece<T>::make(v);
    }
    // sum + f(0) + .. + f(V - 1), of the elements that are this lane's.
    template <typename F> __device__ __forceinline__ float add(float sum, const F &f) const
    {
        float t = sum;
#pragma unroll
        for (int i = 0; i < V; ++i) t += f(i);
        if constexpr (OVERLAPS)
            if (cut > 0) {
                t = sum;
#pragma unroll
                for (int i = 0; i < V; ++i) t += i >= cut ? f(i) : 0.f;
            }
        return t;
    }
};

// mean(v^2) + eps of a row in registers as r = 1 / sqrt of it and the power of two k that v was multiplied with: v / rms = (v k) r.
template <int W, int NP, int V, typename P> __device__ __forceinline__ float row_rsqrt(const float (&v)[NP][V], const P &place, int d, float eps, float &k, float *lds)
{
    float ss = 0.f;
#pragma unroll
    for (int c = 0; c < NP; ++c) ss = place(c).add(ss, [&](int i) { return v[c][i] * v[c][i]; });
    float mean = row_sum<W>(ss, lds) / d + eps;
    k = 1.f;
    if (!in_range(mean)) {
        uint32_t top = 0;
#pragma unroll
        for (int c = 0; c < NP; ++c)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const uint32_t a = __float_as_uint(v[c][i]) & 0x7fffffffu;
                top = place(c).mine && a > top ? a : top;   // (a lane behind the row's end may have loaded what another wavefront has stored since)
            }
        k = range_factor(row_max<W>(top, lds), eps);
        ss = 0.f;
#pragma unroll
        for (int c = 0; c < NP; ++c) ss = place(c).add(ss, [&](int i) { return v[c][i] * k * (v[c][i] * k); });
        mean = row_sum<W>(ss, lds) / d + eps * k * k;
    }
    return 1.f / sqrtf(mean);
}

// A row's y as microscaled values: a block of 32 is in 32 / V neighbouring lanes.  Stores of 2 or 4 bytes, 16 apart: 12289 x 768 with a gate per token
// 21.5 us in 4 bits and 22.7 in 8 for 20.6 as bf16 rows (a conversion of its own 5.7 and 7.3), 4096 x 4096 28.3 and 33.5 for 25.2 (8.6 and 10.7).
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

// With 16384 fp32 columns the registers hold a row and not the weights too (LEAN): those are read again for each row, from the caches, and the
// compiler must not take them out of the loop.
template <bool LEAN, typename T> __device__ __forceinline__ const T *per_row(const T *p)
{
    if constexpr (LEAN) asm volatile("" : "+s"(p));
    return p;
}

// A block takes the rows b, b + gridDim.x, .. (W = 1: each of its wavefronts one of four).  gate_ld: 0 for a gate of one row.  sum and y may
// be x or residual: a row's owners have all of it before the first of them stores.
template <typename T, int MODE, int W, int NP, bool MX>
__global__ __launch_bounds__(W == 16 ? 1024 : 256) void block_norm_kernel(const T *x, const T *__restrict__ post, const T *__restrict__ gate, long long gate_ld,
                                                                        const T *residual, float a, const T *__restrict__ pre, T *sum, T *y,
                                                                        uint8_t *__restrict__ mx, uint8_t *__restrict__ mx_scales, int bits,
                                                                        float *__restrict__ stats, int rows, int d, float eps)
{
    constexpr int V = RowPiece<T>::V, LANES = 64 * W, ROWS = W == 1 ? 4 : 1;
    __shared__ float lds[W];
    const int lane = W == 1 ? threadIdx.x & 63 : threadIdx.x;
    const auto place = [&](int c) { return Place<T, MODE>((lane + c * LANES) * V, d); };
    constexpr bool LEAN = W * NP == 64;
    const auto this_row = [](const T *p) { return per_row<LEAN>(p); };
    for (long long row = (long long)blockIdx.x * ROWS + (W == 1 ? threadIdx.x >> 6 : 0); row < rows; row += (long long)gridDim.x * ROWS) {
        const size_t at0 = (size_t)row * d;
        u32x4 px[NP], pr[NP], pg[NP], po[NP], pw[NP];
#pragma unroll
        for (int c = 0; c < NP; ++c) {
            px[c] = place(c).load(x + at0, d);
            pr[c] = place(c).load(residual + at0, d);
        }
        const auto factors = [&] {
            if (gate)
#pragma unroll
                for (int c = 0; c < NP; ++c) pg[c] = place(c).load(this_row(gate) + (size_t)row * gate_ld, d);
            if (post)
#pragma unroll
                for (int c = 0; c < NP; ++c) po[c] = place(c).load(this_row(post), d);
        };
        const auto weights = [&] {
            if (pre)
#pragma unroll
                for (int c = 0; c < NP; ++c) pw[c] = place(c).load(this_row(pre), d);
        };
        if (!LEAN) {
            factors();
            weights();
        }
        float s[NP][V], k1 = 1.f, r1 = 1.f;
#pragma unroll
        for (int c = 0; c < NP; ++c)
#pragma unroll
            for (int i = 0; i < V; ++i) s[c][i] = RowPiece<T>::get(px[c], i);
        if (MODE == kShared) wait_for_loads();   // sum may be x or residual: in front of the row's barrier everybody has its pieces
        if (post) r1 = row_rsqrt<W, NP, V>(s, place, d, eps, k1, lds);
        else if (MODE == kShared) __syncthreads();
        if (LEAN) factors();
#pragma unroll
        for (int c = 0; c < NP; ++c) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float n = s[c][i] * k1 * r1;
                if (post) n *= RowPiece<T>::get(po[c], i);
                if (gate) n *= RowPiece<T>::get(pg[c], i);
                s[c][i] = fmaf(a, RowPiece<T>::get(pr[c], i), n);
            }
            place(c).store(sum + at0, d, s[c]);
        }
        float k2, r2 = row_rsqrt<W, NP, V>(s, place, d, eps, k2, lds);
        if (stats && lane == 0) *(float2 *)(stats + 2 * row) = make_float2(k1 * r1, k2 * r2);
        if (!pre) continue;
        if (LEAN) weights();
#pragma unroll
        for (int c = 0; c < NP; ++c) {
#pragma unroll
            for (int i = 0; i < V; ++i) s[c][i] = s[c][i] * k2 * r2 * RowPiece<T>::get(pw[c], i);
            if (y) place(c).store(y + at0, d, s[c]);
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

// part: [2][gridDim.x][d] column sums of dy n2 and of ds n1 (TOKEN: times the gate).  d_x and d_residual may be d_y and d_sum: a row's owners have all
// of it in front of its first barrier, and store behind that.
template <typename T, int MODE, int W, int NP, bool TOKEN>
__global__ __launch_bounds__(W == 16 ? 1024 : 256, W == 16 ? 4 : 2) void block_norm_backward_kernel(const T *__restrict__ x, const T *__restrict__ post, const T *__restrict__ gate,
                                                                                 const T *__restrict__ sum, const T *__restrict__ pre,
                                                                                 const float *__restrict__ stats, const T *dy, const T *dsum, float a, T *dx,
                                                                                 T *dres, T *dgate, float *__restrict__ part, int rows, int d)
{
    constexpr int V = RowPiece<T>::V, LANES = 64 * W, ROWS = W == 1 ? 4 : 1;
    __shared__ float lds[2][W];
    __shared__ float cols[W == 1 ? 3 : 1][W == 1 ? 64 * V : 1];
    const int lane = W == 1 ? threadIdx.x & 63 : threadIdx.x, wave = threadIdx.x >> 6;
    const auto place = [&](int c) { return Place<T, MODE>((lane + c * LANES) * V, d); };
    constexpr bool LEAN = W * NP == 64, APART = W == 16 && NP > 1;   // APART: a piece's values are unpacked when it is their turn
    u32x4 pw[NP], po[NP], pc[NP], ps[NP], pg[NP], pd[NP], px[NP], pt[TOKEN ? NP : 1];
    // Column sums; of two and more pieces by 1024 lanes in the LDS (a lane's own, 16 bytes at a time: 2 x 64 KB with 16384 columns), for which there
    // are no registers: 1024 rows of 16384 in bf16 took 169 us with them spilled, 70 so.
    constexpr bool IN_LDS = APART;
    float acc[2][IN_LDS ? 1 : NP][V];
    extern __shared__ f32x4 block_norm_columns[];
    const auto slot = [&](int q, int c, int h) { return block_norm_columns + ((q * NP + c) * (V / 4) + h) * LANES + lane; };
    const auto request = [&](long long row) {
        const size_t at0 = (size_t)row * d;
#pragma unroll
        for (int c = 0; c < NP; ++c) {
            ps[c] = place(c).load(sum + at0, d);
            pg[c] = place(c).load(dy + at0, d);
            px[c] = place(c).load(x + at0, d);
            if constexpr (TOKEN) pt[c] = place(c).load(gate + at0, d);
        }
        if (dsum)
#pragma unroll
            for (int c = 0; c < NP; ++c) pd[c] = place(c).load(dsum + at0, d);
    };
    float ones[V];
#pragma unroll
    for (int i = 0; i < V; ++i) ones[i] = 1.f;
    const auto weight = [&](int c) {
        pw[c] = place(c).load(per_row<LEAN>(pre), d);
        po[c] = post ? place(c).load(per_row<LEAN>(post), d) : RowPiece<T>::make(ones);
        if constexpr (!TOKEN) pc[c] = gate ? place(c).load(per_row<LEAN>(gate), d) : RowPiece<T>::make(ones);
    };
    const auto turn = [&] {
        if (APART) __builtin_amdgcn_sched_barrier(0);
    };
#pragma unroll
    for (int c = 0; c < NP; ++c) {
        if (!LEAN) weight(c);
        pd[c] = u32x4{0, 0, 0, 0};
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if constexpr (!IN_LDS) acc[q][c][i] = 0.f;
                else if (i % 4 == 0) *slot(q, c, i / 4) = f32x4{0.f, 0.f, 0.f, 0.f};
            }
    }
    const float inv_d = 1.f / d;
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
        if (W == 16 && !LEAN)
#pragma unroll
            for (int c = 0; c < NP; ++c) {   // (nothing of them is kept unpacked or multiplied)
                keep_packed(pw[c]);
                keep_packed(po[c]);
                if constexpr (!TOKEN) keep_packed(pc[c]);
            }
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
            if (LEAN) pw[c] = place(c).load(per_row<true>(pre), d);
            along = place(c).add(along, [&](int i) { return RowPiece<T>::get(cg[c], i) * RowPiece<T>::get(pw[c], i) * (RowPiece<T>::get(cs[c], i) * r.y); });
            if (APART) {
                keep_packed(cs[c]);
                keep_packed(cg[c]);
            }
            turn();
        }
        if (MODE == kShared) wait_for_loads();   // d_residual may be d_sum, which nobody has used yet
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
            float v[V], u[V];
            if (LEAN) weight(c);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float n2 = RowPiece<T>::get(cs[c], i) * r2, g = RowPiece<T>::get(cg[c], i), n1 = RowPiece<T>::get(cx[c], i) * r1;
                ds[c][i] = RowPiece<T>::get(cd[c], i) + r2 * (g * RowPiece<T>::get(pw[c], i) - n2 * mn2);
                const float gt = TOKEN ? RowPiece<T>::get(ct[TOKEN ? c : 0], i) : RowPiece<T>::get(pc[c], i), dn = ds[c][i] * n1;
                if constexpr (!IN_LDS) {
                    acc[0][c][i] += g * n2;
                    acc[1][c][i] += TOKEN ? dn * gt : dn;
                } else {
                    acc[0][0][i] = g * n2;
                    acc[1][0][i] = TOKEN ? dn * gt : dn;
                }
                u[i] = dn * gt * RowPiece<T>::get(po[c], i);
                v[i] = a * ds[c][i];
            }
            along = place(c).add(along, [&](int i) { return u[i]; });
            if constexpr (IN_LDS)
#pragma unroll
                for (int q = 0; q < 2; ++q)
#pragma unroll
                    for (int h = 0; h < V / 4; ++h) *slot(q, c, h) += f32x4{acc[q][0][4 * h], acc[q][0][4 * h + 1], acc[q][0][4 * h + 2], acc[q][0][4 * h + 3]};
            place(c).store(dres + at0, d, v);
            if constexpr (TOKEN) {
#pragma unroll
                for (int i = 0; i < V; ++i) v[i] = ds[c][i] * (RowPiece<T>::get(cx[c], i) * r1) * RowPiece<T>::get(po[c], i);
                place(c).store(dgate + at0, d, v);
            }
            if (APART) keep_packed(cx[c]);
            turn();
        }
        const float dot = row_sum_once<W>(along, lds[1]), mn1 = post ? dot * inv_d : 0.f;   // without a norm behind the block d_x is m1, and the sum may overflow
#pragma unroll
        for (int c = 0; c < NP; ++c) {
            float v[V];
            if (LEAN) weight(c);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float gt = TOKEN ? RowPiece<T>::get(ct[TOKEN ? c : 0], i) : RowPiece<T>::get(pc[c], i);
                v[i] = r1 * (ds[c][i] * gt * RowPiece<T>::get(po[c], i) - RowPiece<T>::get(cx[c], i) * r1 * mn1);
            }
            place(c).store(dx + at0, d, v);
            turn();
        }
    }
    // the block's column sums; with a row per wavefront the four wavefronts' are added in their order
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        float *out = part + ((size_t)q * gridDim.x + blockIdx.x) * d;
#pragma unroll
        for (int c = 0; c < NP; ++c) {
            const auto at = place(c);
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
                    if (at.mine && i >= at.cut && at.from + i < d) {
                        if constexpr (IN_LDS) out[at.from + i] = (*slot(q, c, i / 4))[i % 4];
                        else out[at.from + i] = acc[q][c][i];
                    }
        }
    }
}

// The sums over the blocks: COLS columns per block, its 1024 / COLS groups of lanes take the partial rows g, g + groups, .., and are added in
// their order.  blockIdx.y = 0: d_pre; 1: d_post and, where the gate is one row, d_gate.
template <typename T, int COLS>
__global__ __launch_bounds__(1024) void block_norm_weight_sum_kernel(const float *__restrict__ part, const T *__restrict__ post, const T *__restrict__ gate /* one row, or null */,
                                                                     float *__restrict__ dpre, float *__restrict__ dpost, float *__restrict__ dgate, int blocks, int d)
{
    constexpr int GROUPS = 1024 / COLS, PER = 64 / COLS;   // and groups in a wavefront
    __shared__ float t[16][COLS];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane % COLS, col = blockIdx.x * COLS + c;
    const float *p = part + (size_t)blockIdx.y * blocks * d;
    float a = 0.f;
    if (col < d)
        for (int b = wave * PER + lane / COLS; b < blocks; b += 16 * GROUPS) {   // sixteen rows in flight
            float v[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = b + GROUPS * i < blocks ? p[(size_t)(b + GROUPS * i) * d + col] : 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) a += v[i];
        }
#pragma unroll
    for (int m = COLS; m < 64; m *= 2) a += __shfl_xor(a, m);
    if (lane < COLS) t[wave][c] = a;
    __syncthreads();
    if (threadIdx.x < COLS && col < d) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) s += t[i][c];
        if (blockIdx.y == 0) dpre[col] = s;
        else {
            if (dpost) dpost[col] = gate ? s * Storage<T>::load(gate + col) : s;
            if (dgate) dgate[col] = post ? s * Storage<T>::load(post + col) : s;
        }
    }
}

// Calls f.run<T, MODE, W, NP>() for a row of d elements: one wavefront to 128 pieces (the forward, which holds less, to 192: 3001 x 513 in fp32 6.8
// us, 7.8 with four), four to 512, then sixteen: with four the rows of 16384 in bf16 spill (1024 of them: 41 us forward, 303 backward; 36 and 70 with
// sixteen).  Backward, a row per wavefront of 513 to 768 fp32 values has one wavefront per SIMD (21.8 us against 15.1).
template <typename T, bool OVERLAP, typename F> static hipError_t pick_block_row(int d, const F &f)
{
    constexpr int V = RowPiece<T>::V;
    const int pieces = (d + V - 1) / V;
    const auto go = [&](auto mode) {
        constexpr int M = decltype(mode)::value;
        const auto wide = [&](auto w, auto np) {
            constexpr int W = decltype(w)::value, NP = decltype(np)::value;
            if constexpr (M == kOverlapped)
                if (pieces % 64 == 1) return f.template run<T, kShared, W, NP>();
            return f.template run<T, M, W, NP>();
        };
        if (pieces <= 64) return f.template run<T, M, 1, 1>();
        if (pieces <= 128) return f.template run<T, M, 1, 2>();
        if constexpr (F::kThree)
            if (pieces <= 192) return f.template run<T, M, 1, 3>();
        if (pieces <= 256) return wide(std::integral_constant<int, 4>(), std::integral_constant<int, 1>());
        if (pieces <= 512) return wide(std::integral_constant<int, 4>(), std::integral_constant<int, 2>());
        if (pieces <= 1024) return wide(std::integral_constant<int, 16>(), std::integral_constant<int, 1>());
        if (V == 8 || pieces <= 2048) return wide(std::integral_constant<int, 16>(), std::integral_constant<int, 2>());
        if constexpr (V == 4) return wide(std::integral_constant<int, 16>(), std::integral_constant<int, 4>());   // (bf16 rows end at 2048 pieces)
        return hipErrorInvalidValue;
    };
    if (d % V == 0) return go(std::integral_constant<int, kAligned>());
    if constexpr (OVERLAP) {
        if (d < V) return f.template run<T, kByElement, 1, 1>();
        return go(std::integral_constant<int, kOverlapped>());
    } else {
        return go(std::integral_constant<int, kByElement>());
    }
}

template <bool MX> struct BlockNormForward {
    static constexpr bool kThree = true;
    const slicemoe_block_norm_config &c;
    const void *x, *post, *gate, *residual, *pre;
    void *sum, *y;
    uint8_t *mx;
    int bits;
    float *stats;
    hipStream_t s;
    template <typename T, int MODE, int W, int NP> hipError_t run() const
    {
        constexpr int threads = W == 16 ? 1024 : 256, per_block = W == 1 ? 4 : 1;
        const int need = c.T / per_block + (c.T % per_block != 0), most = num_compute_units() * 8;
        const unsigned blocks = need < most ? need : most;
        uint8_t *scales = mx ? mx + mx_tiles(c.T, c.d) * mx_tile_bytes(bits) : nullptr;
        const auto kern = block_norm_kernel<T, MODE, W, NP, MX>;
        kern<<<blocks, threads, 0, s>>>((const T *)x, (const T *)post, (const T *)gate, c.gate == SLICEMOE_GATE_TOKEN ? c.d : 0, (const T *)residual,
                                        c.residual_scale, (const T *)pre, (T *)sum, (T *)y, mx, scales, bits, stats, c.T, c.d, c.eps);
        return hipGetLastError();
    }
};

struct BlockNormBackward {
    static constexpr bool kThree = false;
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
    template <typename T, int MODE, int W, int NP> hipError_t run() const
    {
        constexpr int threads = W == 16 ? 1024 : 256;
        const bool token = c.gate == SLICEMOE_GATE_TOKEN;
        const auto kern = token ? block_norm_backward_kernel<T, MODE, W, NP, true> : block_norm_backward_kernel<T, MODE, W, NP, false>;
        constexpr size_t lds = W == 16 && NP > 1 ? 2 * sizeof(float) * 1024 * NP * RowPiece<T>::V : 0;
        if (lds) {
            const hipError_t e = grant_dynamic_lds((const void *)kern, lds);
            if (e != hipSuccess) return e;
        }
        kern<<<blocks, threads, lds, s>>>((const T *)x, (const T *)post, (const T *)gate, (const T *)sum, (const T *)pre, stats, (const T *)dy, (const T *)dsum,
                                        c.residual_scale, (T *)dx, (T *)dres, (T *)dgate, part, c.T, c.d);   // (no rows: writes zeros to part)
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        const int cols = c.d < 2048 ? 16 : 64;   // (both directions of 3001 x 513: 15.1 us with 16, 16.4 with 64; 256 x 4096: 19.5, 16.2)
        const auto add = cols == 16 ? block_norm_weight_sum_kernel<T, 16> : block_norm_weight_sum_kernel<T, 64>;
        add<<<dim3((c.d + cols - 1) / cols, 2), 1024, 0, s>>>(part, (const T *)post, token ? nullptr : (const T *)gate, dpre, dpost,
                                                              token || !gate ? nullptr : (float *)dgate, blocks, c.d);
        return hipGetLastError();
    }
};

// Two blocks of four wavefronts a CU, or one of sixteen: what is resident, so that partial sums are few.  (65536 x 4096 bf16: 613 us with 512 blocks, 690
// with 256, 667 with 1024; 12289 x 768: 31.9, 34.1, 35.3.)
int block_norm_backward_blocks(const slicemoe_block_norm_config &c)
{
    const int V = c.dtype == SLICEMOE_BF16 ? 8 : 4, pieces = (c.d + V - 1) / V, rows = pieces <= 128 ? 4 : 1;
    const int need = c.T / rows + (c.T % rows != 0), most = num_compute_units() * (pieces > 512 ? 1 : 2);
    return need < 1 ? 1 : need < most ? need : most;
}

hipError_t launch_block_norm(const slicemoe_block_norm_config &c, const void *x, const void *post, const void *gate, const void *residual,
                             const void *pre, void *sum, void *y, uint8_t *mx, int bits, float *stats, hipStream_t s)
{
    if (c.T == 0) return hipSuccess;
    const bool bf16 = c.dtype == SLICEMOE_BF16;
    if (mx) {
        const BlockNormForward<true> f{c, x, post, gate, residual, pre, sum, y, mx, bits, stats, s};
        return bf16 ? pick_block_row<bf16_t, false>(c.d, f) : pick_block_row<float, false>(c.d, f);
    }
    const BlockNormForward<false> f{c, x, post, gate, residual, pre, sum, y, mx, bits, stats, s};
    return bf16 ? pick_block_row<bf16_t, true>(c.d, f) : pick_block_row<float, true>(c.d, f);
}

hipError_t launch_block_norm_backward(const slicemoe_block_norm_config &c, const void *x, const void *post, const void *gate, const void *sum,
                                      const void *pre, const float *stats, const void *dy, const void *dsum, void *dx, void *dres,
                                      float *dpost, void *dgate, float *dpre, float *part, hipStream_t s)
{
    const BlockNormBackward f{c, x, post, gate, sum, pre, stats, dy, dsum, dx, dres, dpost, dgate, dpre, part, block_norm_backward_blocks(c), s};
    return c.dtype == SLICEMOE_BF16 ? pick_block_row<bf16_t, true>(c.d, f) : pick_block_row<float, true>(c.d, f);
}

}  // namespace slicemoe
