// Rows of a norm in the registers of the wavefronts that own them (norm.hip, block_norm.hip): pieces of 16 bytes, sums over a row, and the
// range of its squares.
#pragma once
#include <type_traits>

#include "common.h"
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

// Hides where a piece comes from: its values are unpacked again from here on, not kept in registers.
__device__ __forceinline__ void keep_packed(u32x4 &p) { asm volatile("" : "+v"(p)); }

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

}  // namespace slicemoe
