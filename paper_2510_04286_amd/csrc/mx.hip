// Microscaled values (layout and scales: mx.h): conversion of a matrix, and back.
//
// A thread has a block of 32 values: a tile's 32 rows x 8 blocks are the 256 threads of a block.  Bound by memory; a row's eight blocks are
// read by neighbouring lanes, 512 bytes of it together: 16384 x 1024 in bf16 to 4 bits 8.1 us, to 8 bits 10.3 (8.3 and 9.9 at the rate of a copy),
// 11008 x 4096 19.2 and 23.9.  Back, the same pieces are stored in four parts: 33 us, 22 at that rate.  A transposed matrix is read 64 bytes
// of a row at a time, 128 us: a set of weights is converted once.
#include "mx.h"
#include "norm_row.h"

namespace slicemoe {

constexpr int kMxLaunchBlocks = 1 << 20;   // a launch ends below 2^32 threads

// The 32 values of a block, zeros past the end; at: the first column.
template <typename T, bool TRANSPOSED> __device__ __forceinline__ void load_block(const T *__restrict__ x, int row, int at, int rows, int cols, float (&v)[32])
{
    if constexpr (TRANSPOSED) {   // the row is a column of x
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = row < rows && at + i < cols ? Storage<T>::load(x + (size_t)(at + i) * rows + row) : 0.f;
    } else {
        constexpr int V = RowPiece<T>::V;
        const T *r = x + (size_t)(row < rows ? row : 0) * cols;
        u32x4 p[32 / V];
#pragma unroll
        for (int c = 0; c < 32 / V; ++c) p[c] = load_piece<T, false>(r, row < rows ? at + c * V : cols, cols);
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = RowPiece<T>::get(p[i / V], i % V);
    }
}

template <typename T, int BITS, bool TRANSPOSED>
__global__ __launch_bounds__(256) void mx_quantize_kernel(const T *__restrict__ x, uint8_t *__restrict__ values, uint8_t *__restrict__ scales, int rows, int cols,
                                                        int tiles_k, long long tiles)
{
    // lanes along what is contiguous in x
    const int i = TRANSPOSED ? threadIdx.x & 31 : threadIdx.x >> 3, b = TRANSPOSED ? threadIdx.x >> 5 : threadIdx.x & 7;
    const int ks = b >> 1, h = b & 1;
    for (long long t = blockIdx.x; t < tiles; t += gridDim.x) {
        const int row = (int)(t / tiles_k) * kMxRows + i, at = (int)(t % tiles_k) * kMxCols + 32 * b;
        float v[32];
        load_block<T, TRANSPOSED>(x, row, at, rows, cols, v);
        uint32_t most = 0;
#pragma unroll
        for (int q = 0; q < 32; ++q) {
            const uint32_t a = __float_as_uint(v[q]) & 0x7fffffffu;
            most = a > most ? a : most;
        }
        const uint32_t byte = mx_scale_byte<BITS>(most);
        const float inv = mx_inverse(byte);
        uint32_t q[8];   // four columns each, in the order of their positions
#pragma unroll
        for (int m = 0; m < 8; ++m) {
            const int c = 4 * (2 * (m & 3) + (m >> 2));   // position 4 m
            q[m] = mx_pack4<BITS>(v[c] * inv, v[c + 1] * inv, v[c + 2] * inv, v[c + 3] * inv);
        }
        uint8_t *o = values + t * (1024 * BITS);
        if constexpr (BITS == 4)
            *(u32x4 *)(o + 1024 * ks + 16 * (i + 32 * h)) = u32x4{q[0] | q[1] << 16, q[2] | q[3] << 16, q[4] | q[5] << 16, q[6] | q[7] << 16};
        else {
            *(u32x4 *)(o + 2048 * ks + 1024 * h + 16 * i) = u32x4{q[0], q[1], q[2], q[3]};
            *(u32x4 *)(o + 2048 * ks + 1024 * h + 16 * (i + 32)) = u32x4{q[4], q[5], q[6], q[7]};
        }
        scales[t * 256 + 4 * (i + 32 * h) + ks] = (uint8_t)byte;
    }
}

__device__ __forceinline__ float e2m1_value(uint32_t n)
{
    const uint32_t e = n >> 1 & 3, m = n & 1;
    const float v = e ? (float)(2 + m) * (float)(1u << e) * 0.25f : 0.5f * m;
    return n & 8 ? -v : v;
}
__device__ __forceinline__ float e4m3_value(uint32_t n) { return __builtin_amdgcn_cvt_f32_fp8((int)n, 0); }

template <typename T, int BITS, bool TRANSPOSED>
__global__ __launch_bounds__(256) void mx_dequantize_kernel(const uint8_t *__restrict__ values, const uint8_t *__restrict__ scales, T *__restrict__ x, int rows, int cols,
                                                          int tiles_k, long long tiles)
{
    const int i = TRANSPOSED ? threadIdx.x & 31 : threadIdx.x >> 3, b = TRANSPOSED ? threadIdx.x >> 5 : threadIdx.x & 7;
    const int ks = b >> 1, h = b & 1;
    for (long long t = blockIdx.x; t < tiles; t += gridDim.x) {
        const int row = (int)(t / tiles_k) * kMxRows + i, at = (int)(t % tiles_k) * kMxCols + 32 * b;
        if (row >= rows || at >= cols) continue;
        const float scale = mx_value(scales[t * 256 + 4 * (i + 32 * h) + ks]);
        const uint8_t *o = values + t * (1024 * BITS);
        uint32_t q[8];
        if constexpr (BITS == 4) {
            const u32x4 p = *(const u32x4 *)(o + 1024 * ks + 16 * (i + 32 * h));
#pragma unroll
            for (int m = 0; m < 8; ++m) q[m] = p[m >> 1] >> 16 * (m & 1) & 0xffffu;
        } else {
            const u32x4 p = *(const u32x4 *)(o + 2048 * ks + 1024 * h + 16 * i), r = *(const u32x4 *)(o + 2048 * ks + 1024 * h + 16 * (i + 32));
#pragma unroll
            for (int m = 0; m < 8; ++m) q[m] = m < 4 ? p[m & 3] : r[m & 3];
        }
        float v[32];
#pragma unroll
        for (int m = 0; m < 8; ++m)
#pragma unroll
            for (int c = 0; c < 4; ++c)
                v[4 * (2 * (m & 3) + (m >> 2)) + c] = scale * (BITS == 4 ? e2m1_value(q[m] >> 4 * c & 15) : e4m3_value(q[m] >> 8 * c & 255));
        if constexpr (TRANSPOSED) {
#pragma unroll
            for (int c = 0; c < 32; ++c)
                if (at + c < cols) Storage<T>::store(x + (size_t)(at + c) * rows + row, v[c]);
        } else {
            constexpr int V = RowPiece<T>::V;
#pragma unroll
            for (int c = 0; c < 32; c += V)
                if (at + c < cols) store_piece<T, false>(x + (size_t)row * cols, at + c, cols, v + c);
        }
    }
}

// f(T(), Int<BITS>(), transposed)
template <typename F> static hipError_t mx_pick(const slicemoe_mx_config &c, const F &f)
{
    const auto by_bits = [&](auto t, auto tr) {
        return c.bits == 4 ? f(t, std::integral_constant<int, 4>(), tr) : f(t, std::integral_constant<int, 8>(), tr);
    };
    const auto by_order = [&](auto t) { return c.transposed ? by_bits(t, std::true_type()) : by_bits(t, std::false_type()); };
    return c.dtype == SLICEMOE_BF16 ? by_order(bf16_t()) : by_order(float());
}

hipError_t launch_mx_quantize(const slicemoe_mx_config &c, const void *x, uint8_t *mx, hipStream_t s)
{
    const long long tiles = (long long)mx_tiles(c.rows, c.cols);
    if (tiles == 0) return hipSuccess;
    return mx_pick(c, [&](auto t, auto bits, auto tr) {
        mx_quantize_kernel<decltype(t), decltype(bits)::value, decltype(tr)::value><<<(unsigned)(tiles < kMxLaunchBlocks ? tiles : kMxLaunchBlocks), 256, 0, s>>>(
            (const decltype(t) *)x, mx, mx + tiles * mx_tile_bytes(c.bits), c.rows, c.cols, mx_tiles_k(c.cols), tiles);
        return hipGetLastError();
    });
}
hipError_t launch_mx_dequantize(const slicemoe_mx_config &c, const uint8_t *mx, void *x, hipStream_t s)
{
    const long long tiles = (long long)mx_tiles(c.rows, c.cols);
    if (tiles == 0) return hipSuccess;
    return mx_pick(c, [&](auto t, auto bits, auto tr) {
        mx_dequantize_kernel<decltype(t), decltype(bits)::value, decltype(tr)::value><<<(unsigned)(tiles < kMxLaunchBlocks ? tiles : kMxLaunchBlocks), 256, 0, s>>>(
            mx, mx + tiles * mx_tile_bytes(c.bits), (decltype(t) *)x, c.rows, c.cols, mx_tiles_k(c.cols), tiles);
        return hipGetLastError();
    });
}

}  // namespace slicemoe
