// Microscaled values: 32 consecutive columns of a row share a power of two, each is an e2m1 (4 bits) or e4m3 (8 bits) value times it.
// How they lie in memory, and the conversion of a block; shared by the conversions and products (mx.hip) and the norm that writes
// them (block_norm.hip).
//
// Layout: tiles of 32 rows x 256 columns in the order of the matrix instruction (v_mfma_scale_f32_32x32x64_f8f6f4: lane i + 32 g has 32
// values of row i), so that an operand is loaded, straight or through the LDS, by linear kilobytes.  Tile (rt, kt) is number rt Kt + kt,
// Kt = ceil(cols / 256); what is past the last column is zero.  In a tile, column c has the block c / 32, blocks 2 ks and 2 ks + 1 belong to
// instruction ks, and stands at position p = 16 (c / 4 % 2) + 4 (c / 8 % 4) + c % 4 of its block:
//   4 bits   [ks][lane i + 32 (block % 2)][16 bytes], position p in nibble p: the instruction takes 32 values of one block per lane
//   8 bits   [ks][block % 2][lane i + 32 (p / 16)][16 bytes], position p in byte p % 16: it takes 16 values of each of two blocks per lane
//   scales   behind all values, [tile][lane i + 32 (block % 2)][byte ks]: e + 127 of the block's 2^e, 255 for NaN
// The positions are the order in which an accumulator's lane holds the features of its row (acc_feature), so the hidden rows of the
// gated network leave the accumulators as whole pieces; a sum over columns does not mind their order.
#pragma once
#include "common.h"
#include "mfma.h"
#include "norm.h"

namespace slicemoe {

constexpr int kMxRows = 32, kMxCols = 256;
__host__ __device__ __forceinline__ int mx_tiles_k(int cols) { return (cols + kMxCols - 1) / kMxCols; }
__host__ __device__ __forceinline__ size_t mx_tiles(int rows, int cols) { return (size_t)((rows + kMxRows - 1) / kMxRows) * mx_tiles_k(cols); }
__host__ __device__ __forceinline__ size_t mx_tile_bytes(int bits) { return (size_t)kMxRows * kMxCols / 8 * bits; }
__host__ __device__ __forceinline__ size_t mx_total_bytes(int rows, int cols, int bits) { return mx_tiles(rows, cols) * (mx_tile_bytes(bits) + 256); }

// The scale byte of a block whose largest magnitude has the bits `most`: the least power of two that brings it to at most 6 = 1.5 2^2 (448 =
// 1.75 2^8), so nothing saturates; at least 2^-127.  255 where the block holds an infinity or a NaN.
template <int BITS> __device__ __forceinline__ uint32_t mx_scale_byte(uint32_t most)
{
    const int x = (int)(most >> 23), up = (most & 0x7fffffu) > (BITS == 4 ? 0x400000u : 0x600000u) ? 1 : 0;
    const int e = x - (BITS == 4 ? 2 : 8) + up;
    return x == 255 ? 255u : e < 0 ? 0u : (uint32_t)e;
}
// 2^-e of a scale byte (255: any number).  Below the smallest normal number (e = 127) never: a byte is at most 253.
__device__ __forceinline__ float mx_inverse(uint32_t byte) { return __uint_as_float((254u - (byte > 253u ? 253u : byte)) << 23); }
__device__ __forceinline__ float mx_value(uint32_t byte) { return byte == 255u ? __uint_as_float(0x7fc00000u) : byte == 0 ? 0x1p-127f : __uint_as_float(byte << 23); }

// Four values (already times 2^-e) as 16 bits of e2m1 or 32 bits of e4m3, rounded to nearest even.
__device__ __forceinline__ uint32_t pack_e2m1(float a, float b, float c, float d)
{
    uint32_t p = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, a, b, 1.f, 0);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(p, c, d, 1.f, 1) & 0xffffu;
}
template <int BITS> __device__ __forceinline__ uint32_t mx_pack4(float a, float b, float c, float d)
{
    if constexpr (BITS == 4) return pack_e2m1(a, b, c, d);
    else return pack_e4m3(a, b, c, d);
}

// Byte offset of the four columns 4 m .. 4 m + 3 (m: 0 .. 7) of block kb of a row, and of its scale (from the scales' start).
template <int BITS> __device__ __forceinline__ size_t mx_quad_offset(int row, int kb, int m, int tiles_k)
{
    const size_t tile = (size_t)(row >> 5) * tiles_k + (kb >> 3);
    const int i = row & 31, ks = kb >> 1 & 3, b = kb & 1, p = 16 * (m & 1) + 4 * (m >> 1);
    if constexpr (BITS == 4) return tile * 4096 + ks * 1024 + (i + 32 * b) * 16 + (p >> 1);
    else return tile * 8192 + ks * 2048 + b * 1024 + (i + 32 * (p >> 4)) * 16 + (p & 15);
}
__device__ __forceinline__ size_t mx_scale_offset(int row, int kb, int tiles_k)
{
    return ((size_t)(row >> 5) * tiles_k + (kb >> 3)) * 256 + ((row & 31) + 32 * (kb & 1)) * 4 + (kb >> 1 & 3);
}

}  // namespace slicemoe
