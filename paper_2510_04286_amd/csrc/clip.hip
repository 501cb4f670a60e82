// Global norm of a list of gradient tensors, and its bounding.
//
//   norm = sqrt(sum over all tensors of g^2),   factor = min(1, max_norm / (norm + 1e-6)), 1 if max_norm is infinite,   out = g factor
//
// Two launches per kTensors tensors: every block squares and sums one chunk of one tensor, then every block adds up all chunks'
// sums (from L2, the same order in every block and every run) and scales its chunk.  There are kClipChunks of them and one more for each
// tensor at most: from the third table on one block adds them up in between, since blocks times sums grow with the square of a list's
// length (in each block / once, us: 96 tensors of 10000 values 7.8 / 8.9, 193 of 100000 70 / 60, 10000 of 1000 1294 / 806, 100000 of 1000
// 54397 / 9322).  Squares and sums are
// 64-bit: an fp32 value's square is exact there and cannot overflow, and the vector unit has the rate (one fma per four bytes
// read).  The second pass walks chunks, and the pieces of a chunk, backwards: what the first one read last is still in the
// last-level cache.
//
// HBM-bound: each tensor is read twice (less what the cache held) and written once; outputs are stored past the caches.  1.22 GB: 201 +
// 458 us (6.1 and 5.3 TB/s by what a pass has to move; cached stores take 5% more).  Dozens of small tensors are two launches.  A tensor
// whose values the factor does not change and that is scaled in place is not written.
#include <math.h>

#include "clip.h"

namespace slicemoe {

constexpr int kTensors = 96;   // tensors per launch: their table is a kernel argument, below 4 KB
struct ClipTable {
    const void *in[kTensors];
    void *out[kTensors];
    long long n[kTensors];
    int first[kTensors + 1];      // first chunk of each tensor, counted from this launch's first
    unsigned bf16[kTensors / 32]; // storage of tensor i: bit i % 32 of word i / 32
    int count;
    int chunk;                    // elements per chunk, a multiple of 8
};
static_assert(sizeof(ClipTable) < 4000, "kernel arguments hold 4 KB");

struct Chunk {
    int tensor;
    long long begin, end;
    bool bf16;
};
__device__ __forceinline__ Chunk find_chunk(const ClipTable &t, int b)
{
    int lo = 0, hi = t.count;   // first[lo] <= b < first[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (t.first[mid] <= b) lo = mid;
        else hi = mid;
    }
    Chunk c;
    c.tensor = lo;
    c.begin = (long long)(b - t.first[lo]) * t.chunk;
    c.end = c.begin + t.chunk < t.n[lo] ? c.begin + t.chunk : t.n[lo];
    c.bf16 = t.bf16[lo >> 5] >> (lo & 31) & 1;
    return c;
}

typedef u32x4 __attribute__((aligned(2))) loose;   // a tensor may start at any element

__device__ __forceinline__ double block_sum(double v, double *lds)
{
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) v += __shfl_xor(v, m);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = 0.;
#pragma unroll
    for (int i = 0; i < kClipThreads / 64; ++i) s += lds[i];
    return s;
}

template <bool BF16> __device__ __forceinline__ void add_squares(const u32x4 &p, double (&a)[4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (BF16) {
            const double lo = (double)__uint_as_float(p[i] << 16), hi = (double)__uint_as_float(p[i] & 0xffff0000u);
            a[i] = fma(lo, lo, a[i]);
            a[i] = fma(hi, hi, a[i]);
        } else {
            const double v = (double)__uint_as_float(p[i]);
            a[i] = fma(v, v, a[i]);
        }
    }
}

template <bool BF16> __device__ __forceinline__ double chunk_squares(const ClipTable &t, const Chunk &c)
{
    constexpr int V = BF16 ? 8 : 4, EL = BF16 ? 2 : 4, AHEAD = 8;
    const char *base = (const char *)t.in[c.tensor] + c.begin * EL;
    const int n = (int)(c.end - c.begin), whole = n / V;
    double a[4] = {0., 0., 0., 0.};
    int i = threadIdx.x;
    for (; i + (AHEAD - 1) * kClipThreads < whole; i += AHEAD * kClipThreads) {
        u32x4 p[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) p[k] = ((const loose *)base)[i + k * kClipThreads];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) add_squares<BF16>(p[k], a);
    }
    for (; i < whole; i += kClipThreads) {
        const u32x4 p = ((const loose *)base)[i];
        add_squares<BF16>(p, a);
    }
    for (int j = whole * V + threadIdx.x; j < n; j += kClipThreads) {
        const double v = BF16 ? (double)bf16_to_f32(((const bf16_t *)base)[j]) : (double)((const float *)base)[j];
        a[0] = fma(v, v, a[0]);
    }
    return (a[0] + a[1]) + (a[2] + a[3]);
}

__global__ __launch_bounds__(kClipThreads) void clip_squares_kernel(ClipTable t, double *__restrict__ part)
{
    __shared__ double lds[kClipThreads / 64];
    const Chunk c = find_chunk(t, blockIdx.x);
    const double s = block_sum(c.bf16 ? chunk_squares<true>(t, c) : chunk_squares<false>(t, c), lds);
    if (threadIdx.x == 0) part[blockIdx.x] = s;
}

__device__ __forceinline__ float total_norm(const double *__restrict__ part, int parts, double *lds)
{
    double v = 0.;
    for (int i = threadIdx.x; i < parts; i += kClipThreads) v += part[i];
    return (float)sqrt(block_sum(v, lds));
}

template <bool BF16> __device__ __forceinline__ u32x4 scaled(const u32x4 &p, float f)
{
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (BF16)
            r[i] = (uint32_t)f32_to_bf16(__uint_as_float(p[i] << 16) * f) | (uint32_t)f32_to_bf16(__uint_as_float(p[i] & 0xffff0000u) * f) << 16;
        else
            r[i] = __float_as_uint(__uint_as_float(p[i]) * f);
    }
    return r;
}

// part: all chunks' sums, or none: the norm is in *norm already.
template <bool BF16> __device__ __forceinline__ void scale_chunk(const ClipTable &t, const Chunk &c, const double *__restrict__ part, int parts,
                                                                 float max_norm, float *norm_out, bool write_norm, double *lds)
{
    constexpr int V = BF16 ? 8 : 4, EL = BF16 ? 2 : 4, AHEAD = 8;
    const char *base = (const char *)t.in[c.tensor] + c.begin * EL;
    char *out = (char *)t.out[c.tensor];
    const int n = (int)(c.end - c.begin), whole = out ? n / V : 0;
    // from the chunk's end to its beginning; the first pieces are on their way while the norm is added up
    u32x4 p[AHEAD];
    int i = whole - 1 - (int)threadIdx.x;
#pragma unroll
    for (int k = 0; k < AHEAD; ++k)
        if (i - k * kClipThreads >= 0) p[k] = ((const loose *)base)[i - k * kClipThreads];
    const float norm = part ? total_norm(part, parts, lds) : *norm_out;
    const float q = max_norm / (norm + 1e-6f), f = q > 1.f || max_norm == INFINITY ? 1.f : q;   // (a NaN stays one; inf / inf does not)
    if (write_norm && threadIdx.x == 0) *norm_out = norm;
    if (!out || (f == 1.f && t.out[c.tensor] == t.in[c.tensor])) return;
    out += c.begin * EL;
    while (i >= 0) {
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (i - k * kClipThreads >= 0) __builtin_nontemporal_store(scaled<BF16>(p[k], f), (loose *)out + (i - k * kClipThreads));
        i -= AHEAD * kClipThreads;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (i - k * kClipThreads >= 0) p[k] = ((const loose *)base)[i - k * kClipThreads];
    }
    for (int j = whole * V + threadIdx.x; j < n; j += kClipThreads) {
        if constexpr (BF16) ((bf16_t *)out)[j] = f32_to_bf16(bf16_to_f32(((const bf16_t *)base)[j]) * f);
        else ((float *)out)[j] = ((const float *)base)[j] * f;
    }
}

__global__ __launch_bounds__(kClipThreads) void clip_scale_kernel(ClipTable t, const double *__restrict__ part, int parts, float max_norm,
                                                                  float *norm, bool write_norm)
{
    __shared__ double lds[kClipThreads / 64];
    const Chunk c = find_chunk(t, (int)(gridDim.x - 1 - blockIdx.x));
    write_norm = write_norm && blockIdx.x == 0;
    if (c.bf16) scale_chunk<true>(t, c, part, parts, max_norm, norm, write_norm, lds);
    else scale_chunk<false>(t, c, part, parts, max_norm, norm, write_norm, lds);
}

__global__ __launch_bounds__(kClipThreads) void clip_norm_kernel(const double *__restrict__ part, int parts, float *norm_out)
{
    __shared__ double lds[kClipThreads / 64];
    const float norm = total_norm(part, parts, lds);
    if (threadIdx.x == 0) *norm_out = norm;
}

// Elements per chunk: about kClipChunks chunks of all tensors together, at least two pieces of 16 bytes per thread.
ClipPlan clip_plan(const slicemoe_grad *g, int count)
{
    ClipPlan p;
    double total = 0;
    int tensors = 0;
    for (int i = 0; i < count; ++i) {
        total += (double)g[i].n;
        tensors += g[i].n > 0;
    }
    p.once = tensors > 2 * kTensors;
    const double each = ceil(total / kClipChunks / 4096.) * 4096.;
    p.chunk = each < 4096. ? 4096 : each > (double)(1 << 29) ? 1 << 29 : (int)each;
    p.chunks = 0;
    for (int i = 0; i < count; ++i) p.chunks += (g[i].n + p.chunk - 1) / p.chunk;
    return p;
}

hipError_t launch_clip_grads(const slicemoe_grad *g, int count, const ClipPlan &plan, float max_norm, float *norm, double *part, hipStream_t s)
{
    bool scale = false;   // whether any tensor is written
    for (int pass = 0; pass < 2; ++pass) {
        int at = 0, done = 0;
        bool norm_written = plan.once;
        while (done < count) {
            ClipTable t;
            t.count = 0;
            t.chunk = plan.chunk;
            t.first[0] = 0;
            for (unsigned &w : t.bf16) w = 0;
            for (; done < count && t.count < kTensors; ++done) {
                if (g[done].n == 0) continue;
                const int k = t.count++;
                t.in[k] = g[done].grad;
                t.out[k] = g[done].out;
                t.n[k] = g[done].n;
                t.first[k + 1] = t.first[k] + (int)((g[done].n + plan.chunk - 1) / plan.chunk);
                if (g[done].dtype == SLICEMOE_BF16) t.bf16[k >> 5] |= 1u << (k & 31);
                scale = scale || g[done].out;
            }
            if (t.count == 0) break;
            const int blocks = t.first[t.count];
            if (pass == 0) clip_squares_kernel<<<blocks, kClipThreads, 0, s>>>(t, part + at);
            else {
                clip_scale_kernel<<<blocks, kClipThreads, 0, s>>>(t, plan.once ? nullptr : part, (int)plan.chunks, max_norm, norm, !norm_written);
                norm_written = true;
            }
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            at += blocks;
        }
        if (pass == 0 && (plan.once || !scale)) {   // (nothing to scale: the norm alone)
            clip_norm_kernel<<<1, kClipThreads, 0, s>>>(part, (int)plan.chunks, norm);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess || !scale) return e;
        }
    }
    return hipSuccess;
}

}  // namespace slicemoe
