// Products of microscaled matrices on the scaled matrix instruction, and the gated network on them (layout: mx.h).
//
//   product    y = addend + X W^T                          rows X in 4 or 8 bits, features W in 4
//   network    a = silu(x Wg) * (x Wu) as rows in the same bits, y = addend + a Wd
//
// As in the layer's kernels the product is computed transposed: the features are the instruction's first operand, the rows its second, so a lane's
// accumulators are features of one row: 16 of the 32 of a block, the other 16 in lane ^ 32.  The hidden rows' block maximum is thus one exchange
// away, and their values leave as whole pieces in the order the second product reads them.
//
// v_mfma_scale_f32_32x32x64 takes 32 cycles of a SIMD with both operands in 4 bits, 64 with either in 8.
#include <type_traits>

#include "gemm_tile.h"
#include "mx.h"
#include "mx_gemm.h"
#include "norm_row.h"

namespace slicemoe {

// A packed matrix: values, scales, tiles of 256 columns, tiles of 32 rows.
struct MxMatrix {
    const uint8_t *v, *s;
    int tiles;     // of rows
};
static MxMatrix mx_matrix(const void *p, int rows, int cols, int bits)
{
    const uint8_t *v = (const uint8_t *)p;
    return {v, v + mx_tiles(rows, cols) * mx_tile_bytes(bits), (rows + kMxRows - 1) / kMxRows};
}

struct MxArgs {
    MxMatrix x, w, w2;   // w2: the up projection of a pair
    int T, N, Kt;        // rows, features (of one image), tiles of 256 along the contraction
    int tiles_r, tiles_f;   // blocks along the rows, along the features
    // product
    const void *addend;
    void *y;
    // pair: the hidden rows
    uint8_t *h, *hs;
    int hKt;             // their tiles of 256 columns
};

// acc += features (4 bits) x rows (BITS), instruction KS of a tile of 256 columns; fs, rs: the scale words of the lane.
template <int BITS, int KS> __device__ __forceinline__ f32x16 mx_mfma(const i32x8 &f, const i32x8 &r, f32x16 acc, int fs, int rs)
{
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(f, r, acc, 4, BITS == 4 ? 4 : 0, KS, fs, KS, rs);
}
__device__ __forceinline__ i32x8 frag4(const u32x4 &a) { return i32x8{(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0}; }
__device__ __forceinline__ i32x8 frag8(const u32x4 &a, const u32x4 &b)
{
    return i32x8{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]};
}

__device__ __forceinline__ float gated(float g, float u) { return g / (1.f + __expf(-g)) * u; }

// Eight consecutive features f .. f + 7 of a row: addend added, rounded, stored.
template <typename T> __device__ __forceinline__ void store_features(const T *addend, T *y, long long row, int f, int N, const float (&v)[8])
{
    typedef RowPiece<T> P;
    const size_t at = (size_t)row * N + f;
    if (f + 8 <= N) {
        float o[8];
#pragma unroll
        for (int c = 0; c < 8; c += P::V) {
            u32x4 a = {0, 0, 0, 0};
            if (addend) a = *(const loose *)(addend + at + c);
#pragma unroll
            for (int i = 0; i < P::V; ++i) o[c + i] = v[c + i] + (addend ? P::get(a, i) : 0.f);
        }
#pragma unroll
        for (int c = 0; c < 8; c += P::V) *(loose *)(y + at + c) = P::make(o + c);
    } else
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (f + i < N) Storage<T>::store(y + at + i, v[i] + (addend ? Storage<T>::load(addend + at + i) : 0.f));
}

// A block of hidden values: a[p] is position 16 g + p of block kb of a row (the lane's 16 accumulators), the rest is in lane ^ 32.
template <int BITS> __device__ __forceinline__ void store_hidden(const MxArgs &A, int row, int kb, int g, const float (&a)[16])
{
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const uint32_t u = __float_as_uint(a[i]) & 0x7fffffffu;
        most = u > most ? u : most;
    }
    const auto sw = __builtin_amdgcn_permlane32_swap(most, most, false, false);
    most = sw[0] > sw[1] ? sw[0] : sw[1];
    const uint32_t byte = mx_scale_byte<BITS>(most);
    const float inv = mx_inverse(byte);
    uint32_t q[4];
#pragma unroll
    for (int m = 0; m < 4; ++m) q[m] = mx_pack4<BITS>(a[4 * m] * inv, a[4 * m + 1] * inv, a[4 * m + 2] * inv, a[4 * m + 3] * inv);
    uint8_t *o = A.h + mx_quad_offset<BITS>(row, kb, g, A.hKt);   // (columns 4 g: position 16 g)
    if constexpr (BITS == 4) *(uint2 *)o = make_uint2(q[0] | q[1] << 16, q[2] | q[3] << 16);
    else *(u32x4 *)o = u32x4{q[0], q[1], q[2], q[3]};
    if (g == 0) A.hs[mx_scale_offset(row, kb, A.hKt)] = (uint8_t)byte;
}

// ------------------------------------------------------------------------------ tiles
// One block of four wavefronts, 2 x 2, each with TR x TF fragments of 32 rows and features.  DUAL: half of a wavefront's feature tiles
// come from w, half from w2.  A step is 128 bytes of a row: 256 columns in 4 bits, 128 in 8; its images come straight from memory to the
// LDS as linear kilobytes and are read as they lie.  A ring of SLOTS images; one barrier per step, a fragment before its end: behind it
// the next step's images have landed for every wavefront, and the present ones, whose last fragments are in registers, are free for the
// step SLOTS ahead.
template <int BITS_, bool DUAL_, int TR_, int TF_> struct MxTile {
    static constexpr int BITS = BITS_, TR = TR_, TF = TF_;
    static constexpr bool DUAL = DUAL_;
    static constexpr int IMAGES = DUAL ? 2 : 1, FT = TF / IMAGES;      // feature tiles of one image per wavefront
    static constexpr int RT = 2 * TR, FB = 2 * TF;                     // tiles of 32 per block: rows, features (of all images)
    static constexpr int BR = 32 * RT, BF = 32 * FB / IMAGES;          // rows, features of one image per block
    static constexpr int KS = BITS == 4 ? 4 : 2;                       // instructions along a step
    static constexpr int F_TILE = KS * 1024;                           // bytes of a feature tile in a step; a row tile: 4096
    static constexpr int R_BYTES = RT * 4096, F_BYTES = FB * F_TILE, S_BYTES = (RT + FB) * 256;
    static constexpr int SLOT = R_BYTES + F_BYTES + S_BYTES;
    static constexpr int SLOTS = BITS == 4 ? 2 : 3;
    static constexpr int LDS = SLOTS * SLOT;
    static constexpr int R_TILES = RT / 4, F_TILES = FB / 4;           // tiles that a wavefront requests
    static constexpr int LOADS = 4 * R_TILES + KS * F_TILES + 1;       // instructions per wavefront and step
    static_assert(RT % 4 == 0 && FB % 4 == 0 && (RT + FB == 16 || RT + FB == 8), "scales: a kilobyte per wavefront, or per pair of them");
    static_assert(LDS <= 160 * 1024, "");
};

template <typename S> __device__ __forceinline__ void mx_steps(f32x16 (&acc)[S::TF][S::TR], const MxArgs &A, int r0, int f0, char *lds)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wr = wave >> 1, wf = wave & 1;
    const int steps = A.Kt * (4 / S::KS);
    const uint32_t lds0 = (uint32_t)(uintptr_t)as_lds(lds);
    // tile i of the block's features: image 0's, then image 1's
    const auto feature_tile = [&](int i) {
        const int per = S::FB / S::IMAGES, t = f0 + i % per;
        return t < A.w.tiles ? t : A.w.tiles - 1;
    };
    const uint8_t *rp[S::R_TILES], *fp[S::F_TILES];
#pragma unroll
    for (int i = 0; i < S::R_TILES; ++i) {
        const int t = r0 + wave * S::R_TILES + i;
        rp[i] = A.x.v + (size_t)(t < A.x.tiles ? t : A.x.tiles - 1) * A.Kt * (1024 * S::BITS);
    }
#pragma unroll
    for (int i = 0; i < S::F_TILES; ++i) {
        const int t = wave * S::F_TILES + i;
        fp[i] = (S::DUAL && t >= S::FB / 2 ? A.w2.v : A.w.v) + (size_t)feature_tile(t) * A.Kt * 4096;
    }
    // Scales: a kilobyte is four tiles; the block's RT row tiles, then its FB feature tiles.  (128 x 128 tiles: two kilobytes, each twice.)
    constexpr int S_KB = S::S_BYTES / 1024;
    const int sk = wave % S_KB;
    const uint8_t *sp;
    {
        const int st = 4 * sk + (lane >> 4), t = r0 + st, f = st - S::RT;
        const bool rows = st < S::RT;
        const size_t tile = rows ? (t < A.x.tiles ? t : A.x.tiles - 1) : feature_tile(f);
        sp = (rows ? A.x.s : S::DUAL && f >= S::FB / 2 ? A.w2.s : A.w.s) + tile * A.Kt * 256 + 16 * (lane & 15);
    }
    const uint32_t lane16 = 16 * lane;
    int at = 0, slot = 0;   // of the next request
    const auto request = [&](auto index) {
        constexpr int I = decltype(index)::value;
        const uint32_t to = lds0 + slot * S::SLOT;
        if constexpr (I < S::F_TILES * S::KS) {
            constexpr int i = I / S::KS, q = I % S::KS;
            if constexpr (q == 0) set_lds_target(to + S::R_BYTES + (wave * S::F_TILES + i) * S::F_TILE);
            load_lds_1k<1024 * q>((const char *)fp[i], lane16);
        } else if constexpr (I < S::F_TILES * S::KS + 4 * S::R_TILES) {
            constexpr int i = (I - S::F_TILES * S::KS) / 4, q = (I - S::F_TILES * S::KS) % 4;
            if constexpr (q == 0) set_lds_target(to + (wave * S::R_TILES + i) * 4096);
            load_lds_1k<1024 * q>((const char *)rp[i], lane16);
        } else {
            set_lds_target(to + S::R_BYTES + S::F_BYTES + 1024 * sk);
            load_lds_1k<0>((const char *)(sp + (size_t)(at >> (S::KS == 4 ? 0 : 1)) * 256));
        }
    };
    const auto requested = [&]() {
        ++at;
        slot = slot + 1 == S::SLOTS ? 0 : slot + 1;
#pragma unroll
        for (int i = 0; i < S::R_TILES; ++i) rp[i] += 4096;
#pragma unroll
        for (int i = 0; i < S::F_TILES; ++i) fp[i] += S::F_TILE;
    };

    typedef typename std::conditional<S::BITS == 4, u32x4, i32x8>::type rfrag;
    rfrag rf[2][S::TR];
    u32x4 ff[2][S::TF];
    int rs[S::TR], fs[S::TF], rn[S::TR], fn[S::TF];   // scale words of this step, and of the next
    int cur = 0, odd = 0;                             // slot being read; 8 bits: which half of a tile of 256 columns it is
    const auto read = [&](int set, int ks, int i) {   // fragment i of instruction ks: the first features', all rows', the other features'
        const char *image = lds + cur * S::SLOT;
        if (i >= 1 && i <= S::TR) {
            const char *p = image + (wr * S::TR + i - 1) * 4096 + lane16;
            if constexpr (S::BITS == 4) rf[set][i - 1] = *(const u32x4 *)(p + 1024 * ks);
            else rf[set][i - 1] = frag8(*(const u32x4 *)(p + 2048 * ks), *(const u32x4 *)(p + 2048 * ks + 1024));
        } else {
            const int t = i == 0 ? 0 : i - S::TR;
            const int in = t < S::FT ? wf * S::FT + t : S::FB / 2 + wf * S::FT + t - S::FT;
            ff[set][t] = *(const u32x4 *)(image + S::R_BYTES + in * S::F_TILE + 1024 * ks + lane16);
        }
    };
    const auto read_scales = [&]() {
        const char *p = lds + cur * S::SLOT + S::R_BYTES + S::F_BYTES + 4 * lane;
#pragma unroll
        for (int u = 0; u < S::TR; ++u) rn[u] = *(const int *)(p + (wr * S::TR + u) * 256);
#pragma unroll
        for (int t = 0; t < S::TF; ++t)
            fn[t] = *(const int *)(p + (S::RT + (t < S::FT ? wf * S::FT + t : S::FB / 2 + wf * S::FT + t - S::FT)) * 256);
    };
    const auto take_scales = [&]() {   // (the instruction's byte is a constant: the second half's two are moved down)
        const int shift = S::BITS == 8 ? 16 * odd : 0;
#pragma unroll
        for (int u = 0; u < S::TR; ++u) rs[u] = (int)((uint32_t)rn[u] >> shift);
#pragma unroll
        for (int t = 0; t < S::TF; ++t) fs[t] = (int)((uint32_t)fn[t] >> shift);
    };
    constexpr int NM = S::TR * S::TF, NF = S::TR + S::TF;
    // The matrix instructions of index K along the step, with the reads of the next and the requests [FROM, TO) between them.
    const auto part = [&](auto k, auto reads, int next, auto from, auto to) {
        constexpr int K = decltype(k)::value, FROM = decltype(from)::value, TO = decltype(to)::value;
        constexpr bool READS = decltype(reads)::value;
        for_range<0, NM>([&](auto mm) {
            constexpr int M = decltype(mm)::value, t = M / S::TR, u = M % S::TR;
            i32x8 r;
            if constexpr (S::BITS == 4) r = frag4(rf[K & 1][u]);
            else r = rf[K & 1][u];
            acc[t][u] = mx_mfma<S::BITS, K>(frag4(ff[K & 1][t]), r, acc[t][u], fs[t], rs[u]);
            if constexpr (READS)
#pragma unroll
                for (int i = M * NF / NM; i < (M + 1) * NF / NM; ++i) read((K + 1) & 1, next, i);
            for_range<FROM + M *(TO - FROM) / NM, FROM + (M + 1) * (TO - FROM) / NM>(request);
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    constexpr Int<0> none = {};
    constexpr Int<S::LOADS> all = {};
    constexpr Int<S::LOADS / 2> half = {};
    typedef std::true_type Yes;
    typedef std::false_type No;
    // A step.  REST: it begins with the second half of the requests of the step SLOTS - 1 ahead; behind its barrier, in front of its last
    // part, follow (ASKS) the first half of the step SLOTS ahead.  NEXT: there is a next step.
    const auto step = [&](auto rest, auto asks, auto nxt) {
        constexpr bool REST = decltype(rest)::value, ASKS = decltype(asks)::value, NEXT = decltype(nxt)::value;
        for_range<0, S::KS - 1>([&](auto k) {
            constexpr int K = decltype(k)::value;
            if constexpr (REST && K == 0) {
                part(k, Yes(), K + 1, half, all);
                requested();
            } else
                part(k, Yes(), K + 1, none, none);
        });
        constexpr Int<S::KS - 1> last = {};
        if constexpr (NEXT) {
            wait_loads_and_barrier<REST ? (S::SLOTS - 2) * S::LOADS : 0>();   // all but what was requested behind the next step's images
            cur = cur + 1 == S::SLOTS ? 0 : cur + 1;
            read_scales();
            if constexpr (ASKS) part(last, Yes(), 0, none, half);
            else part(last, Yes(), 0, none, none);
            odd ^= 1;
            take_scales();
        } else
            part(last, No(), 0, none, none);
    };
    for (int i = 0; i < S::SLOTS - 1 && i < steps; ++i) {
        for_range<0, S::LOADS>(request);
        requested();
    }
    if (steps >= S::SLOTS) {
        for_range<0, S::LOADS / 2>(request);
        wait_loads_and_barrier<(S::SLOTS - 2) * S::LOADS + S::LOADS / 2>();
    } else
        wait_loads_and_barrier<0>();
    read_scales();
    take_scales();
#pragma unroll
    for (int i = 0; i < NF; ++i) read(0, 0, i);
    int left = steps - S::SLOTS;
    for (; left > 0; --left) step(Yes(), Yes(), Yes());
    if (left == 0) step(Yes(), No(), Yes());
    if (S::SLOTS == 3 && steps >= 2) step(No(), No(), Yes());
    step(No(), No(), No());
}

template <typename S, typename T> __global__ __launch_bounds__(256, 1) void mx_tile_kernel(MxArgs A)
{
    extern __shared__ __align__(1024) char lds[];
    const TilePlace place = tile_of(blockIdx.x, A.tiles_r, A.tiles_f, 1);
    const int r0 = place.r * S::RT, f0 = place.f * (S::FB / S::IMAGES);   // tiles of 32
    f32x16 acc[S::TF][S::TR];
#pragma unroll
    for (int t = 0; t < S::TF; ++t)
#pragma unroll
        for (int u = 0; u < S::TR; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[t][u][i] = 0.f;
    mx_steps<S>(acc, A, r0, f0, lds);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wr = wave >> 1, wf = wave & 1, j = lane & 31, g = lane >> 5;
#pragma unroll
    for (int u = 0; u < S::TR; ++u) {
        const int rt = r0 + wr * S::TR + u;
        if (rt >= A.x.tiles) continue;
        const int row = 32 * rt + j;
#pragma unroll
        for (int t = 0; t < S::FT; ++t) {
            const int ft = f0 + wf * S::FT + t;
            if constexpr (S::DUAL) {
                if (ft >= 8 * A.hKt) continue;
                float a[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float v = gated(acc[t][u][i], acc[S::FT + t][u][i]);
                    a[i] = 32 * ft + acc_feature(i, g) < A.N ? v : 0.f;   // (what is past the last row of the weights is anything)
                }
                store_hidden<S::BITS>(A, row, ft, g, a);
            } else {
#pragma unroll
                for (int q = 0; q < 2; ++q) {   // lanes j and j + 32 trade halves: each has eight consecutive features of its row
                    float v[8];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc[t][u][8 * q + i]), __float_as_uint(acc[t][u][8 * q + 4 + i]), false, false);
                        v[i] = __uint_as_float(sw[0]);
                        v[4 + i] = __uint_as_float(sw[1]);
                    }
                    const int f = 32 * ft + 16 * q + 8 * g;
                    if (row < A.T) store_features<T>((const T *)A.addend, (T *)A.y, row, f, A.N, v);
                }
            }
        }
    }
}

template <typename S, typename T> static hipError_t run_tiles(MxArgs A, int f_tiles, hipStream_t s)
{
    A.tiles_r = (A.x.tiles + S::RT - 1) / S::RT;
    A.tiles_f = (f_tiles + S::FB / S::IMAGES - 1) / (S::FB / S::IMAGES);
    const auto kern = mx_tile_kernel<S, T>;
    const hipError_t e = grant_dynamic_lds((const void *)kern, S::LDS);
    if (e != hipSuccess) return e;
    kern<<<(unsigned)(A.tiles_r * A.tiles_f), 256, S::LDS, s>>>(A);
    return hipGetLastError();
}

template <int BITS, bool DUAL, typename T> static hipError_t run_product(const MxArgs &A, hipStream_t s)
{
    const int f_tiles = DUAL ? 8 * A.hKt : A.w.tiles;
    return run_tiles<MxTile<BITS, DUAL, 4, 4>, T>(A, f_tiles, s);
}

size_t mx_product_workspace(const slicemoe_mx_product_config &c) { return 0; }

hipError_t launch_mx_product(const slicemoe_mx_product_config &c, const uint8_t *x, const uint8_t *w, const void *addend, void *y, char *ws, hipStream_t s)
{
    if (c.T == 0) return hipSuccess;
    MxArgs A = {};
    A.x = mx_matrix(x, c.T, c.K, c.bits);
    A.w = mx_matrix(w, c.N, c.K, 4);
    A.T = c.T;
    A.N = c.N;
    A.Kt = mx_tiles_k(c.K);
    A.addend = addend;
    A.y = y;
    if (c.bits == 4) return c.dtype == SLICEMOE_BF16 ? run_product<4, false, bf16_t>(A, s) : run_product<4, false, float>(A, s);
    return c.dtype == SLICEMOE_BF16 ? run_product<8, false, bf16_t>(A, s) : run_product<8, false, float>(A, s);
}

size_t gated_mx_workspace(const slicemoe_gated_config &c, int bits)
{
    return align_up(mx_total_bytes(c.T, c.H, bits), 256) + 256;   // (never 0)
}

hipError_t launch_gated_mx(const slicemoe_gated_config &c, int bits, const uint8_t *x, const slicemoe_gated_weights_mx &w, const void *addend, void *y,
                           char *ws, hipStream_t s)
{
    if (c.T == 0) return hipSuccess;
    MxArgs A = {};
    A.x = mx_matrix(x, c.T, c.d, bits);
    A.w = mx_matrix(w.Wg, c.H, c.d, 4);
    A.w2 = mx_matrix(w.Wu, c.H, c.d, 4);
    A.T = c.T;
    A.N = c.H;
    A.Kt = mx_tiles_k(c.d);
    A.h = (uint8_t *)ws;
    A.hs = A.h + mx_tiles(c.T, c.H) * mx_tile_bytes(bits);
    A.hKt = mx_tiles_k(c.H);
    const hipError_t e = bits == 4 ? run_product<4, true, bf16_t>(A, s) : run_product<8, true, bf16_t>(A, s);
    if (e != hipSuccess) return e;
    const slicemoe_mx_product_config p = {c.T, c.H, c.d, bits, SLICEMOE_BF16};
    return launch_mx_product(p, A.h, (const uint8_t *)w.Wd, addend, y, ws, s);
}

}  // namespace slicemoe
