// Products of microscaled matrices on the scaled matrix instruction, and the gated network on them (layout: mx.h).
//
//   product    y = addend + X W^T                          rows X in 4 or 8 bits, features W in 4
//   network    a = silu(x Wg) * (x Wu) as rows in the same bits, y = addend + a Wd
//
// As in the layer's kernels the product is computed transposed: the features are the instruction's first operand, the rows its second, so a lane's
// accumulators are features of one row: 16 of the 32 of a block, the other 16 in lane ^ 32.  The hidden rows' block maximum is thus one exchange
// away, and their values leave as whole pieces in the order the second product reads them.
//
// v_mfma_scale_f32_32x32x64 takes 32 cycles of a SIMD with both operands in 4 bits, 64 with either in 8; with random values in the operands the
// chip's power limit allows 6.1 and 3.7 PFLOP/s from registers alone (zeros: 8.8).
//
// Up to 64 rows, bound by the weights, one pass over them straight to the registers (16 rows in 8 bits, the network with d 4096, H 11008: 12.6 + 7.0 us for 45
// and 22.5 MB); else tiles of 128 x 128 and 256 x 256 through the LDS (4096 rows, 4096 x 11008 in 4 bits, medians of 64 passes: the pair 201 us = 3.7
// PFLOP/s, the second product 83 = 4.4).  Wide results and short contractions are bound by the results: 16384 x 1024 x 2816 with an addend takes 53 us in one
// process and 65 in another (least 52 in both), its 184 MB of addend and y 36 at the rate of a copy.
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
    int tiles_r, tiles_f, splits;   // blocks along the rows, along the features, shares of the contraction
    // product
    const void *addend;
    void *y;             // shares: the sums of each, [splits][T][N] float
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

// Rows of 8 bits in two parts.  The instruction adds the products of eight columns in the place of the largest and drops what is below 2^-13 of it: some
// 1e-5 of the magnitudes that are added up, nothing beside the rounding of bf16 storage, but a hundred times fp32's.  With fp32 storage (WHOLE) the values of
// 4 and more (products of 2^1 .. 2^11.4, in steps of 2^-2: all of their bits are kept) and the others (below 2^4.6; at most the bit 2^-10 of values below
// 2^-5 is lost) are multiplied one after the other: `small` are the others, the large ones stay in r.  us with an addend, one instruction / two: 16 rows 11008
// 4096 7.8 / 8.2, 64 rows 4096 4096 6.8 / 9.1, 200 4096 4096 13.5 / 21.8, 1024 2816 1024 11.7 / 21, 4096 11008 4096 142 / 219, 16384 1024 2816 93 / 112.
template <int BITS, typename T> constexpr bool kMxWhole = BITS == 8 && std::is_same<T, float>::value;
__device__ __forceinline__ void split_word(i32x8 &r, i32x8 &small, int i)
{
    const uint32_t v = (uint32_t)r[i], over = (v & 0x7f7f7f7fu) + 0x38383838u;   // a byte's sign bit: its magnitude is 0x48 = 2^2 or more
    const uint32_t large = v & __builtin_amdgcn_perm(over << 8, over, 0x090b080au);   // (each byte the sign of one of `over`)
    r[i] = (int)large;
    small[i] = (int)(v ^ large);
}
__device__ __forceinline__ i32x8 small_part(i32x8 &r)
{
    i32x8 small;
#pragma unroll
    for (int i = 0; i < 8; ++i) split_word(r, small, i);
    return small;
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
// come from w, half from w2.  A step is KS instructions of 64 columns (256 columns, or 128); its images come straight from memory to the
// LDS as linear kilobytes and are read as they lie.  A ring of SLOTS images; one barrier per step, a fragment before its end: behind it
// the next step's images have landed for every wavefront, and the present ones, whose last fragments are in registers, are free for the
// step SLOTS ahead.
template <int BITS_, bool DUAL_, int TR_, int TF_, int KS_, int SLOTS_, bool WHOLE_> struct MxTile {
    static constexpr int BITS = BITS_, TR = TR_, TF = TF_;
    static constexpr bool DUAL = DUAL_, WHOLE = WHOLE_;
    static constexpr int IMAGES = DUAL ? 2 : 1, FT = TF / IMAGES;      // feature tiles of one image per wavefront
    static constexpr int RT = 2 * TR, FB = 2 * TF;                     // tiles of 32 per block: rows, features (of all images)
    static constexpr int BR = 32 * RT, BF = 32 * FB / IMAGES;          // rows, features of one image per block
    static constexpr int KS = KS_;                                     // instructions along a step
    static constexpr int F_TILE = KS * 1024, R_TILE = F_TILE * BITS / 4;   // bytes of a tile in a step: features, rows
    static constexpr int R_KB = R_TILE / 1024;
    static constexpr int R_BYTES = RT * R_TILE, F_BYTES = FB * F_TILE, S_BYTES = (RT + FB) * 256;
    static constexpr int SLOT = R_BYTES + F_BYTES + S_BYTES;
    static constexpr int SLOTS = SLOTS_;
    static constexpr int LDS = SLOTS * SLOT;
    static constexpr int R_TILES = RT / 4, F_TILES = FB / 4;           // tiles that a wavefront requests
    static constexpr int LOADS = R_KB * R_TILES + KS * F_TILES + 1;       // instructions per wavefront and step
    static_assert(RT % 4 == 0 && FB % 4 == 0 && RT + FB <= 16, "scales: a kilobyte per wavefront at most");
    static constexpr int PER_CU = 160 * 1024 / LDS, PER_SIMD = PER_CU < 1 ? 1 : PER_CU > 3 ? 3 : PER_CU;   // blocks, wavefronts
    static_assert(LDS <= 160 * 1024, "");
};

template <typename S> __device__ __forceinline__ void mx_steps(f32x16 (&acc)[S::TF][S::TR], const MxArgs &A, int r0, int f0, int k0, int k1, char *lds)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wr = wave >> 1, wf = wave & 1;
    const int steps = (k1 - k0) * (4 / S::KS);   // tiles [k0, k1) of 256 columns
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
        rp[i] = A.x.v + ((size_t)(t < A.x.tiles ? t : A.x.tiles - 1) * A.Kt + k0) * (1024 * S::BITS);
    }
#pragma unroll
    for (int i = 0; i < S::F_TILES; ++i) {
        const int t = wave * S::F_TILES + i;
        fp[i] = (S::DUAL && t >= S::FB / 2 ? A.w2.v : A.w.v) + ((size_t)feature_tile(t) * A.Kt + k0) * 4096;
    }
    // Scales: a kilobyte is four tiles; the block's RT row tiles, then its FB feature tiles.  (Fewer than four kilobytes: some twice.)
    constexpr int S_KB = S::S_BYTES / 1024;
    const int sk = wave % S_KB;
    const uint8_t *sp;
    {
        const int st = 4 * sk + (lane >> 4), t = r0 + st, f = st - S::RT;
        const bool rows = st < S::RT;
        const size_t tile = rows ? (t < A.x.tiles ? t : A.x.tiles - 1) : feature_tile(f);
        sp = (rows ? A.x.s : S::DUAL && f >= S::FB / 2 ? A.w2.s : A.w.s) + (tile * A.Kt + k0) * 256 + 16 * (lane & 15);
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
        } else if constexpr (I < S::F_TILES * S::KS + S::R_KB * S::R_TILES) {
            constexpr int i = (I - S::F_TILES * S::KS) / S::R_KB, q = (I - S::F_TILES * S::KS) % S::R_KB;
            if constexpr (q == 0) set_lds_target(to + (wave * S::R_TILES + i) * S::R_TILE);
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
        for (int i = 0; i < S::R_TILES; ++i) rp[i] += S::R_TILE;
#pragma unroll
        for (int i = 0; i < S::F_TILES; ++i) fp[i] += S::F_TILE;
    };

    typedef typename std::conditional<S::BITS == 4, u32x4, i32x8>::type rfrag;
    rfrag rf[2][S::TR];
    i32x8 small[2][S::WHOLE ? S::TR : 1];
    u32x4 ff[2][S::TF];
    int rs[S::TR], fs[S::TF], rn[S::TR], fn[S::TF];   // scale words of this step, and of the next
    int cur = 0, odd = 0;                             // slot being read; 8 bits: which half of a tile of 256 columns it is
    const auto read = [&](int set, int ks, int i) {   // fragment i of instruction ks: the first features', all rows', the other features'
        const char *image = lds + cur * S::SLOT;
        if (i >= 1 && i <= S::TR) {
            const char *p = image + (wr * S::TR + i - 1) * S::R_TILE + lane16;
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
        const int shift = S::KS == 2 ? 16 * odd : 0;
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
        constexpr int ALL = S::WHOLE ? 2 * NM : NM;   // (in two parts: the next fragments are read in the first half and taken apart in the second)
        for_range<0, ALL>([&](auto mm) {
            constexpr int M = decltype(mm)::value, t = M % NM / S::TR, u = M % S::TR;
            i32x8 r;
            if constexpr (S::BITS == 4) r = frag4(rf[K & 1][u]);
            else if constexpr (M < NM) r = rf[K & 1][u];
            else r = small[K & 1][u];
            acc[t][u] = mx_mfma<S::BITS, K>(frag4(ff[K & 1][t]), r, acc[t][u], fs[t], rs[u]);
            if constexpr (READS && M < NM)
#pragma unroll
                for (int i = M * NF / NM; i < (M + 1) * NF / NM; ++i) read((K + 1) & 1, next, i);
            if constexpr (S::WHOLE)
                if constexpr (READS && M >= NM) {
                    constexpr int W = 8 * S::TR;
#pragma unroll
                    for (int i = (M - NM) * W / NM; i < (M - NM + 1) * W / NM; ++i) split_word(rf[(K + 1) & 1][i / 8], small[(K + 1) & 1][i / 8], i % 8);
                }
            for_range<FROM + M *(TO - FROM) / ALL, FROM + (M + 1) * (TO - FROM) / ALL>(request);
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
    if constexpr (S::WHOLE)
#pragma unroll
        for (int u = 0; u < S::TR; ++u) small[0][u] = small_part(rf[0][u]);
    int left = steps;
    for (; left > S::SLOTS; --left) step(Yes(), Yes(), Yes());
    if (left == S::SLOTS) {
        step(Yes(), No(), Yes());
        --left;
    }
    for (; left > 1; --left) step(No(), No(), Yes());
    step(No(), No(), No());
}

// Lanes j and j + 32 trade halves of 16 features: each has eight consecutive ones of its row, 16 q + 8 g of the tile.
__device__ __forceinline__ void eight_features(const f32x16 &acc, int q, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc[8 * q + i]), __float_as_uint(acc[8 * q + 4 + i]), false, false);
        v[i] = __uint_as_float(sw[0]);
        v[4 + i] = __uint_as_float(sw[1]);
    }
}

// A tile of the product.  Rows of whole pieces of eight features go through the LDS, 32 rows of a wavefront at a time, so that memory sees
// whole lines (as they lie in the accumulators an access is 32 bytes of each of 32 rows); the addend's pieces of 32 rows are requested
// together, those of the next 32 in front of the stores of these.
template <typename S, typename T>
__device__ __forceinline__ void store_tile(const f32x16 (&acc)[S::TF][S::TR], const MxArgs &A, int rt0, int ft0, int lane, int wave, char *lds)
{
    typedef RowPiece<T> P;
    const T *addend = (const T *)A.addend;
    T *y = (T *)A.y;
    const int j = lane & 31, g = lane >> 5;
    if (A.N % 8 != 0) {
#pragma unroll
        for (int u = 0; u < S::TR; ++u)
#pragma unroll
            for (int t = 0; t < S::FT; ++t)
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const int row = 32 * (rt0 + u) + j, f = 32 * (ft0 + t) + 16 * q + 8 * g;
                    float v[8];
                    eight_features(acc[t][u], q, v);
                    if (row < A.T) store_features<T>(addend, y, row, f, A.N, v);
                }
        return;
    }
    constexpr int W = 8 / P::V;                                   // 16-byte accesses of eight features
    constexpr int COLS = 32 * S::FT, STRIDE = COLS + 4;           // floats of a row in the LDS
    constexpr int LANES = COLS / 8, ROWS = 64 / LANES, N = 32 / ROWS;   // lanes per row, rows per access, accesses of 32 rows
    static_assert(4 * 32 * STRIDE * 4 <= S::LDS, "a part of the LDS for every wavefront");
    float *mine = (float *)lds + wave * (32 * STRIDE);
    const int r = lane / LANES, c = 8 * (lane % LANES), f = 32 * ft0 + c;
    constexpr int SETS = S::TR == 4 && W == 2 ? 1 : 2;            // (beside 256 accumulators two sets of fp32 pieces do not fit)
    u32x4 a[SETS][N][W];
    const auto request = [&](int u) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int row = 32 * (rt0 + u) + ROWS * i + r;
            const T *p = addend + (size_t)(row < A.T ? row : A.T - 1) * A.N + (f < A.N ? f : 0);
#pragma unroll
            for (int w = 0; w < W; ++w) a[u % SETS][i][w] = *(const u32x4 *)(p + w * P::V);
        }
    };
    const auto tile = [&](auto with) {
        constexpr bool ADD = decltype(with)::value;
        if constexpr (ADD && SETS == 2) request(0);
#pragma unroll
        for (int u = 0; u < S::TR; ++u) {
            if constexpr (ADD)
                if (u + SETS - 1 < S::TR) request(u + SETS - 1);
            wave_lds_sync();   // the last 32 rows have been read
#pragma unroll
            for (int t = 0; t < S::FT; ++t)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *(f32x4 *)(mine + j * STRIDE + 32 * t + 8 * q + 4 * g) =
                        f32x4{acc[t][u][4 * q], acc[t][u][4 * q + 1], acc[t][u][4 * q + 2], acc[t][u][4 * q + 3]};
            wave_lds_sync();
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int row = 32 * (rt0 + u) + ROWS * i + r;
                const float *m = mine + (ROWS * i + r) * STRIDE + c;
                const f32x4 lo = *(const f32x4 *)m, hi = *(const f32x4 *)(m + 4);
                float v[8];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[e] = lo[e];
                    v[4 + e] = hi[e];
                }
                if constexpr (ADD)
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] += P::get(a[u % SETS][i][e / P::V], e % P::V);
                if (row < A.T && f < A.N)
#pragma unroll
                    for (int w = 0; w < W; ++w) *(u32x4 *)(y + (size_t)row * A.N + f + w * P::V) = P::make(v + w * P::V);
            }
        }
    };
    lds_barrier();   // every wavefront is past its last fragment
    if (addend) tile(std::true_type());
    else tile(std::false_type());
}

template <typename S, typename T> __global__ __launch_bounds__(256, S::PER_SIMD) void mx_tile_kernel(MxArgs A)
{
    extern __shared__ __align__(1024) char lds[];
    const TilePlace place = tile_of(blockIdx.x, A.tiles_r, A.tiles_f, A.splits);
    const int r0 = place.r * S::RT, f0 = place.f * (S::FB / S::IMAGES);   // tiles of 32
    f32x16 acc[S::TF][S::TR];
#pragma unroll
    for (int t = 0; t < S::TF; ++t)
#pragma unroll
        for (int u = 0; u < S::TR; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[t][u][i] = 0.f;
    mx_steps<S>(acc, A, r0, f0, (int)((long long)A.Kt * place.split / A.splits), (int)((long long)A.Kt * (place.split + 1) / A.splits), lds);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wr = wave >> 1, wf = wave & 1, j = lane & 31, g = lane >> 5;
    const int rt0 = r0 + wr * S::TR, ft0 = f0 + wf * S::FT;
    if constexpr (S::DUAL) {
#pragma unroll
        for (int u = 0; u < S::TR; ++u) {
            if (rt0 + u >= A.x.tiles) continue;
#pragma unroll
            for (int t = 0; t < S::FT; ++t) {
                const int ft = ft0 + t;
                if (ft >= 8 * A.hKt) continue;
                float a[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float v = gated(acc[t][u][i], acc[S::FT + t][u][i]);
                    a[i] = 32 * ft + acc_feature(i, g) < A.N ? v : 0.f;   // (what is past the last row of the weights is anything)
                }
                store_hidden<S::BITS>(A, 32 * (rt0 + u) + j, ft, g, a);
            }
        }
    } else {
        if (A.splits > 1) A.y = (float *)A.y + (size_t)place.split * A.T * A.N;
        store_tile<S, T>(acc, A, rt0, ft0, lane, wave, lds);
    }
}

// y = addend + the shares' sums, in their order; four elements a thread.
template <typename T> __global__ __launch_bounds__(256) void mx_sum_kernel(const float *__restrict__ part, int splits, long long n, const T *addend, T *y)
{
    const long long at = ((long long)blockIdx.x * 256 + threadIdx.x) * 4;
    if (at >= n) return;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (at + 4 <= n && n % 4 == 0) {
        for (int s = 0; s < splits; ++s) {
            const f32x4 p = *(const f32x4 *)(part + s * n + at);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] += p[i];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] += addend ? Storage<T>::load(addend + at + i) : 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) Storage<T>::store(y + at + i, v[i]);
        return;
    }
    for (int i = 0; i < 4 && at + i < n; ++i) {
        float t = 0.f;
        for (int s = 0; s < splits; ++s) t += part[s * n + at + i];
        Storage<T>::store(y + at + i, t + (addend ? Storage<T>::load(addend + at + i) : 0.f));
    }
}

// shares: [splits][T][N] float of workspace (splits > 1)
template <typename S, typename T> static hipError_t run_tiles(MxArgs A, int f_tiles, int splits, float *shares, hipStream_t s)
{
    A.tiles_r = (A.x.tiles + S::RT - 1) / S::RT;
    A.tiles_f = (f_tiles + S::FB / S::IMAGES - 1) / (S::FB / S::IMAGES);
    A.splits = splits;
    const void *addend = A.addend;
    void *y = A.y;
    const auto launch = [&](auto kern) {
        const hipError_t e = grant_dynamic_lds((const void *)kern, S::LDS);
        if (e != hipSuccess) return e;
        kern<<<(unsigned)(A.tiles_r * A.tiles_f * splits), 256, S::LDS, s>>>(A);
        return hipGetLastError();
    };
    if (splits == 1) return launch(mx_tile_kernel<S, T>);
    if constexpr (!S::DUAL) {
        A.addend = nullptr;
        A.y = shares;
        const hipError_t e = launch(mx_tile_kernel<S, float>);
        if (e != hipSuccess) return e;
        const long long n = (long long)A.T * A.N;
        mx_sum_kernel<T><<<(unsigned)((n + 1023) / 1024), 256, 0, s>>>(shares, splits, n, (const T *)addend, (T *)y);
    }
    return hipGetLastError();
}

// ------------------------------------------------------------------------------ few rows
// Up to 32 TR rows: bound by the weights, which cross memory once.  A block has 32 features (of one or two images), its eight wavefronts the
// tiles of 256 columns in turn, whose fragments go straight from memory to registers (nobody else in the block needs them).  Their sums
// meet in the LDS, added in the wavefronts' order; behind it a row's 32 features are in 16 neighbouring lanes.
constexpr int kFewWaves = 8;   // (sixteen: equal or slower, d 4096, H 11008, 32 rows in 8 bits 25.8 us against 24.0)
template <int BITS, bool DUAL, int TR> struct MxFewStep {
    static constexpr int IMAGES = DUAL ? 2 : 1, RP = BITS == 4 ? 4 : 8;
    u32x4 f[IMAGES][4], r[TR][RP];
    int fs[IMAGES], rs[TR];
    __device__ __forceinline__ void load(const MxArgs &A, int ft, int kt, int lane)
    {
#pragma unroll
        for (int m = 0; m < IMAGES; ++m) {
            const MxMatrix &w = m ? A.w2 : A.w;
            const size_t t = (size_t)ft * A.Kt + kt;
            const u32x4 *p = (const u32x4 *)(w.v + t * 4096) + lane;
#pragma unroll
            for (int i = 0; i < 4; ++i) f[m][i] = __builtin_nontemporal_load(p + 64 * i);
            fs[m] = *((const int *)(w.s + t * 256) + lane);
        }
#pragma unroll
        for (int u = 0; u < TR; ++u) {
            const size_t t = (size_t)(u < A.x.tiles ? u : 0) * A.Kt + kt;
            const u32x4 *p = (const u32x4 *)(A.x.v + t * (1024 * BITS)) + lane;
            const bool there = 32 * u + (lane & 31) < A.T;   // (the others are not fetched)
#pragma unroll
            for (int i = 0; i < RP; ++i) r[u][i] = u32x4{0, 0, 0, 0};
            rs[u] = 0;
            if (there) {
#pragma unroll
                for (int i = 0; i < RP; ++i) r[u][i] = p[64 * i];
                rs[u] = *((const int *)(A.x.s + t * 256) + lane);
            }
        }
    }
    template <bool WHOLE> __device__ __forceinline__ void multiply(f32x16 (&acc)[IMAGES][TR]) const
    {
        for_range<0, 4>([&](auto k) {
            constexpr int K = decltype(k)::value;
#pragma unroll
            for (int u = 0; u < TR; ++u) {
                i32x8 b;
                if constexpr (BITS == 4) b = frag4(r[u][K]);
                else b = frag8(r[u][2 * K], r[u][2 * K + 1]);
                if constexpr (WHOLE) {
                    const i32x8 small = small_part(b);
#pragma unroll
                    for (int m = 0; m < IMAGES; ++m) acc[m][u] = mx_mfma<BITS, K>(frag4(f[m][K]), small, acc[m][u], fs[m], rs[u]);
                }
#pragma unroll
                for (int m = 0; m < IMAGES; ++m) acc[m][u] = mx_mfma<BITS, K>(frag4(f[m][K]), b, acc[m][u], fs[m], rs[u]);
            }
        });
    }
};

template <int BITS, bool DUAL, int TR, typename T> __global__ __launch_bounds__(64 * kFewWaves, TR == 1 ? 4 : 2) void mx_few_kernel(MxArgs A)
{
    typedef MxFewStep<BITS, DUAL, TR> Step;
    constexpr int IMAGES = Step::IMAGES, KW = kFewWaves;
    extern __shared__ __align__(16) float sums[];   // [KW][IMAGES][64 lanes][16], pieces of four swizzled over the 64 banks
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int ft = blockIdx.x;
    f32x16 acc[IMAGES][TR];
#pragma unroll
    for (int m = 0; m < IMAGES; ++m)
#pragma unroll
        for (int u = 0; u < TR; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[m][u][i] = 0.f;
    if (ft < A.w.tiles)
#pragma unroll 1
        for (int kt = wave; kt < A.Kt; kt += KW) {
            Step a;
            a.load(A, ft, kt, lane);
            a.template multiply<kMxWhole<BITS, T>>(acc);
        }
    // thread -> row, and positions p, p + 1 of its block: p = 16 g + 4 q + c is feature 8 q + 4 g + c
    const int row = tid >> 4 & 31, p = 2 * (tid & 15), g = p >> 4, from = row + 32 * g;
    const int at = from * 16 + 4 * ((p >> 2 & 3) ^ (from >> 2 & 3)) + (p & 3), f = 32 * ft + 8 * (p >> 2 & 3) + 4 * g + (p & 3);
#pragma unroll
    for (int u = 0; u < TR; ++u) {
        if (u > 0) __syncthreads();
#pragma unroll
        for (int m = 0; m < IMAGES; ++m)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *(f32x4 *)(sums + ((wave * IMAGES + m) * 64 + lane) * 16 + 4 * (q ^ (lane >> 2 & 3))) =
                    f32x4{acc[m][u][4 * q], acc[m][u][4 * q + 1], acc[m][u][4 * q + 2], acc[m][u][4 * q + 3]};
        __syncthreads();
        const int R = 32 * u + row;
        if (R >= A.T) continue;   // (a row's lanes together)
        float v[IMAGES][2];
#pragma unroll
        for (int m = 0; m < IMAGES; ++m) {
            v[m][0] = v[m][1] = 0.f;
#pragma unroll
            for (int w = 0; w < KW; ++w) {
                const float2 t = *(const float2 *)(sums + (w * IMAGES + m) * 1024 + at);
                v[m][0] += t.x;
                v[m][1] += t.y;
            }
        }
        if constexpr (DUAL) {
            float a[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float h = gated(v[0][i], v[IMAGES - 1][i]);
                a[i] = f + i < A.N ? h : 0.f;   // (what is past the last row of the weights is anything)
            }
            uint32_t most = __float_as_uint(a[0]) & 0x7fffffffu, other = __float_as_uint(a[1]) & 0x7fffffffu;
            most = other > most ? other : most;
            const auto larger = [&](int o) { most = (uint32_t)o > most ? (uint32_t)o : most; };
            larger(lane_move<0xB1>((int)most));
            larger(lane_move<0x4E>((int)most));
            larger(lane_move<0x141>((int)most));
            larger(lane_move<0x140>((int)most));
            const uint32_t byte = mx_scale_byte<BITS>(most);
            const float inv = mx_inverse(byte);
            const uint32_t q = mx_pack4<BITS>(a[0] * inv, a[1] * inv, 0.f, 0.f);
            uint8_t *o = A.h + mx_quad_offset<BITS>(R, ft, 2 * (p >> 2 & 3) + g, A.hKt) + (p & 3) * BITS / 8;
            if constexpr (BITS == 4) *o = (uint8_t)q;
            else *(uint16_t *)o = (uint16_t)q;
            if (p == 0) A.hs[mx_scale_offset(R, ft, A.hKt)] = (uint8_t)byte;
        } else {
            const size_t y = (size_t)R * A.N + f;
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (f + i < A.N) Storage<T>::store((T *)A.y + y + i, v[0][i] + (A.addend ? Storage<T>::load((const T *)A.addend + y + i) : 0.f));
        }
    }
}

// Up to 16 TR rows (groups of 16) and few features: 16 of them a block, so that twice as many CUs draw on the memory, on the instruction of 16 x 16
// results and 128 columns (lane i + 16 g: row i and, in 4 bits, block g of four; in 8 bits 16 values each of block g / 2 and of block 2 + g / 2; the scale of
// block b from lane i + 16 b; result r of lane i + 16 g: feature 4 g + r of row i).
template <int BITS, int TR, typename T> __global__ __launch_bounds__(1024, 4) void mx_half_kernel(MxArgs A)
{
    constexpr int KW = 16, RP = BITS == 4 ? 1 : 2;
    __shared__ __align__(16) float sums[KW][TR * 256];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int ft = blockIdx.x >> 1, i = lane & 15, g = lane >> 4;
    const uint32_t piece = 1024 * (g >> 1) + 512 * (g & 1) + 16 * i, scale = 128 * (g & 1) + 4 * i;   // of row i of a tile
    const uint32_t half = 16 * (blockIdx.x & 1);
    // thread -> row and feature
    const int row = tid >> 4, f = tid & 15, F = 32 * ft + half + f;
    const bool out = tid < 256 * TR && row < A.T && F < A.N;
    const size_t y = (size_t)row * A.N + F;
    const float addend = out && A.addend ? Storage<T>::load((const T *)A.addend + y) : 0.f;
    f32x4 acc[TR];
#pragma unroll
    for (int u = 0; u < TR; ++u) acc[u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (int kt = wave; kt < A.Kt; kt += KW) {
        const size_t t = (size_t)ft * A.Kt + kt;
        u32x4 w[2], r[TR][2][RP];
        int rs[TR];
#pragma unroll
        for (int j = 0; j < 2; ++j) w[j] = __builtin_nontemporal_load((const u32x4 *)(A.w.v + t * 4096 + 2048 * j + piece + 16 * half));
        const int ws = *(const int *)(A.w.s + t * 256 + scale + 4 * half) >> 8 * (g >> 1);
#pragma unroll
        for (int u = 0; u < TR; ++u) {
            rs[u] = 0;
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int q = 0; q < RP; ++q) r[u][j][q] = u32x4{0, 0, 0, 0};
            if (16 * u + i < A.T) {   // (the others are not fetched)
                const size_t xt = (size_t)(u >> 1) * A.Kt + kt;
                const uint8_t *x = A.x.v + xt * (1024 * BITS) + piece + 256 * (u & 1);
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int q = 0; q < RP; ++q) r[u][j][q] = *(const u32x4 *)(x + 2048 * (RP * j + q));
                rs[u] = *(const int *)(A.x.s + xt * 256 + scale + 64 * (u & 1)) >> 8 * (g >> 1);
            }
        }
        for_range<0, 2>([&](auto jj) {
            constexpr int J = decltype(jj)::value;
#pragma unroll
            for (int u = 0; u < TR; ++u) {
                i32x8 b;
                if constexpr (BITS == 4) b = frag4(r[u][J][0]);
                else b = frag8(r[u][J][0], r[u][J][RP - 1]);
                if constexpr (kMxWhole<BITS, T>)
                    acc[u] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(frag4(w[J]), small_part(b), acc[u], 4, 0, 2 * J, ws, 2 * J, rs[u]);
                acc[u] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(frag4(w[J]), b, acc[u], 4, BITS == 4 ? 4 : 0, 2 * J, ws, 2 * J, rs[u]);
            }
        });
    }
#pragma unroll
    for (int u = 0; u < TR; ++u) *(f32x4 *)(sums[wave] + 256 * u + 4 * lane) = acc[u];
    __syncthreads();
    if (!out) return;
    const int at = 256 * (row >> 4) + 64 * (f >> 2) + 4 * (row & 15) + (f & 3);
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < KW; ++k) v += sums[k][at];
    Storage<T>::store((T *)A.y + y, v + addend);
}

template <int BITS, bool DUAL, int TR, typename T> static hipError_t run_few(const MxArgs &A, int f_tiles, hipStream_t s)
{
    const auto kern = mx_few_kernel<BITS, DUAL, TR, T>;
    constexpr size_t lds = (size_t)kFewWaves * (DUAL ? 2 : 1) * 4096;
    const hipError_t e = grant_dynamic_lds((const void *)kern, lds);
    if (e != hipSuccess) return e;
    kern<<<(unsigned)f_tiles, 64 * kFewWaves, lds, s>>>(A);
    return hipGetLastError();
}

// Which kernel a product takes: few rows, tiles of 128 x 128 (several blocks a CU), or of 256 x 256 (one).
// us, few rows / tiles: 8 bits 64 rows 4096 11008 11.6 / 13.0, 11008 4096 12.7 / 14.8, 1024 2816 4.6 / 6.5; 32 rows 9.1 / 12.8, 10.0 / 12.8, 3.8 / 6.1.  4 bits
// 64 rows 8.6 / 9.8, 9.0 / 14.3, 4.3 / 5.7; fp32 storage, 8 bits, 64 rows 15.9 / 22.7, 18.4 / 19.6, 5.3 / 9.6; 64 rows 11008 11008, a second round of blocks, 22.5 / 22.2 in
// 4 bits, 29.4 / 26.1 in 8, 34.0 / 38.8 with fp32 storage; in the network see `second_round`.
// With few rows, 16 features a block while every block has a CU, 32 else; us, 16 / 32 of them: 16 rows in 8 bits 11008 4096 7.5 / 8.9, 4096 4096 4.2 / 5.0,
// 2816 1024 2.8 / 3.5, 64 rows 12.5 / 15.0, 6.1 / 7.5, 4.7 / 5.2; beyond, 4096 5120 5.5 / 5.1, 11008 8192 13.4 / 11.2.
constexpr int kFewRows = 64;
constexpr int kMostSplits = 8, kSplitBlocks = 512;   // shares of the contraction at most, and blocks of all shares together
struct MxChoice {
    bool large;
    int splits;
    long long blocks;
};
// us of a step of 256 columns, fitted to products of 66 to 16384 rows at K 1024 to 11008 (T, K, N: 128 tiles / 256 tiles, us):
//   4 bits   2048 4096 11008: 55.2 / 57.6   4096 4096 11008: 104.5 / 93.5   4096 11008 4096: 93.0 / 77.8   2048 11008 4096: 49.0 / 59.2   1024 2816 1024: 7.8 / 18.6
//   8 bits   2048 4096 11008: 76.3 / 87.2   4096 4096 11008: 144 / 137   4096 11008 4096: 131 / 117   2048 11008 4096: 69.3 / 97.5   1024 2816 1024: 10.2 / 28.5
// and in shares, 128 tiles, 1 / 2 / 4 / 8 of them: 4 bits 66 11008 4096 18.1 / 13.7 / 12.0 / 13.1, 200 11008 4096 19.1 / 16.1 / 17.4 / 20.3, 512 11008 4096 20.3 / 22.3 /
// 27.8; 8 bits 66 11008 4096 27.0 / 18.0 / 13.9 / 14.1, 128 11008 4096 27.7 / 19.4 / 16.6 / 17.5, 512 11008 4096 30.4 / 27.9 / 31.9.
// With fp32 storage and rows of 8 bits, whose parts are multiplied one after the other, 128 tiles / 256 tiles: 4096 11008 4096 257 / 218, 4096 4096 11008 312 / 285,
// 2048 11008 4096 133 / 176; shares 66 11008 4096 65 / 39 / 25 / 20, 200 4096 4096 28.3 / 21.8 / 22.4 / 24.9, 512 11008 4096 71 / 50.
struct MxCosts {
    double one, each, start;   // 128 tiles: a block alone on its CU, every further one, beginning and end of a block
    int per_cu;
    double large, large_start;
};
static constexpr MxCosts kMxCosts4 = {0.48, 0.55, 2.7, 2, 1.55, 9.0}, kMxCosts8 = {0.73, 0.72, 3.0, 2, 2.45, 9.0},
                         kMxCosts8Whole = {1.46, 1.44, 3.0, 2, 4.9, 9.0};   // (twice the instructions)
static MxChoice choose(long long T, int f_tiles, int Kt, int N, int bits, bool dual, bool whole)
{
    const MxCosts &c = bits == 4 ? kMxCosts4 : whole ? kMxCosts8Whole : kMxCosts8;
    const long long cus = num_compute_units(), per = dual ? 2 : 4;
    const auto blocks = [&](int rows, int tiles) { return ((T + rows - 1) / rows) * ((f_tiles + tiles - 1) / tiles); };
    const long long small = blocks(128, per), large = blocks(256, 2 * per);
    MxChoice best = {true, 1, large};
    const long long left = large % cus;   // a partial round's steps are shorter: 1.3 of 2 with half of the chip
    double least = Kt * c.large * (large / cus + (left ? 0.6 + 0.4 * left / cus : 0)) + c.large_start * ((large + cus - 1) / cus);
    for (int s = 1; s <= kMostSplits && s <= Kt; s *= 2) {
        const long long n = small * s, round = cus * c.per_cu, rest = n % round;
        if (s > 1 && (dual || n > kSplitBlocks)) break;
        const auto depth = [&](long long b) { return b == 0 ? 0 : c.one + c.each * ((double)b / cus > 1 ? (double)b / cus - 1 : 0); };
        double t = (double)Kt / s * (n / round * depth(round) + depth(rest)) + c.start * ((n + round - 1) / round);
        if (s > 1) t += 5 + (double)s * T * N * 8 / 4e6;   // the shares' addition: a launch, and their sums through the caches
        if (t < least) {
            least = t;
            best = {false, s, n};
        }
    }
    return best;
}
// Bytes of the shares' sums, for this and every smaller batch: as many of them as the rule above can choose.
static size_t shares_bytes(long long T, int N, int Kt)
{
    if (T <= kFewRows || Kt < 2) return 0;
    const long long tiles_f = (N + 127) / 128, rows = kSplitBlocks / tiles_f * 128;
    return (size_t)(kMostSplits * T < rows ? kMostSplits * T : rows) * N * 4;
}

template <int BITS, bool DUAL, typename T> static hipError_t run_product(const MxArgs &A, float *shares, hipStream_t s)
{
    constexpr bool WHOLE = kMxWhole<BITS, T>;
    const int f_tiles = DUAL ? 8 * A.hKt : A.w.tiles;
    // A pair of more than 32 rows has one block of few rows a CU: a second round of them loses to the tiles.  The network, us, few rows / tiles for the pair: 48
    // rows, H 11008, 4 bits d 512 15.8 / 13.2, 1024 16.9 / 13.9, 2048 19.8 / 17.4, 4096 26.7 / 21.6, 8 bits 19.1 / 16.0, 21.4 / 17.9, 24.7 / 22.8, 33.5 / 28.5; H 8448,
    // d 4096 23.8 / 19.8, 29.2 / 25.8; H 16384 32.3 / 28.5, 40.9 / 35.5; 33 rows, H 11008, d 4096 25.5 / 21.3, 32.1 / 27.6.  In one round few rows are the faster ones:
    // H 8192 4 bits d 1024 12.7 / 13.3, 4096 18.0 / 19.7, 8 bits 14.8 / 16.1, 21.8 / 25.6; and up to 32 rows, of which a CU has two blocks, in two rounds near
    // the tiles: 32 rows, H 11008, 4 bits d 1024 12.6 / 12.1, 4096 21.4 / 19.9, 8 bits 14.4 / 14.8, 24.3 / 25.3, 17 rows 11.7 / 11.8, 19.7 / 19.9, 13.7 / 14.3, 23.0 / 24.4.
    const bool second_round = DUAL && A.T > 32 && f_tiles > num_compute_units();
    if (A.T <= kFewRows && !second_round) {
        if constexpr (!DUAL)
            if (2 * f_tiles <= num_compute_units()) {
                const auto kern = A.T <= 16 ? mx_half_kernel<BITS, 1, T> : A.T <= 32 ? mx_half_kernel<BITS, 2, T> : mx_half_kernel<BITS, 4, T>;
                kern<<<(unsigned)(2 * f_tiles), 1024, 0, s>>>(A);
                return hipGetLastError();
            }
        return A.T > 32 ? run_few<BITS, DUAL, 2, T>(A, f_tiles, s) : run_few<BITS, DUAL, 1, T>(A, f_tiles, s);
    }
    const MxChoice c = choose(A.T, f_tiles, A.Kt, A.N, BITS, DUAL, WHOLE);
    if (c.large) return run_tiles<MxTile<BITS, DUAL, 4, 4, BITS == 4 ? 4 : 2, BITS == 4 ? 2 : 3, WHOLE>, T>(A, f_tiles, 1, nullptr, s);
    // Rings of 128 x 128 tiles.  8 bits: three images, two blocks a CU (us with two images and three blocks / three and two: 1024 11008 4096 55.4 / 37.1, the pair
    // 1024 4096 11008 83 / 80, 16384 1024 2816 48.3 / 48.4).  4 bits: four images of half the step, two blocks a CU (with two whole ones / so: the network, 1024
    // rows, 4096 11008 91.3 / 85.4, 256 rows, 1024 2816 16.0 / 14.8, 16384 1024 2816 110.7 / 110.6), where no CU has a second block three whole ones (700
    // 11008 4096 29.9 / 25.7 / 21.6; with a second block 512 4096 11008 19.3 / 19.7 / 20.9).
    // Short contractions in 8 bits, where results count, take three blocks a CU; without an addend / with one, two blocks against three: 16384 256 768 11.3 : 10.1 /
    // 14.2 : 12.1, 16384 512 1408 20.1 : 19.3 / 24.2 : 23.2, 16384 1024 2816 46.5 : 46.9 / 52.6 : 51.5, 4096 1024 2816 15.6 : 15.7 / 18.5 : 17.7; beyond, 16384 1280 3456
    // 66.2 : 66.2 / 72.3 : 73.9, 4096 1536 2816 19.4 : 20.4 / 22.1 : 22.0, 4096 2560 2816 27.7 : 29.4 / 29.1 : 31.1; of at most two blocks a CU 4096 512 1408 with an
    // addend 9.0 : 9.5.
    const int cus = num_compute_units();
    if constexpr (BITS == 8) {
        if (A.Kt <= 4 && c.blocks > 2 * cus) return run_tiles<MxTile<8, DUAL, 2, 2, 2, 2, WHOLE>, T>(A, f_tiles, c.splits, shares, s);
        return run_tiles<MxTile<8, DUAL, 2, 2, 2, 3, WHOLE>, T>(A, f_tiles, c.splits, shares, s);
    } else if (c.blocks <= cus) return run_tiles<MxTile<4, DUAL, 2, 2, 4, 3, false>, T>(A, f_tiles, c.splits, shares, s);
    else return run_tiles<MxTile<4, DUAL, 2, 2, 2, 4, false>, T>(A, f_tiles, c.splits, shares, s);
}

size_t mx_product_workspace(const slicemoe_mx_product_config &c) { return align_up(shares_bytes(c.T, c.N, mx_tiles_k(c.K)), 256); }

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
    float *f = (float *)ws;
    if (c.bits == 4) return c.dtype == SLICEMOE_BF16 ? run_product<4, false, bf16_t>(A, f, s) : run_product<4, false, float>(A, f, s);
    return c.dtype == SLICEMOE_BF16 ? run_product<8, false, bf16_t>(A, f, s) : run_product<8, false, float>(A, f, s);
}

// The hidden rows, and behind them the second product's workspace.
static size_t hidden_bytes(const slicemoe_gated_config &c, int bits) { return align_up(mx_total_bytes(c.T, c.H, bits), 256) + 256; }   // (never 0)
static slicemoe_mx_product_config second_product(const slicemoe_gated_config &c, int bits) { return {c.T, c.H, c.d, bits, SLICEMOE_BF16}; }
size_t gated_mx_workspace(const slicemoe_gated_config &c, int bits) { return hidden_bytes(c, bits) + mx_product_workspace(second_product(c, bits)); }

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
    const hipError_t e = bits == 4 ? run_product<4, true, bf16_t>(A, nullptr, s) : run_product<8, true, bf16_t>(A, nullptr, s);
    if (e != hipSuccess) return e;
    return launch_mx_product(second_product(c, bits), A.h, (const uint8_t *)w.Wd, addend, y, ws + hidden_bytes(c, bits), s);
}

}  // namespace slicemoe
