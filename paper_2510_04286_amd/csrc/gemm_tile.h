// Matrix-product tiles for the gated feed-forward network (gated_ffn.hip): C[rows, features] = R F^T over a list of segments, with
// fp32 accumulation, operands in memory in either order.
//
// One block of four wavefronts owns a tile.  As in the layer's kernels the product is computed transposed: the features' operand F is
// the matrix instruction's first, the rows' operand R its second, so a lane's accumulators are features of one row.
//
// A step of the contraction is 128 bytes of a row: 64 bf16 values or 128 e4m3 ones.  Its images in the LDS come straight from memory
// (global_load_lds, 16 bytes per lane): 1 KB per instruction, linear in the lane, so the arrangement that keeps the reads free of
// bank conflicts is made by which 16 bytes a lane asks for.
//   K-contiguous operands ([row][k] in memory): 128 bytes per row, piece c of row i at place c ^ (i / 2 % 8); a fragment is one
//     ds_read_b128 (lane = row, eight consecutive k).
//   K-major operands ([k][row] in memory): rows of k, blocks of 64 bytes (32 rows) XORed with k & 3; a fragment is two
//     ds_read_b64_tr_b16, which hand every lane the four k of its row.
//
// Each operand has a ring of images, the rows' one longer than the features' where the LDS has room for it (3 + 2 images of 32 KB).
// Fragments are read AHEAD quarters before their use, between the matrix instructions; that many quarters before a step's end stands
// its one barrier: behind it the next step's images have landed for every wavefront and the present ones, whose last fragments are
// in registers, are free for the requests two and three steps ahead.
//
// What it took (up projections of T 8192, d 4096, H 11008, us): plain double buffering with the loads and reads in front of the matrix
// instructions 1363; requests one by one between them 1264; no branch per request, LDS targets set once in four 1105; LDS rows on 64 banks
// (32 before: a tenth of the cycles were conflicts), the rows' ring a step longer 1063.  Loads alone take 840 of them, matrix
// instructions and LDS reads without loads 730.  Fragments a quarter ahead instead of a step: equal, or up to 7% slower.
// Groups of 4 to 16 row tiles instead of 8: no gain.  64-byte pieces of rows: a CU draws 57 instead of 95 bytes per ns from L2.
//
// Edges: rows and columns past an operand's end are read at its last one (their products are never stored); a step that reaches past
// the end of K takes those 16-byte pieces from a page of zeros, in both operands.
#pragma once
#include <type_traits>

#include "lds_rows.h"
#include "wavefront.h"

namespace slicemoe {

constexpr int kMaxSegments = 12;
// One product of a launch.  Leading dimensions and K in bytes; K is what is read of a K-contiguous row, a whole number of 16-byte
// pieces, and the number of k times 2 for K-major operands.
struct GemmProblem {
    const char *r[kMaxSegments], *f[kMaxSegments], *f2[kMaxSegments];   // f2: the second image of the features (gate and up)
    long long ldr, ldf;
    int nr, nf;          // rows, features (of one image)
    int K;               // bytes
    int segments;
    int tiles_r, tiles_f;
    int splits;          // shares of the contraction, each a range of steps
};

__device__ const uint4 g_zero_piece[1] = {};

enum { kKContiguous = 0, kKMajor = 1 };

typedef int i32x8 __attribute__((ext_vector_type(8)));

template <int I> using Int = std::integral_constant<int, I>;
// f(Int<A>()), .. f(Int<B - 1>())
template <int A, int B, typename F> __device__ __forceinline__ void for_range(const F &f)
{
    if constexpr (A < B) {
        f(Int<A>());
        for_range<A + 1, B>(f);
    }
}


// 1 KB from memory to the LDS: lane l's 16 bytes go to M0 + AT + 16 l and come from base + offset + AT (the instruction's own offset
// moves both).  Written out, because the compiler would wait for all of them in front of every LDS read; the waits are in the
// pipeline below.  Nothing else in these kernels writes M0.
__device__ __forceinline__ void set_lds_target(uint32_t at) { asm volatile("s_mov_b32 m0, %0\n\ts_nop 0" ::"s"(at) : "memory"); }
template <int AT> __device__ __forceinline__ void load_lds_1k(const char *base, uint32_t offset)
{
    asm volatile("global_load_lds_dwordx4 %0, %1 offset:%2" ::"v"(offset), "s"(base), "n"(AT) : "memory");
}
template <int AT> __device__ __forceinline__ void load_lds_1k(const char *address)
{
    asm volatile("global_load_lds_dwordx4 %0, off offset:%1" ::"v"(address), "n"(AT) : "memory");
}
template <int N> __device__ __forceinline__ void wait_loads_and_barrier()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// The image of one operand: N rows of the tile (a multiple of 32), filled by WAVES wavefronts.  Wavefront w has the kilobytes
// PER_WAVE w + i, four of them (or all) from one LDS target.
template <int LAYOUT, int N, int WAVES> struct TileImage {
    static constexpr int BYTES = N * 128, PER_WAVE = N / 8 / WAVES;
    static constexpr int K_PER_PIECE = 512 / N;   // rows of k per kilobyte (K-major)
    static constexpr int BIAS = 3 * 1024;            // what the instruction's own offset adds at most is taken off the base, added to the offsets
    static __device__ __forceinline__ int block_swizzle(int k) { return N >= 128 ? k & 3 : N == 64 ? k >> 1 & 1 : 0; }
    // K-contiguous: which 16 bytes of its row a lane fetches (see FragmentReader: 16 rows at a time, two to the 64 banks)
    static __device__ __forceinline__ int piece_of(int kb, int lane) { return (lane & 7) ^ ((kb & 1) << 2 | lane >> 4); }

    // This lane's offsets from the tile's corner (the operand's row `first`, step 0 of K).
    static __device__ __forceinline__ void offsets(uint32_t (&o)[PER_WAVE], int wave, int lane, int first, int rows, uint32_t ld)
    {
#pragma unroll
        for (int i = 0; i < PER_WAVE; ++i) {
            const int kb = wave * PER_WAVE + i;
            if constexpr (LAYOUT == kKContiguous) {
                const int row = 8 * kb + (lane >> 3), last = rows - 1 - first;
                o[i] = (uint32_t)(row < last ? row : last) * ld + 16u * piece_of(kb, lane);
            } else {
                const int k = kb * K_PER_PIECE + lane / (N / 8), last = (rows - 1 - first) >> 3;
                const int c = (lane % (N / 8)) ^ block_swizzle(k) << 2;
                o[i] = (uint32_t)k * ld + 16u * (c < last ? c : last);
            }
            o[i] += BIAS - 1024 * (i & 3);
        }
    }
    static __device__ __forceinline__ const char *corner(const char *p, int first, long long ld)
    {
        return (LAYOUT == kKContiguous ? p + first * ld : p + 2ll * first) - BIAS;
    }
    static __device__ __forceinline__ long long step_bytes(long long ld) { return LAYOUT == kKContiguous ? 128 : 64 * ld; }

    // Requests kilobyte i of this wavefront's share of the image of one step.  TAIL: the last step of K, of which `left` bytes are there.
    template <bool TAIL, int I> static __device__ __forceinline__ void request(uint32_t lds, const char *base, const uint32_t (&o)[PER_WAVE], int wave, int lane, int left)
    {
        if constexpr (I % 4 == 0) set_lds_target(lds + 1024 * (wave * PER_WAVE + I));
        if constexpr (!TAIL) load_lds_1k<1024 * (I & 3)>(base, o[I]);
        else {
            const int kb = wave * PER_WAVE + I;
            const bool there = LAYOUT == kKContiguous ? 16 * piece_of(kb, lane) < left : 2 * (kb * K_PER_PIECE + lane / (N / 8)) < left;
            load_lds_1k<1024 * (I & 3)>(there ? base + o[I] : (const char *)g_zero_piece - 1024 * (I & 3));
        }
    }
};

// Reads fragments of 32 rows (tile `t` of a wavefront whose first row of 32 is block `wb` of the image).
template <int LAYOUT, int N, bool E4M3> struct FragmentReader {
    typedef typename std::conditional<E4M3, i32x8, bf16x8>::type frag;
    uint32_t base[4];
    __device__ __forceinline__ void init(int wb, int lane)
    {
        const int i = lane & 31, g = lane >> 5;
        if constexpr (LAYOUT == kKContiguous) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {   // E4M3: 32 bytes of a row, pieces 4 ks + 2 g and the next; else pieces 2 ks + g
                const int c = E4M3 ? 4 * (q >> 1) + 2 * g + (q & 1) : 2 * q + g;
                base[q] = (wb * 32 + i) * 128 + ((c ^ (i >> 1 & 7)) << 4);
            }
        } else {
            const int q = lane >> 2 & 3;   // which of four k this lane fetches
#pragma unroll
            for (int t = 0; t < 4; ++t)
                base[t] = (8 * g + q) * (2 * N) + (((wb + t) ^ TileImage<LAYOUT, N, 1>::block_swizzle(q)) & (N / 32 - 1)) * 64 + 32 * (lane >> 4 & 1) + 8 * (lane & 3);
        }
    }
    __device__ __forceinline__ frag read(const char *image, int t, int ks) const
    {
        if constexpr (LAYOUT == kKContiguous) {
            if constexpr (E4M3) {
                union {
                    uint4 h[2];
                    i32x8 v;
                } r;
                r.h[0] = *(const uint4 *)(image + base[2 * ks] + t * 4096);
                r.h[1] = *(const uint4 *)(image + base[2 * ks + 1] + t * 4096);
                return r.v;
            } else
                return *(const bf16x8 *)(image + base[ks] + t * 4096);
        } else {
            const char *p = image + base[t] + ks * 16 * (2 * N);
            return read_transposed(as_lds(p), as_lds(p + 4 * (2 * N)));
        }
    }
};

// TR x TF fragments of 32 rows and features per wavefront, WR x WF = 4 wavefronts.  DUAL: the first half of a wavefront's feature
// tiles comes from f, the second from f2 (the same features of two matrices).  SR, SF: images in the rings of the two operands.
template <int TR_, int TF_, int WR_, int WF_, int RL_, int FL_, bool DUAL_, bool E4M3_, int SR_, int SF_> struct TileShape {
    static constexpr int TR = TR_, TF = TF_, WR = WR_, WF = WF_, RL = RL_, FL = FL_, SR = SR_, SF = SF_;
    static constexpr bool DUAL = DUAL_, E4M3 = E4M3_;
    static_assert(WR * WF == 4 && TR <= 4 && TF <= 4, "four wavefronts, at most 128 x 128 each");
    static_assert(SF >= 2 && (SR == SF || SR == SF + 1), "see the waits");
    static constexpr int IMAGES = DUAL ? 2 : 1, FT = TF / IMAGES;   // feature tiles per image and wavefront
    static constexpr int BR = 32 * TR * WR, BF = 32 * FT * WF;      // rows, features (of one image) per block
    typedef TileImage<RL, BR, 4> RI;
    typedef TileImage<FL, BF, 4> FI;
    static constexpr int R_BYTES = RI::BYTES, F_BYTES = IMAGES * FI::BYTES;
    static constexpr int R_LOADS = RI::PER_WAVE, F_LOADS = IMAGES * FI::PER_WAVE;   // instructions per wavefront and step
    static constexpr int LDS = SR * R_BYTES + SF * F_BYTES;
    static constexpr int KS = E4M3 ? 2 : 4;                              // matrix-instruction steps (quarters, halves) per step
    static constexpr int AHEAD = KS - 1;                                 // quarters between a fragment's read and its use
};

// acc[feature tile][row tile] += the steps [s0, s1) of the problem's contraction (counted through its segments).
template <typename S>
__device__ __forceinline__ void mma_steps(f32x16 (&acc)[S::TF][S::TR], const GemmProblem &p, int row0, int f0, int s0, int s1, char *lds)
{
    typedef typename S::RI RI;
    typedef typename S::FI FI;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wr = wave / S::WF, wf = wave % S::WF;
    const int n = s1 - s0;
    if (n <= 0) return;
    const uint32_t lds0 = (uint32_t)(uintptr_t)as_lds(lds);
    uint32_t ro[RI::PER_WAVE], fo[FI::PER_WAVE];
    RI::offsets(ro, wave, lane, row0, p.nr, (uint32_t)p.ldr);
    FI::offsets(fo, wave, lane, f0, p.nf, (uint32_t)p.ldf);
    FragmentReader<S::RL, S::BR, S::E4M3> rr;
    FragmentReader<S::FL, S::BF, S::E4M3> fr;
    rr.init(wr * S::TR, lane);
    fr.init(wf * S::FT, lane);

    // Where the next request of each operand comes from (segment, step of it, pointer) and goes to (image of its ring).
    const int per_segment = (p.K + 127) >> 7;
    uint64_t rstep = RI::step_bytes(p.ldr), fstep = FI::step_bytes(p.ldf);
    asm volatile("" : "+s"(rstep), "+s"(fstep));   // (kept in registers: fetched again inside the loop they would make it wait for every LDS read)
    int rseg = s0 / per_segment, rat = s0 - rseg * per_segment, rslot = 0, fseg = rseg, fat = rat, fslot = 0;
    const char *rp, *fp, *fp2 = nullptr;
    const auto enter_r = [&]() { rp = RI::corner(p.r[rseg], row0, p.ldr) + rat * rstep; };
    const auto enter_f = [&]() {
        fp = FI::corner(p.f[fseg], f0, p.ldf) + fat * fstep;
        if constexpr (S::DUAL) fp2 = FI::corner(p.f2[fseg], f0, p.ldf) + fat * fstep;
    };
    enter_r();
    enter_f();
    // kilobytes [from, to) of a step's requests: the features' first, then the rows'; TAIL: either may be in the last step of its segment
    const auto pieces = [&](auto tail, auto from, auto to, int rleft, int fleft) {
        constexpr bool TAIL = decltype(tail)::value;
        for_range<decltype(from)::value, decltype(to)::value>([&](auto index) {
            constexpr int I = decltype(index)::value, G = I - FI::PER_WAVE, R = I - S::F_LOADS;
            const uint32_t f_to = lds0 + S::SR * S::R_BYTES + fslot * S::F_BYTES;
            if constexpr (R >= 0) RI::template request<TAIL, R>(lds0 + rslot * S::R_BYTES, rp, ro, wave, lane, rleft);
            else if constexpr (G >= 0) FI::template request<TAIL, G>(f_to + FI::BYTES, fp2, fo, wave, lane, fleft);
            else FI::template request<TAIL, I>(f_to, fp, fo, wave, lane, fleft);
        });
    };
    const auto next_r = [&]() {   // (within a segment)
        rslot = rslot + 1 == S::SR ? 0 : rslot + 1;
        ++rat;
        rp += rstep;
    };
    const auto next_f = [&]() {
        fslot = fslot + 1 == S::SF ? 0 : fslot + 1;
        ++fat;
        fp += fstep;
        if constexpr (S::DUAL) fp2 += fstep;
    };
    const auto advance_r = [&]() {
        next_r();
        if (rat == per_segment) {
            rat = 0;
            if (++rseg < p.segments) enter_r();
        }
    };
    const auto advance_f = [&]() {
        next_f();
        if (fat == per_segment) {
            fat = 0;
            if (++fseg < p.segments) enter_f();
        }
    };
    typedef typename FragmentReader<S::RL, S::BR, S::E4M3>::frag frag;
    constexpr int SETS = S::AHEAD + 1;
    static_assert(S::KS % SETS == 0, "quarter q has the set q % SETS in every step");
    frag rf[SETS][S::TR], ff[SETS][S::TF];
    // fragment i of quarter ks of the step in the rings' present images, in the order of their first use: the first features', all
    // rows', the other features'
    int rcur = 0, fcur = 0;
    const auto read = [&](int set, int ks, int i) {
        const char *rimage = lds + rcur * S::R_BYTES, *fimage = lds + S::SR * S::R_BYTES + fcur * S::F_BYTES;
        if (i >= 1 && i <= S::TR) rf[set][i - 1] = rr.read(rimage, i - 1, ks);
        else {
            const int t = i == 0 ? 0 : i - S::TR;
            ff[set][t] = fr.read(fimage + (t / S::FT) * FI::BYTES, t % S::FT, ks);
        }
    };
    const auto multiply = [&](int set, int m) {
        const int t = m / S::TR, u = m % S::TR;
        if constexpr (S::E4M3)   // (scales of 2^0)
            acc[t][u] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(ff[set][t], rf[set][u], acc[t][u], 0, 0, 0, 0x7f7f7f7f, 0, 0x7f7f7f7f);
        else
            acc[t][u] = mfma_bf16(ff[set][t], rf[set][u], acc[t][u]);
    };
    // One quarter: its matrix instructions, with the reads of quarter `ahead` and the requests [FROM, TO) of a later step between them.
    // A wavefront issues in order, and one that asks for several kilobytes in a row stands still until the memory pipeline has taken
    // them: each request has its own place.
    constexpr int NM = S::TR * S::TF, NF = S::TR + S::TF;
    const auto quarter = [&](int now, auto reads, int ahead, auto tail, auto from, auto to, int rleft, int fleft) {
        constexpr bool READS = decltype(reads)::value;
        constexpr int FROM = decltype(from)::value, TO = decltype(to)::value;
        for_range<0, NM>([&](auto mm) {
            constexpr int M = decltype(mm)::value;
            multiply(now % SETS, M);
            if constexpr (READS)
#pragma unroll
                for (int i = M * NF / NM; i < (M + 1) * NF / NM; ++i) read(ahead % SETS, ahead, i);
            pieces(tail, Int<FROM + M *(TO - FROM) / NM>(), Int<FROM + (M + 1) * (TO - FROM) / NM>(), rleft, fleft);
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    // Behind a barrier: the last AHEAD quarters of one step and the others of the next one, with the requests: the features' (needed
    // first) in the first quarter, the rows' in the later ones.  LOADS: how many of them (0, the features', all).
    const auto step = [&](auto tail, auto loads) {
        rcur = rcur + 1 == S::SR ? 0 : rcur + 1;
        fcur = fcur + 1 == S::SF ? 0 : fcur + 1;
        const int rleft = p.K - 128 * rat, fleft = p.K - 128 * fat;
        for_range<0, S::KS>([&](auto qq) {
            constexpr int Q = decltype(qq)::value, F = S::F_LOADS, R = decltype(loads)::value - F;
            constexpr auto upto = [](int q) { return R + F == 0 || q == 0 ? 0 : F + R * (q - 1) / (S::KS - 1); };
            quarter((Q + S::KS - S::AHEAD) % S::KS, std::true_type(), Q, tail, Int<upto(Q)>(), Int<upto(Q + 1)>(), rleft, fleft);
        });
    };
    constexpr Int<0> none = {};
    constexpr Int<S::F_LOADS> features = {};
    constexpr Int<S::F_LOADS + S::R_LOADS> all = {};
    // What may be on its way at a step's barrier: all that was requested after the next step's images.
    constexpr int IN_FLIGHT = (S::SF - 2) * (S::R_LOADS + S::F_LOADS) + (S::SR - S::SF) * S::R_LOADS;

    for (int i = 0; i < S::SF && i < n; ++i) {
        pieces(std::true_type(), none, all, p.K - 128 * rat, p.K - 128 * fat);
        advance_r();
        advance_f();
    }
    if (S::SR > S::SF && n >= S::SR) {
        pieces(std::true_type(), features, all, p.K - 128 * rat, 0);
        advance_r();
    }
    if (n >= S::SR) wait_loads_and_barrier<IN_FLIGHT + S::R_LOADS + S::F_LOADS>();
    else wait_loads_and_barrier<0>();
#pragma unroll
    for (int q = 0; q < S::AHEAD; ++q)
#pragma unroll
        for (int i = 0; i < NF; ++i) read(q % SETS, q, i);
#pragma unroll
    for (int q = 0; q + S::AHEAD < S::KS; ++q) quarter(q, std::true_type(), q + S::AHEAD, std::false_type(), none, none, 0, 0);
    int todo = n - S::SR;   // steps that request both operands
    const auto whole_steps = [&](int count) {
        for (; count > 0; --count) {
            wait_loads_and_barrier<IN_FLIGHT>();
            step(std::false_type(), all);
            next_r();
            next_f();
        }
    };
    const auto until_last = [&]() { return per_segment - 1 - (rat > fat ? rat : fat); };   // of either operand's segment
    for (int c; c = until_last(), c < todo;) {
        whole_steps(c);
        wait_loads_and_barrier<IN_FLIGHT>();
        step(std::true_type(), all);
        advance_r();
        advance_f();
        todo -= c + 1;
    }
    whole_steps(todo);
    if (S::SR > S::SF && n >= S::SR) {   // the features' last step
        wait_loads_and_barrier<IN_FLIGHT>();
        step(std::true_type(), features);
    }
    for (int s = n < S::SF ? n - 1 : S::SF - 1; s > 0; --s) {
        wait_loads_and_barrier<0>();
        step(std::false_type(), none);
    }
    lds_barrier();   // every wavefront is past its last read: the caller may use the LDS
#pragma unroll
    for (int q = S::KS - S::AHEAD; q < S::KS; ++q) quarter(q, std::false_type(), 0, std::false_type(), none, none, 0, 0);
}

// Few rows: a tile of 32 TR rows and 32 FT features (of one or two images) per block, each wavefront with every fourth step of the
// contraction, images and a ring of SLOTS of its own: no barrier, and as much of the weights in flight as the LDS holds.
template <int TR_, int FT_, int FL_, bool DUAL_, bool E4M3_, int BLOCKS> struct FewShape {
    static constexpr int TR = TR_, FT = FT_, FL = FL_, IMAGES = DUAL_ ? 2 : 1, KS = E4M3_ ? 2 : 4;
    static constexpr bool DUAL = DUAL_, E4M3 = E4M3_;
    static constexpr int BR = 32 * TR, BF = 32 * FT;
    typedef TileImage<kKContiguous, BR, 1> RI;
    typedef TileImage<FL, BF, 1> FI;
    static constexpr int SLOT = RI::BYTES + IMAGES * FI::BYTES, LOADS = RI::PER_WAVE + IMAGES * FI::PER_WAVE;
    static constexpr int FIT = 160 * 1024 / (4 * SLOT * BLOCKS), SLOTS = FIT < 4 ? FIT : 4;   // BLOCKS: per CU
    static_assert(SLOTS >= 1 && LOADS * (SLOTS - 1) < 64, "the wait counts to 63");
    static constexpr int STRIDE = BF + 4;                                    // floats of a row in the sums
    static constexpr int SUMS = 4 * IMAGES * BR * STRIDE * 4;
    static constexpr int LDS = 4 * SLOTS * SLOT > SUMS ? 4 * SLOTS * SLOT : SUMS;
};

// put(row of the tile, feature of the tile, eight values for each image) for the steps [s0, s1), the wavefronts' sums added in their order.
template <typename S, typename PUT> __device__ __forceinline__ void few_rows(const GemmProblem &p, int row0, int f0, int s0, int s1, char *lds, const PUT &put)
{
    typedef typename S::RI RI;
    typedef typename S::FI FI;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    constexpr int NT = S::IMAGES * S::FT;   // feature tiles: those of the first image, then those of the second
    f32x16 acc[NT][S::TR];
#pragma unroll
    for (int m = 0; m < NT; ++m)
#pragma unroll
        for (int u = 0; u < S::TR; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[m][u][i] = 0.f;

    const int n = (s1 - s0 - wave + 3) >> 2;   // this wavefront's steps (none: <= 0)
    char *mine = lds + wave * S::SLOTS * S::SLOT;
    const uint32_t mine0 = (uint32_t)(uintptr_t)as_lds(mine);
    uint32_t ro[RI::PER_WAVE], fo[FI::PER_WAVE];
    RI::offsets(ro, 0, lane, row0, p.nr, (uint32_t)p.ldr);
    FI::offsets(fo, 0, lane, f0, p.nf, (uint32_t)p.ldf);
    FragmentReader<kKContiguous, S::BR, S::E4M3> rr;
    FragmentReader<S::FL, S::BF, S::E4M3> fr;
    rr.init(0, lane);
    fr.init(0, lane);
    const int per_segment = (p.K + 127) >> 7;
    int seg = (s0 + wave) / per_segment, at = s0 + wave - seg * per_segment, slot = 0;
    const char *rp, *fp, *fp2 = nullptr;   // of the segment
    const auto enter = [&]() {
        rp = RI::corner(p.r[seg], row0, p.ldr);
        fp = FI::corner(p.f[seg], f0, p.ldf);
        if constexpr (S::DUAL) fp2 = FI::corner(p.f2[seg], f0, p.ldf);
    };
    if (n > 0) enter();
    const uint64_t rstep = RI::step_bytes(p.ldr), fstep = FI::step_bytes(p.ldf);
    const int segments = p.segments, K = p.K;
    const auto request = [&]() {
        const int left = K - 128 * at;
        const uint32_t to = mine0 + slot * S::SLOT;
        for_range<0, RI::PER_WAVE>([&](auto i) { RI::template request<true, decltype(i)::value>(to, rp + at * rstep, ro, 0, lane, left); });
        for_range<0, FI::PER_WAVE>([&](auto i) { FI::template request<true, decltype(i)::value>(to + RI::BYTES, fp + at * fstep, fo, 0, lane, left); });
        if constexpr (S::DUAL)
            for_range<0, FI::PER_WAVE>([&](auto i) { FI::template request<true, decltype(i)::value>(to + RI::BYTES + FI::BYTES, fp2 + at * fstep, fo, 0, lane, left); });
        slot = slot + 1 == S::SLOTS ? 0 : slot + 1;
        at += 4;
        if (at >= per_segment) {
            do {
                at -= per_segment;
                ++seg;
            } while (at >= per_segment);
            if (seg < segments) enter();
        }
    };
    for (int i = 0; i < S::SLOTS && i < n; ++i) request();
    int cur = 0;
    for (int j = 0; j < n; ++j) {
        if (j + S::SLOTS <= n) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(S::LOADS *(S::SLOTS - 1)) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        const char *image = mine + cur * S::SLOT;
        cur = cur + 1 == S::SLOTS ? 0 : cur + 1;
        typename FragmentReader<S::FL, S::BF, S::E4M3>::frag rf[S::KS][S::TR], ff[S::KS][NT];
#pragma unroll
        for (int k = 0; k < S::KS; ++k) {
#pragma unroll
            for (int u = 0; u < S::TR; ++u) rf[k][u] = rr.read(image, u, k);
#pragma unroll
            for (int m = 0; m < NT; ++m) ff[k][m] = fr.read(image + RI::BYTES + m / S::FT * FI::BYTES, m % S::FT, k);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the image is in registers: its place is free
        if (j + S::SLOTS < n) request();
#pragma unroll
        for (int k = 0; k < S::KS; ++k)
#pragma unroll
            for (int m = 0; m < NT; ++m)
#pragma unroll
                for (int u = 0; u < S::TR; ++u) {
                    if constexpr (S::E4M3)
                        acc[m][u] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(ff[k][m], rf[k][u], acc[m][u], 0, 0, 0, 0x7f7f7f7f, 0, 0x7f7f7f7f);
                    else
                        acc[m][u] = mfma_bf16(ff[k][m], rf[k][u], acc[m][u]);
                }
    }
    lds_barrier();   // every wavefront is done with its images
    float *sums = (float *)lds;
#pragma unroll
    for (int m = 0; m < NT; ++m)
#pragma unroll
        for (int u = 0; u < S::TR; ++u)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *(f32x4 *)(sums + ((wave * S::IMAGES + m / S::FT) * S::BR + 32 * u + (lane & 31)) * S::STRIDE + 32 * (m % S::FT) + 8 * q + 4 * (lane >> 5)) =
                    f32x4{acc[m][u][4 * q], acc[m][u][4 * q + 1], acc[m][u][4 * q + 2], acc[m][u][4 * q + 3]};
    lds_barrier();
    constexpr int PIECES = S::BF / 8;   // eight features of a row per thread
    for (int i = tid; i < PIECES * S::BR; i += 256) {
        const int row = i / PIECES, col = 8 * (i % PIECES);
        float v[S::IMAGES][8];
#pragma unroll
        for (int m = 0; m < S::IMAGES; ++m) {
            f32x4 a = {0.f, 0.f, 0.f, 0.f}, b = a;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float *q = sums + ((w * S::IMAGES + m) * S::BR + row) * S::STRIDE + col;
                a += *(const f32x4 *)q;
                b += *(const f32x4 *)(q + 4);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[m][e] = a[e];
                v[m][4 + e] = b[e];
            }
        }
        put(row, col, v);
    }
}

// Which tile and share of the contraction a block has: blocks of one XCD (blockIdx % 8) take consecutive tiles, in groups of eight row
// tiles, so that the operands they share stay in its L2.
struct TilePlace {
    int r, f, split;
};
__device__ __forceinline__ TilePlace tile_of(int block, int tiles_r, int tiles_f, int splits)
{
    const int total = tiles_r * tiles_f * splits, q = total >> 3, rem = total & 7, x = block & 7;
    int i = x * q + (x < rem ? x : rem) + (block >> 3);
    TilePlace t;
    t.split = i / (tiles_r * tiles_f);
    i -= t.split * tiles_r * tiles_f;
    const int group = 8 * tiles_f, first = i / group * 8, rows = tiles_r - first < 8 ? tiles_r - first : 8, in = i % group;
    t.f = in / rows;
    t.r = first + in % rows;
    return t;
}

}  // namespace slicemoe
