// Gather-fused MFMA products of bf16 tensors of any alignment and any extents (gfx950): the
// resized layer's forward, dX and dW (paper Sec. 3.1) in the canonical form
//     D[i, j] = sum_c A(i, c) * B(j, c)
// on 64-wide wavefronts with the 16 x 16 x 32 MFMA and fp32 accumulation, for what the kernels
// with 16-byte aligned rows do not take: unaligned tensors, and products with few tiles.  The kept-index list is applied while the operand tiles
// travel into LDS, and the epilogue writes the result at its original positions together with the
// imputed values, so no compacted copy of an operand exists and one pass gives the normal shape.
//
// What bounds it.  Not the matrix cores: loads of 2-byte granularity that are waited for, and a
// chip that is not full.  So
//   * no load of tile elements stands under a branch (at a join the compiler waits for every load in
//     flight; lists are read under uniform branches, a stage ahead): rows and columns are clamped, a chunk at the end of a row is read from the row's last elements and
//     shifted into place, contraction indices past the end become zeros on the way into LDS;
//   * a stage is 16 KB of each operand (32 KB with 512 threads), requested two stages ahead;
//   * plain operands come in 16-byte loads at 2-byte alignment; kept columns come as the dword that
//     starts at the element (loads of 16 bits run at a quarter of the rate), two to an LDS word;
//   * tiles of 128 x 128, 64 x 64 or 32 x 32 by how many of them there are; the 32 x 32 tiles split
//     each stage's contraction over the four wavefronts, the 64 x 64 ones with 512 threads over two
//     groups of four.
// Measured against the kernel before this one (128 x 128 tiles, element loads under branches; three
// quarters of an axis kept): 985 x 1001 x 771 forward 151 -> 18 us, both backward products 253 -> 38;
// 4095 x 2001 x 1999 forward 544 -> 120 us (205 TFLOP/s), backward 1570 -> 229; accumulating
// 8192 x 4096 x 229 from misaligned rows 201 -> 70 us.
//
// LDS formats (bf16):
//   P  [row][contraction]  tensors whose contiguous axis is the contraction axis: ds_read_b128
//   Q  [contraction][row]  tensors whose contiguous axis is the other one: transposing reads
#pragma once

#include <algorithm>
#include <cstdio>
#include <type_traits>

#include "zr_act.h"
#include "zr_common.h"

namespace zr {

namespace {

constexpr int NP = 4;            // pieces a stage is brought in: 16 bytes of each operand per thread

typedef uint16_t E;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4_any __attribute__((ext_vector_type(4), aligned(2)));      // 16 bytes at any element
typedef uint32_t u1_any __attribute__((aligned(2)));                          // 4 bytes at any element

// R x R tiles, NT threads, BK contraction indices a stage (64 bytes of each operand per thread)
template <int R, int NT> struct Geo {
    static constexpr int BK = 32 * NT / R;
    static constexpr int PP = BK / 2 + 4;                 // words per row of format P: 16 rows of a fragment on 16 bank groups
    static constexpr int PQ = R / 2;                      // words per contraction index of format Q (swizzled)
    static constexpr int WORDS = R * PP;                  // LDS words of one operand's stage (the larger format)
    static_assert(WORDS >= BK * PQ, "format P is the larger one");
    // Format Q keeps 16-byte chunk `ch` of contraction index c at chunk ch ^ swz(c).  The transposing
    // reads of 32 lanes take 32 bytes from each of the contraction indices 8 g .. 8 g + 3 and
    // 8 g + 8 .. 8 g + 11: the swizzle gives these eight pieces eight different groups of 8 banks.
    static __device__ __forceinline__ constexpr int swz(int c)
    {
        return R == 128 ? 2 * ((c & 3) | ((c >> 1) & 4)) : R == 64 ? 2 * (((c >> 1) & 1) | ((c >> 2) & 2)) : 2 * ((c >> 3) & 1);
    }
};

struct View {
    const E* base;
    int64_t ld;
    const int32_t* map_s;       // row list on the strided axis or nullptr
    const int32_t* map_c;       // kept list on the contiguous axis or nullptr (the gathering loaders)
    int n_s, n_c;               // memory extents
};

struct Args {
    View A, B;
    int I, J, C;
    E* out;
    int64_t ldo;
    int epilogue;
    const int32_t* keep;
    int out_full;
    int tiles_i, tiles_j;
    const E* prev;              // Same imputation source (layout of out) or nullptr
    int accumulate;             // add the old contents of out (plain epilogue)
    int alternate;              // 64 x 64 tiles of 256 threads: every other stage goes to a second sum
};
struct FinishArgs : Args {
    Finish f;
    int j_base = 0;             // first column of D that the launch covers (the other kernels' tiles lie before it)
};

// element e of the result is element e + sh of v, 0 past its end (sh >= 0)
__device__ __forceinline__ u4 shifted(u4 v, int sh)
{
    const uint64_t lo = (uint64_t)v.x | ((uint64_t)v.y << 32), hi = (uint64_t)v.z | ((uint64_t)v.w << 32);
    const int s = 16 * (sh & 3);
    const uint64_t a = s ? (lo >> s) | (hi << (64 - s)) : lo, b = hi >> s;
    const uint64_t l = sh >= 8 ? 0 : sh >= 4 ? b : a, h = sh >= 4 ? 0 : b;
    u4 r;
    r.x = (uint32_t)l; r.y = (uint32_t)(l >> 32); r.z = (uint32_t)h; r.w = (uint32_t)(h >> 32);
    return r;
}

// ---------------------------------------------------------------------------
// Loaders.  Both LDS formats are lines (P: tile rows, Q: contraction indices) of elements that are
// neighbours in memory.  A loader keeps one stage of its operand in registers (begin, then fetch of
// four pieces) and writes it to LDS a stage later (commit, piece by piece).  Tile rows beyond the
// operand's extent repeat its last row (they only feed results that are never stored);
// contraction indices past C become zero (commit with TAIL, which only the last stage needs).
// ---------------------------------------------------------------------------
template <int R, int NT, bool P> struct Lines {
    static constexpr int BK = Geo<R, NT>::BK;
    static constexpr int COUNT = P ? R : BK;              // lines of a stage
    static constexpr int LEN = P ? BK : R;                // elements of a line
    // LDS word of 16-byte chunk ch of a line
    static __device__ __forceinline__ int chunk_at(int line, int ch)
    {
        return P ? line * Geo<R, NT>::PP + ch * 4 : line * Geo<R, NT>::PQ + (ch ^ Geo<R, NT>::swz(line)) * 4;
    }
};

// No list on the contiguous axis, which has at least 8 elements; optional row list.
template <int R, int NT, bool P_> struct Plain {
    static constexpr bool P = P_;
    typedef Lines<R, NT, P> L;
    static constexpr int CPL = L::LEN / 8, LPP = NT / CPL;       // chunks per line, lines per piece
    static constexpr bool ONE_STAGE = false;
    static_assert(L::COUNT == NP * LPP, "four pieces");
    const E* ptr[NP];       // P: the lines; Q: the lines of the stage being fetched, at this thread's column
    const E* colp;
    int row_[NP];           // Q: memory rows of the next stage
    int off_;               // P: element offset of the stage being fetched
    int sh_;                // Q: how far the clamp moved the column
    bool edge_;             // Q, uniform: the tile reaches past the stored rows' end
    u4 v[NP];

    __device__ __forceinline__ void rows_for(const View& op, int c0, int C, int tid)
    {
#pragma unroll
        for (int it = 0; it < NP; ++it) row_[it] = min(c0 + tid / CPL + LPP * it, C - 1);
        if (op.map_s) {
#pragma unroll
            for (int it = 0; it < NP; ++it) row_[it] = op.map_s[row_[it]];
        }
    }
    __device__ __forceinline__ void init(const View& op, int r0, int rlim, int C, int tid)
    {
        if constexpr (P) {
            int row[NP];
#pragma unroll
            for (int it = 0; it < NP; ++it) row[it] = min(r0 + tid / CPL + LPP * it, rlim - 1);
            if (op.map_s) {
#pragma unroll
                for (int it = 0; it < NP; ++it) row[it] = op.map_s[row[it]];
#pragma unroll
                for (int it = 0; it < NP; ++it) row[it] = clamp_idx(row[it], op.n_s);
            }
#pragma unroll
            for (int it = 0; it < NP; ++it) ptr[it] = op.base + (size_t)row[it] * (size_t)op.ld;
        } else {
            const int col = r0 + (tid % CPL) * 8, cc = min(col, op.n_c - 8);
            edge_ = r0 + R > op.n_c;
            sh_ = col - cc;
            colp = op.base + cc;
            rows_for(op, 0, C, tid);
        }
    }
    __device__ __forceinline__ void begin(const View& op, int c0, int C, int tid)
    {
        if constexpr (P) {
            // a chunk that would reach past the contraction range is read from its last eight
            // elements and shifted into place by commit
            off_ = min(c0 + (tid % CPL) * 8, C - 8);
        } else {
#pragma unroll
            for (int it = 0; it < NP; ++it) ptr[it] = colp + (size_t)clamp_idx(row_[it], op.n_s) * (size_t)op.ld;
            rows_for(op, c0 + L::BK, C, tid);
        }
    }
    template <int PC> __device__ __forceinline__ void fetch(const View&, int, int, int)
    {
        v[PC] = *(const u4_any*)(P ? ptr[PC] + off_ : ptr[PC]);
    }
    template <int PC, bool TAIL> __device__ __forceinline__ void commit(uint32_t* lds, int c0, int C, int tid) const
    {
        const int line = tid / CPL + LPP * PC;
        u4 x = v[PC];
        if constexpr (P) {
            if constexpr (TAIL) {
                const int c = c0 + (tid % CPL) * 8;
                x = shifted(x, c - min(c, C - 8));
            }
        } else {
            if (edge_) x = shifted(x, sh_);
            if constexpr (TAIL) {
                const bool ok = c0 + line < C;
                x.x = ok ? x.x : 0u; x.y = ok ? x.y : 0u; x.z = ok ? x.z : 0u; x.w = ok ? x.w : 0u;
            }
        }
        *(u4*)(lds + L::chunk_at(line, tid % CPL)) = x;
    }
};

// Kept list on the contiguous axis (of at least 2 elements): a thread owns two neighbours of the
// list, one LDS word, in every line it visits, so a wavefront's load runs along the (ascending)
// list in one memory row, or a few.
template <int R, int NT, bool P_> struct Gather {
    static constexpr bool P = P_;
    typedef Lines<R, NT, P> L;
    static constexpr bool ONE_STAGE = false;
    static constexpr int WPL = L::LEN / 2;                       // words per line
    static constexpr int LPI = NT / WPL;                         // lines per step of the workgroup
    static constexpr int N = L::COUNT / LPI;                     // words per thread
    static_assert(N == 4 * NP, "four words a piece");
    const E* base_;
    int64_t ld_;
    int line0_, llast_;     // first line of this thread in memory, last line there is
    const int32_t* list_;
    uint32_t a_, b_;        // columns of the stage being fetched
    int na_, nb_;           // list entries of the one after (P)
    uint32_t sel_, nsel_;   // byte selectors of the stage being written and of the one being fetched
    uint32_t lo[N], hi[N];

    // the dword that starts at the element; at the row's last element the one before it
    // (rounded down to aligned dwords instead, loads take the same time)
    __device__ __forceinline__ void columns(int a, int b, int n_c, bool oka, bool okb)
    {
        a = clamp_idx(a, n_c);
        b = clamp_idx(b, n_c);
        a_ = (uint32_t)min(a, n_c - 2);
        b_ = (uint32_t)min(b, n_c - 2);
        // v_perm byte selectors: 0-3 pick from lo, 4-7 from hi, 0x0c gives 0
        const uint32_t s0 = oka ? ((uint32_t)a == a_ ? 0x0100u : 0x0302u) : 0x0c0cu;
        const uint32_t s1 = okb ? ((uint32_t)b == b_ ? 0x0504u : 0x0706u) : 0x0c0cu;
        nsel_ = s0 | (s1 << 16);
    }
    __device__ __forceinline__ void entries(int c0, int C, int tid)
    {
        na_ = list_[min(c0 + 2 * (tid % WPL), C - 1)];
        nb_ = list_[min(c0 + 2 * (tid % WPL) + 1, C - 1)];
    }
    __device__ __forceinline__ void init(const View& op, int r0, int rlim, int C, int tid)
    {
        base_ = op.base; ld_ = op.ld; list_ = op.map_c;
        nsel_ = 0;
        if constexpr (P) {
            line0_ = r0 + tid / WPL;
            llast_ = rlim - 1;
            entries(0, C, tid);
        } else {
            llast_ = C - 1;
            const int j = r0 + 2 * (tid % WPL);
            columns(list_[min(j, rlim - 1)], list_[min(j + 1, rlim - 1)], op.n_c, true, true);
        }
    }
    __device__ __forceinline__ void begin(const View& op, int c0, int C, int tid)
    {
        sel_ = nsel_;
        if constexpr (P) {
            const int c = c0 + 2 * (tid % WPL);
            columns(na_, nb_, op.n_c, c < C, c + 1 < C);
            entries(c0 + L::BK, C, tid);
        } else {
            line0_ = c0 + tid / WPL;
        }
    }
    template <int PC> __device__ __forceinline__ void fetch(const View&, int, int, int)
    {
#pragma unroll
        for (int it = 4 * PC; it < 4 * PC + 4; ++it) {
            int line = min(line0_ + LPI * it, llast_);
            // (the same for a wavefront whose 64 threads share a line: scalar address arithmetic)
            if constexpr (WPL >= 64) line = __builtin_amdgcn_readfirstlane(line);
            const E* row = base_ + (int64_t)line * ld_;
            lo[it] = *(const u1_any*)(row + a_);
            hi[it] = *(const u1_any*)(row + b_);
        }
    }
    template <int PC, bool TAIL> __device__ __forceinline__ void commit(uint32_t* lds, int c0, int C, int tid) const
    {
        const int w = tid % WPL;
#pragma unroll
        for (int it = 4 * PC; it < 4 * PC + 4; ++it) {
            const int line = tid / WPL + LPI * it;
            uint32_t x = __builtin_amdgcn_perm(hi[it], lo[it], sel_);
            if constexpr (!P && TAIL) x = c0 + line < C ? x : 0u;
            lds[L::chunk_at(line, w / 4) + w % 4] = x;
        }
    }
};

// Element by element through whatever lists there are: for products with a contiguous extent
// below what the loaders above read at a time.  A thread owns two neighbours of every line it
// visits; lists are read once per tile (tile rows) or per stage (contraction indices).
template <int R, int NT, bool P_> struct Any {
    static constexpr bool P = P_;
    typedef Lines<R, NT, P> L;
    static constexpr int WPL = L::LEN / 2, LPI = NT / WPL, N = L::COUNT / LPI;
    static_assert(N == 4 * NP, "four words a piece");
    static constexpr bool ONE_STAGE = R != 32;            // (the host's rule: larger tiles are for contractions below eight)
    int line_[N];           // lines of the stage being fetched
    int a_, b_;             // columns of the stage being fetched
    uint32_t lo[N], hi[N];
    __device__ __forceinline__ void lines(const View& op, int first, int last, int tid)
    {
#pragma unroll
        for (int it = 0; it < N; ++it) line_[it] = min(first + tid / WPL + LPI * it, last);
        if (op.map_s) {
#pragma unroll
            for (int it = 0; it < N; ++it) line_[it] = op.map_s[line_[it]];
#pragma unroll
            for (int it = 0; it < N; ++it) line_[it] = clamp_idx(line_[it], op.n_s);
        }
    }
    __device__ __forceinline__ void columns(const View& op, int first, int last, int tid)
    {
        a_ = min(first + 2 * (tid % WPL), last);
        b_ = min(first + 2 * (tid % WPL) + 1, last);
        if (op.map_c) {
            a_ = clamp_idx(op.map_c[a_], op.n_c);
            b_ = clamp_idx(op.map_c[b_], op.n_c);
        }
    }
    __device__ __forceinline__ void init(const View& op, int r0, int rlim, int, int tid)
    {
        if constexpr (P) lines(op, r0, rlim - 1, tid);
        else columns(op, r0, rlim - 1, tid);
    }
    __device__ __forceinline__ void begin(const View& op, int c0, int C, int tid)
    {
        if constexpr (P) columns(op, c0, C - 1, tid);
        else lines(op, c0, C - 1, tid);
    }
    template <int PC> __device__ __forceinline__ void fetch(const View& op, int, int, int)
    {
#pragma unroll
        for (int it = 4 * PC; it < 4 * PC + 4; ++it) {
            const E* line = op.base + (size_t)line_[it] * (size_t)op.ld;
            lo[it] = line[a_];
            hi[it] = line[b_];
        }
    }
    template <int PC, bool TAIL> __device__ __forceinline__ void commit(uint32_t* lds, int c0, int C, int tid) const
    {
        const int w = tid % WPL;
#pragma unroll
        for (int it = 4 * PC; it < 4 * PC + 4; ++it) {
            const int line = tid / WPL + LPI * it;
            uint32_t l = lo[it], h = hi[it];
            if constexpr (TAIL) {
                const int c = c0 + (P ? 2 * w : line);
                l = c < C ? l : 0u;
                h = c + (P ? 1 : 0) < C ? h : 0u;
            }
            lds[L::chunk_at(line, w / 4) + w % 4] = l | (h << 16);
        }
    }
};

// Operand of a 16 x 16 x 32 MFMA: tile rows r0 .. r0 + 15 (lane & 15), eight contraction indices
// from 8 (lane >> 4) of the 32 that start at k0.
template <int R, int NT, bool P>
__device__ __forceinline__ bf16x8 fragment(const uint32_t* lds, int r0, int k0, int lane)
{
    union { u4 u; v4i16 h[2]; bf16x8 b; } x;
    if constexpr (P) {
        x.u = *(const u4*)(lds + (r0 + (lane & 15)) * Geo<R, NT>::PP + k0 / 2 + 4 * (lane >> 4));
    } else {
        // a 16-lane group reads 4 contraction indices x 16 rows; its lane n gets row n's four
        typedef __attribute__((address_space(3))) v4i16* lp;
        const int t16 = lane & 15, c = k0 + 8 * (lane >> 4) + (t16 >> 2), col = r0 + 4 * (t16 & 3);
        const uint32_t* p = lds + c * Geo<R, NT>::PQ + (((col >> 3) ^ Geo<R, NT>::swz(c)) << 2) + ((col & 7) >> 1);
        x.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)p);
        x.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(p + 4 * Geo<R, NT>::PQ));       // (the same swizzle)
    }
    return x.b;
}

__device__ __forceinline__ uint32_t two(float a, float b) { return f32_to_bf16_bits(a) | (f32_to_bf16_bits(b) << 16); }

// One workgroup's tile `lin` of a product (PAIRED: of one that may be asked to alternate between two sums; FinishArgs: with bias,
// activation and so on before the results are stored).
template <template <int, int, bool> class LA_, bool AP, template <int, int, bool> class LB_, bool BP, int R, int NT, bool PAIRED = false, class G = Args>
__device__ __forceinline__ void gemm_body(const G& g, uint32_t* smem, const int lin)
{
    typedef LA_<R, NT, AP> LA;
    typedef LB_<R, NT, BP> LB;
    constexpr int BK = Geo<R, NT>::BK;
    constexpr bool ONE_STAGE = LA::ONE_STAGE || LB::ONE_STAGE;
    constexpr int OP_WORDS = Geo<R, NT>::WORDS, STAGE = 2 * OP_WORDS;
    constexpr int WAVES = NT / 64;
    constexpr int T = R == 32 ? 2 : R / 32;                           // 16 x 16 results per wavefront and direction
    constexpr int WPT = R == 32 ? 1 : 4;                              // wavefronts that share a tile ...
    constexpr int KG = WAVES / WPT;                                   // ... and groups of them that share the contraction
    constexpr bool SPLIT = KG > 1;
    constexpr int STEPS = BK / KG / 32;                               // 32-deep steps per wavefront and stage
    constexpr int CP = R + 4;                                         // row pitch of the result tile (floats)
    constexpr int TAB = 512;                                          // original columns per pass of the column scatter
    constexpr int PART = SPLIT ? KG * R * CP : 0;                     // the groups' sums
    static_assert(R * CP + PART + 2 * R + TAB <= 2 * STAGE, "the epilogue fits the stages");

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;

    if (lin >= g.tiles_i * g.tiles_j) return;
    const int grp_sz = 4 * g.tiles_j;
    const int first_i = lin / grp_sz * 4, within = lin % grp_sz;
    const int rows_in = min(4, g.tiles_i - first_i);
    int j0 = within / rows_in * R;
    const int i0 = (first_i + within % rows_in) * R;
    if constexpr (std::is_same_v<G, FinishArgs>) j0 += g.j_base;

    const int wr0 = WPT == 1 ? 0 : ((wave >> 1) & 1) * (R / 2), wc0 = WPT == 1 ? 0 : (wave & 1) * (R / 2);
    const int k0 = wave / WPT * (BK / KG);

    // (tiles of 512 threads add up the two halves of each stage, 128 deep, on their own; ALT: the same order on 256 threads,
    // whose stages are those halves)
    constexpr bool ALT = PAIRED && R == 64 && NT == 256;
    f32x4 acc[T][T], other[ALT ? T : 1][ALT ? T : 1];
#pragma unroll
    for (int a = 0; a < T; ++a)
#pragma unroll
        for (int b = 0; b < T; ++b)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                acc[a][b][r] = 0.f;
                if constexpr (ALT) other[a][b][r] = 0.f;
            }

    // While stage k is multiplied, stage k + 1 (requested during stage k - 1) goes from registers
    // to the other LDS buffer and stage k + 2 is requested, a piece at a time between the MFMAs.
    LA la;
    LB lb;
    const int KT = (g.C + BK - 1) / BK;
    la.init(g.A, i0, g.I, g.C, tid);
    lb.init(g.B, j0, g.J, g.C, tid);
    auto begin = [&](int kt) { la.begin(g.A, kt * BK, g.C, tid); lb.begin(g.B, kt * BK, g.C, tid); };
    auto fetch = [&](int kt, auto piece) {
        la.template fetch<decltype(piece)::value>(g.A, kt * BK, g.C, tid);
        lb.template fetch<decltype(piece)::value>(g.B, kt * BK, g.C, tid);
    };
    auto commit = [&](uint32_t* stage, int kt, auto piece, auto tail) {
        la.template commit<decltype(piece)::value, decltype(tail)::value>(stage, kt * BK, g.C, tid);
        lb.template commit<decltype(piece)::value, decltype(tail)::value>(stage + OP_WORDS, kt * BK, g.C, tid);
    };
    auto all = [](auto f) {
        f(std::integral_constant<int, 0>());
        f(std::integral_constant<int, 1>());
        f(std::integral_constant<int, 2>());
        f(std::integral_constant<int, 3>());
    };
    begin(0);
    all([&](auto p) { fetch(0, p); });
    if constexpr (!ONE_STAGE) begin(1);  // (past the end of a short contraction: valid addresses, zeros)
    all([&](auto p) {
        commit(smem, 0, p, std::true_type());
        if constexpr (!ONE_STAGE) fetch(1, p);
    });
    __syncthreads();

    // fetches: there is a stage k + 2; else stage k + 1, if there is one, is the last
    auto step = [&](int kt, auto commits, auto fetches) {
        const uint32_t* as = smem + (kt & 1) * STAGE;
        const uint32_t* bs = as + OP_WORDS;
        uint32_t* nx = smem + ((kt + 1) & 1) * STAGE;
        if constexpr (decltype(commits)::value) begin(kt + 2);
        all([&](auto piece) {
            constexpr int PC = decltype(piece)::value;
            if constexpr (decltype(commits)::value)
                commit(nx, kt + 1, piece, std::integral_constant<bool, !decltype(fetches)::value>());
            if constexpr (decltype(fetches)::value) fetch(kt + 2, piece);
#pragma unroll
            for (int k = PC * STEPS / NP; k < (PC + 1) * STEPS / NP; ++k) {
                bf16x8 af[T], bf[T];
#pragma unroll
                for (int a = 0; a < T; ++a) af[a] = fragment<R, NT, AP>(as, wr0 + 16 * a, k0 + 32 * k, lane);
#pragma unroll
                for (int b = 0; b < T; ++b) bf[b] = fragment<R, NT, BP>(bs, wc0 + 16 * b, k0 + 32 * k, lane);
#pragma unroll
                for (int a = 0; a < T; ++a)
#pragma unroll
                    for (int b = 0; b < T; ++b)
                        acc[a][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(af[a], bf[b], acc[a][b], 0, 0, 0);
            }
        });
        if constexpr (ALT) {
            if (g.alternate) {
#pragma unroll
                for (int a = 0; a < T; ++a)
#pragma unroll
                    for (int b = 0; b < T; ++b) {
                        const f32x4 x = acc[a][b];
                        acc[a][b] = other[a][b];
                        other[a][b] = x;
                    }
            }
        }
        __syncthreads();
    };
    int kt = 0;
    if constexpr (!ONE_STAGE) {
        for (; kt + 2 < KT; ++kt) step(kt, std::true_type(), std::true_type());
        if (kt + 1 < KT) step(kt++, std::true_type(), std::false_type());
    }
    step(kt, std::false_type(), std::false_type());

    if constexpr (ALT) {
        if (g.alternate) {
#pragma unroll
            for (int a = 0; a < T; ++a)
#pragma unroll
                for (int b = 0; b < T; ++b)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[a][b][r] += other[a][b][r];
        }
    }

    // ---- result tile in LDS, in fp32 --------------------------------------------
    float* Cs = (float*)smem;
    float* dst = SPLIT ? Cs + R * CP + wave / WPT * (R * CP) : Cs;
#pragma unroll
    for (int a = 0; a < T; ++a)
#pragma unroll
        for (int b = 0; b < T; ++b)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                dst[(wr0 + 16 * a + 4 * (lane >> 4) + r) * CP + wc0 + 16 * b + (lane & 15)] = acc[a][b][r];
    if constexpr (SPLIT) {
        // the groups' sums, in their order
        __syncthreads();
        for (int q = tid; q < R * R / 4; q += NT) {
            const int at = q / (R / 4) * CP + q % (R / 4) * 4;
            f32x4 sum = *(const f32x4*)(Cs + R * CP + at);
#pragma unroll
            for (int w = 1; w < KG; ++w) {
                const f32x4 x = *(const f32x4*)(Cs + (w + 1) * (R * CP) + at);
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[e] += x[e];
            }
            *(f32x4*)(Cs + at) = sum;
        }
    }
    int* sidx = (int*)(smem + R * CP + PART);
    const int rows_valid = min(R, g.I - i0), cols_valid = min(R, g.J - j0);
    const bool scatter_c = g.epilogue == EPI_COL_SCATTER, scatter_r = g.epilogue == EPI_ROW_SCATTER;
    if (scatter_c && tid < cols_valid) sidx[tid] = clamp_idx(g.keep[j0 + tid], g.out_full);
    if (scatter_r && tid < rows_valid) sidx[tid] = clamp_idx(g.keep[i0 + tid], g.out_full);
    __syncthreads();

    if constexpr (std::is_same_v<G, FinishArgs>) {
        const int start = !scatter_c || j0 == 0 ? 0 : sidx[0];
        const int end = !scatter_c ? 0 : j0 + R >= g.J ? g.out_full : clamp_idx(g.keep[j0 + R], g.out_full);
        finish_tile<NT, R, TAB, 4>(g.f, g.out, g.ldo, Cs, CP, i0, rows_valid, j0, cols_valid, scatter_c ? sidx : nullptr, start, end, sidx + 2 * R, tid);
        return;
    }
    if (scatter_c) {
        // The tile owns the original columns from its first kept column (0 for the first tile) up to
        // the next tile's first kept column (the full width for the last tile).  A table says which
        // result column, if any, belongs to each; then whole rows of owned columns leave, kept and
        // imputed ones together, two columns to a thread.
        int* tab = sidx + 2 * R;
        const int start = j0 == 0 ? 0 : sidx[0];
        const int end = j0 + R >= g.J ? g.out_full : clamp_idx(g.keep[j0 + R], g.out_full);
        // a long range behind the tile's last kept column needs no table
        const int last = max(start, sidx[cols_valid - 1] + 1), mid = end - last >= 512 ? last : end;
        for (int base = start; base < mid; base += TAB) {
            const int width = min(TAB, mid - base);
            for (int q = tid; q < TAB; q += NT) tab[q] = -1;
            __syncthreads();
            if (tid < cols_valid) {
                const int p = sidx[tid] - base;
                if (p >= 0 && p < width) tab[p] = tid;
            }
            __syncthreads();
            for (int cb = 0; cb < width; cb += 128) {
                // 64, 32 or 16 lanes to a row by what is left of the columns
                const int left = width - cb, lpr = left > 64 ? 64 : left > 32 ? 32 : 16, rpw = 64 / lpr;
                const int q = cb + 2 * (lane & (lpr - 1));
                if (q >= width) continue;
                const int ja = tab[q], jb = tab[q + 1];
                const bool pair = q + 1 < width;
                E* o = g.out + (size_t)i0 * (size_t)g.ldo + base + q;
                const E* pv = g.prev ? g.prev + (size_t)i0 * (size_t)g.ldo + base + q : nullptr;
                const int step = WAVES * rpw;
                constexpr int UB = 8;
                for (int r0 = wave * rpw + lane / lpr; r0 < rows_valid; r0 += step * UB) {
                    uint32_t x[UB];
#pragma unroll
                    for (int u = 0; u < UB; ++u) x[u] = 0u;
                    if (pv && (ja < 0 || jb < 0)) {
                        // (a position is read and written by this thread only, also where the
                        // previous tensor is the output itself)
                        if (pair) {
#pragma unroll
                            for (int u = 0; u < UB; ++u)
                                x[u] = *(const u1_any*)(pv + (size_t)min(r0 + step * u, rows_valid - 1) * (size_t)g.ldo);
                        } else {
#pragma unroll
                            for (int u = 0; u < UB; ++u)
                                x[u] = pv[(size_t)min(r0 + step * u, rows_valid - 1) * (size_t)g.ldo];
                        }
                    }
#pragma unroll
                    for (int u = 0; u < UB; ++u) {
                        const int row = min(r0 + step * u, rows_valid - 1);
                        if (ja >= 0) x[u] = (x[u] & 0xffff0000u) | f32_to_bf16_bits(Cs[row * CP + ja]);
                        if (jb >= 0) x[u] = (x[u] & 0xffffu) | (f32_to_bf16_bits(Cs[row * CP + jb]) << 16);
                    }
#pragma unroll
                    for (int u = 0; u < UB; ++u) {
                        if (r0 + step * u >= rows_valid) break;
                        E* p = o + (size_t)(r0 + step * u) * (size_t)g.ldo;
                        if (pair) *(u1_any*)p = x[u];
                        else *p = (E)x[u];
                    }
                }
            }
            __syncthreads();
        }
        // and leaves 16 bytes a lane
        for (int r0 = wave; r0 < rows_valid && mid < end; r0 += 4 * WAVES) {
            for (int p = mid + lane * 8; p < end; p += 512) {
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int row = r0 + WAVES * u;
                    if (row >= rows_valid) break;
                    const size_t off = (size_t)(i0 + row) * (size_t)g.ldo + p;
                    if (p + 8 <= end) {
                        u4 v = u4{0u, 0u, 0u, 0u};
                        if (g.prev) v = *(const u4_any*)(g.prev + off);
                        *(u4_any*)(g.out + off) = v;
                    } else {
                        for (int e = 0; e < end - p; ++e) g.out[off + e] = g.prev ? g.prev[off + e] : E(0);
                    }
                }
            }
        }
        return;
    }

    constexpr int CPR = R / 8, CHUNKS = (R * CPR + NT - 1) / NT;
    if (g.accumulate && R * CPR % NT == 0 && rows_valid == R && cols_valid == R && g.tiles_i * g.tiles_j > 512) {
        // a whole tile: its old values are requested together (not where every tile has a place at once: 128 x 128, 18 deep,
        // 448 tiles 10.3 us, 11.3 with it; 1500 tiles 0.86 to 0.97 of the time)
        E* o[CHUNKS];
        u4 old[CHUNKS];
#pragma unroll
        for (int it = 0; it < CHUNKS; ++it) {
            const int q = tid + NT * it;
            o[it] = g.out + (size_t)(i0 + q / CPR) * (size_t)g.ldo + j0 + q % CPR * 8;
            old[it] = *(const u4_any*)o[it];
        }
#pragma unroll
        for (int it = 0; it < CHUNKS; ++it) {
            const int q = tid + NT * it;
            const float* c = Cs + q / CPR * CP + q % CPR * 8;
            const f32x4 x0 = *(const f32x4*)c, x1 = *(const f32x4*)(c + 4);
            u4 w;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const f32x4 x = e < 2 ? x0 : x1;
                w[e] = two(x[2 * (e & 1)] + __uint_as_float(old[it][e] << 16), x[2 * (e & 1) + 1] + __uint_as_float(old[it][e] & 0xffff0000u));
            }
            *(u4_any*)o[it] = w;
        }
        return;
    }
#pragma unroll
    for (int it = 0; it < CHUNKS; ++it) {
        const int q = tid + NT * it;
        const int row = q / CPR, j = (q % CPR) * 8;
        if (row >= rows_valid || j >= cols_valid) continue;
        E* o = g.out + (size_t)(scatter_r ? sidx[row] : i0 + row) * (size_t)g.ldo + j0 + j;
        f32x4 x0 = *(const f32x4*)(Cs + row * CP + j), x1 = *(const f32x4*)(Cs + row * CP + j + 4);
        if (j + 8 <= cols_valid) {
            if (g.accumulate) {
                const u4 old = *(const u4_any*)o;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    x0[2 * e] += __uint_as_float(old[e] << 16);
                    x0[2 * e + 1] += __uint_as_float(old[e] & 0xffff0000u);
                    x1[2 * e] += __uint_as_float(old[e + 2] << 16);
                    x1[2 * e + 1] += __uint_as_float(old[e + 2] & 0xffff0000u);
                }
            }
            u4 w;
            w.x = two(x0[0], x0[1]); w.y = two(x0[2], x0[3]); w.z = two(x1[0], x1[1]); w.w = two(x1[2], x1[3]);
            *(u4_any*)o = w;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (j + e < cols_valid) {
                    const float x = e < 4 ? x0[e & 3] : x1[e & 3];
                    o[e] = (E)f32_to_bf16_bits(g.accumulate ? bf16_bits_to_f32(o[e]) + x : x);
                }
        }
    }
    if (scatter_r) {
        // the dropped rows this tile owns (same ownership rule as above): every lane looks one row
        // up, the wavefront then writes the dropped ones together
        const int start = i0 == 0 ? 0 : sidx[0];
        const int end = i0 + R >= g.I ? g.out_full : clamp_idx(g.keep[i0 + R], g.out_full);
        for (int base = start + wave * 64; base < end; base += NT) {
            const int mine = base + lane;
            bool dropped = false;
            if (mine < end) {
                const int ii = lower_bound_lds(sidx, rows_valid, mine);
                dropped = !(ii < rows_valid && sidx[ii] == mine);
            }
            unsigned long long todo = __ballot(dropped);
            while (todo) {
                // a row to every CPR lanes, 16 bytes a lane
                int p = -1;
#pragma unroll
                for (int u = 0; u < 64 / CPR; ++u) {
                    if (todo && u == lane / CPR) p = base + (__ffsll((long long)todo) - 1);
                    todo &= todo - 1;                         // (0 stays 0)
                }
                const int j = lane % CPR * 8;
                if (p < 0 || j >= cols_valid) continue;
                const size_t off = (size_t)p * (size_t)g.ldo + j0 + j;
                if (j + 8 <= cols_valid) {
                    u4 v = u4{0u, 0u, 0u, 0u};
                    if (g.prev) v = *(const u4_any*)(g.prev + off);
                    *(u4_any*)(g.out + off) = v;
                } else {
                    for (int e = 0; e < cols_valid - j; ++e) g.out[off + e] = g.prev ? g.prev[off + e] : E(0);
                }
            }
        }
    }
}

// every XCD gets a contiguous range of tiles, ordered in groups of 4 tile rows
template <template <int, int, bool> class LA, bool AP, template <int, int, bool> class LB, bool BP, int R, int NT>
__global__ __launch_bounds__(NT, 512 / NT) void gemm_kernel(const Args g)
{
    extern __shared__ __align__(16) uint32_t smem[];
    gemm_body<LA, AP, LB, BP, R, NT>(g, smem, (int)((blockIdx.x % 8) * (gridDim.x / 8) + blockIdx.x / 8));
}

// the same, with bias, activation and so on
template <template <int, int, bool> class LA, bool AP, template <int, int, bool> class LB, bool BP, int R, int NT>
__global__ __launch_bounds__(NT, 512 / NT) void act_kernel(const FinishArgs g)
{
    extern __shared__ __align__(16) uint32_t smem[];
    gemm_body<LA, AP, LB, BP, R, NT>(g, smem, (int)((blockIdx.x % 8) * (gridDim.x / 8) + blockIdx.x / 8));
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
template <template <int, int, bool> class LA, bool AP, template <int, int, bool> class LB, bool BP, int R, int NT, class G>
int launch_inst(const G& a, const char* name, hipStream_t stream)
{
    constexpr int smem = 2 * 2 * Geo<R, NT>::WORDS * 4;
    constexpr bool finishes = std::is_same_v<G, FinishArgs>;
    const auto fn = [] { if constexpr (finishes) return act_kernel<LA, AP, LB, BP, R, NT>; else return gemm_kernel<LA, AP, LB, BP, R, NT>; }();
    static AttrFlags attr_set;      // per instantiation and device
    if (!ensure_max_dynamic_lds((const void*)fn, smem, &attr_set)) return ZR_ERR_HIP;
    if (debug_names_wanted())
        snprintf(g_debug.last_kernel, sizeof(g_debug.last_kernel), "%s_kernel<%s, %d, %d>", finishes ? "act" : "gemm", name, R, NT);
    G k = a;
    k.tiles_i = (a.I + R - 1) / R;
    k.tiles_j = (a.J + R - 1) / R;
    if constexpr (finishes) k.tiles_j = (a.J - a.j_base + R - 1) / R;
    const int64_t tiles = (int64_t)k.tiles_i * k.tiles_j;
    if (tiles > 0x7ffffff0) return ZR_ERR_LIMIT;
    hipLaunchKernelGGL(fn, dim3((unsigned)((tiles + 7) / 8 * 8)), dim3(NT), smem, stream, k);
    return hip_status(hipGetLastError());
}

template <template <int, int, bool> class LA, bool AP, template <int, int, bool> class LB, bool BP, class G>
int launch_shape(const G& a, const char* name, hipStream_t stream)
{
    const int64_t t64 = (int64_t)((a.I + 63) / 64) * ((a.J + 63) / 64), t128 = (int64_t)((a.I + 127) / 128) * ((a.J + 127) / 128);
    // 32 x 32 tiles below 96 of 64 x 64 (dW 376 x 471 over 985 tokens: 48 tiles, 8 us against 15; 985 x 501 x 353:
    // 96 tiles, 14.1 against 13.6);
    if (forced_tiles()) return launch_inst<LA, AP, LB, BP, 128, 256>(a, name, stream);
    if (t64 < 96) return launch_inst<LA, AP, LB, BP, 32, 256>(a, name, stream);
    // 512 threads on a 64 x 64 tile while each has a compute unit to itself (985 x 1001 x 578
    // plain 14.1 -> 12.8 us, dW 2024 tokens 27.4 -> 24.7; 288 tiles: 25.0 -> 31.3, so not there; on
    // 32 x 32 tiles within 5 %, on either side); below two stages of the others it gains nothing
    // (256 deep, kept columns gathered, 128 tiles 15.1 -> 12.9);
    if (adds_in_groups(a.I, a.J, a.C)) return launch_inst<LA, AP, LB, BP, 64, 512>(a, name, stream);
    // 128 x 128 tiles once there is one for every compute unit (M x K x N = 4001 x 752 x 1003: 256 tiles
    // 28.8 us against 39.0 on 64 x 64; 4001 x 1001 x 752: 192 tiles 49.2 against 40.5), or for half of them
    // where kept columns of A are gathered (1024 deep, 160 tiles: 27.3 against 35.4, both operands 40.5 against 60.8;
    // 128 tiles: 27.0 against 24.4)
    constexpr bool gathers_a = AP && std::is_same<LA<128, 256, AP>, Gather<128, 256, AP>>::value;
    if (t128 >= 256 || (gathers_a && t128 > 128)) return launch_inst<LA, AP, LB, BP, 128, 256>(a, name, stream);
    return launch_inst<LA, AP, LB, BP, 64, 256>(a, name, stream);
}

// The element loaders.  A contraction of less than eight is one stage of any tile shape, however
// little of the stage it fills, so the larger tiles mean fewer of them (accumulating, 3 deep, us on
// 128 x 128 / 64 x 64 / 32 x 32 tiles: 8192 x 4096 43 / 72 / 267, 1000 x 1000 10.1 / 7.8 / 11.2); otherwise
// the result has less than eight rows or columns, and the narrowest tiles waste least.
template <template <int, int, bool> class LA, bool AP, template <int, int, bool> class LB, bool BP, class G>
int launch_short(const G& a, const char* name, hipStream_t stream)
{
    if (a.C < 8) {
        const int64_t t64 = (int64_t)((a.I + 63) / 64) * ((a.J + 63) / 64), t128 = (int64_t)((a.I + 127) / 128) * ((a.J + 127) / 128);
        if (t128 >= 192) return launch_inst<LA, AP, LB, BP, 128, 256>(a, name, stream);
        if (t64 >= 96) return launch_inst<LA, AP, LB, BP, 64, 256>(a, name, stream);
    }
    return launch_inst<LA, AP, LB, BP, 32, 256>(a, name, stream);
}

inline Args args_of(const GemmDesc& d)
{
    Args a;
    a.A = View{(const E*)d.A.base, d.A.ld, d.A.map_strided, d.A.map_contig, d.A.n_strided, d.A.n_contig};
    a.B = View{(const E*)d.B.base, d.B.ld, d.B.map_strided, d.B.map_contig, d.B.n_strided, d.B.n_contig};
    a.I = d.I; a.J = d.J; a.C = d.C;
    a.out = (E*)d.out; a.ldo = d.ldo; a.epilogue = d.epilogue; a.keep = d.keep_idx; a.out_full = d.out_full;
    a.tiles_i = a.tiles_j = 0;
    a.prev = (const E*)d.prev; a.accumulate = d.accumulate ? 1 : 0;
    a.alternate = 0;
    return a;
}

inline bool too_short(const GemmDesc& d, const Operand& o) { return o.map_contig ? o.n_contig < 2 : (o.c_contig ? d.C : o.n_contig) < 8; }

}  // namespace

}  // namespace zr
