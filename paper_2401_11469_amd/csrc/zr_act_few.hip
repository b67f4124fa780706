// Forward products of up to 16 rows with bias, activation, gate, dropout and residual (bf16, gfx950): a decoding step.
//
// The weight shard has to be read once, 2 bytes for 2 M FLOP, and nothing else counts but how soon its loads are under way and how
// the chip is filled: the wavefronts of a workgroup share its features and take the steps of the contraction in turn, all of one
// wavefront's requested together (up to U), so that a shard of 4096 x 2752 is in flight as a whole.  The partial sums meet in LDS; a
// thread has asked for the bias, gate and residual of its element before the loop.
//   W stored [N x K]  rows of W are rows of the 16 x 16 x 32 MFMA as they are.  Of its 16 x 16 results a few rows of X need few: with
//                     M <= R = 4 or 8 the operands hold R features and rows of X, of 16 / R neighbouring stretches of the
//                     contraction each, and the results on the block diagonal are added up.  So a workgroup can have 16, 8 or 4
//                     features (small shards fill the chip) and reads 64, 128 or 256 bytes of a row at a time.  A kept list picks rows.
//   W stored [K x N]  32 features, 64 bytes of 32 rows a step, through 2.5 KB of LDS of the wavefront's own and the transposing read;
//                     neighbours, which share cache lines, run on one XCD.  A kept list picks rows of W and elements of X.
#include <cstdio>
#include <type_traits>

#include "zr_act.h"

namespace zr {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short v4i16 __attribute__((ext_vector_type(4)));


struct FewArgs {
    const Bf* X; int64_t ldx;
    const Bf* W; int64_t ldw;
    const int32_t* rows;        // [N x K]: the kept rows of W, or nullptr; [K x N]: the kept contraction indices, or nullptr
    int extent;                 // of the axis that they index
    int M, J, C;                // rows of X, features multiplied, contraction
    int x_extent;               // columns of X that may be read: C, or with zeros behind it a multiple of 64
    int N;                      // features of the output
    Bf* out; int64_t ldo;
    Finish f;
};

__device__ __forceinline__ bf16x8 as_frag(u4 v)
{
    union { u4 u; bf16x8 b; } x;
    x.u = v;
    return x.b;
}

// What is needed of one element of the output beside its sum.
struct Beside {
    float bias = 0.f, gate = 1.f, residual = 0.f;
    __device__ __forceinline__ void load(const Finish& f, int row, int col)
    {
        if (f.bias) bias = one_of((const Bf*)f.bias + col);
        if (f.gate) gate = one_of((const Bf*)f.gate + (size_t)row * (size_t)f.ldg + col);
        if (f.residual) residual = one_of((const Bf*)f.residual + (size_t)row * (size_t)f.ldr + col);
    }
    __device__ __forceinline__ void finish(const Finish& f, Bf* out, int64_t ldo, int row, int col, float z) const
    {
        float a, unused;
        z += bias;
        if (f.Z) put_one((Bf*)f.Z + (size_t)row * (size_t)f.ldz + col, z);
        act_one<false, false>(f.act, z, a, unused);
        a *= gate;
        if (f.drop) a = Draw(f.rng[0], f.rng[1], (uint32_t)row, (uint32_t)col >> 3).kept_at(col & 7, f.drop) ? a * f.factor : 0.f;
        put_one(out + (size_t)row * (size_t)ldo + col, a + residual);
    }
};

// ---- W stored [N x K] ----
constexpr int ROW_WAVES = 8;
template <int R, int U>
__global__ __launch_bounds__(64 * ROW_WAVES) void act_few_rows_kernel(const FewArgs g)
{
    constexpr int WAVES = ROW_WAVES, NT = 64 * WAVES, STRETCH = 16 / R, STEP = 32 * STRETCH;
    __shared__ __align__(16) float part[WAVES][R][17];
    __shared__ int sidx[R];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int j0 = (int)blockIdx.x * R, features = min(R, g.J - j0);
    // row of a fragment, its stretch, and which eight of the 32 contraction indices
    const int r16 = lane & (R - 1), k = 32 * ((lane & 15) / R) + 8 * (lane >> 4);
    const bool scatter = g.rows != nullptr;

    // this thread's element of the output, and what lies there
    static_assert(16 * R <= NT, "a thread for every element");
    Beside beside;
    const int my_m = tid / R, my_n = tid % R;
    const bool mine = my_m < g.M && my_n < features;
    if (scatter) {
        if (tid < features) sidx[tid] = clamp_idx(g.rows[j0 + tid], g.extent);
    } else if (mine) {
        beside.load(g.f, my_m, j0 + my_n);
    }
    const Bf* xrow = g.X + (size_t)min(r16, g.M - 1) * (size_t)g.ldx;
    int row = j0 + min(r16, features - 1);
    if (scatter) row = clamp_idx(g.rows[row], g.extent);
    const Bf* wrow = g.W + (size_t)row * (size_t)g.ldw;

    f4 acc = f4{0.f, 0.f, 0.f, 0.f};
    const int steps = (g.C + STEP - 1) / STEP;
    for (int s0 = wave; s0 < steps; s0 += WAVES * U) {
        u4 w[U], x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) w[u] = *(const u4*)(wrow + min((s0 + WAVES * u) * STEP + k, g.C - 8));       // (C is a multiple of 8)
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = *(const u4*)(xrow + min((s0 + WAVES * u) * STEP + k, g.C - 8));
#pragma unroll
        for (int u = 0; u < U; ++u) {
            // (past the end: zeros, of both, since what was read instead may be no number)
            const bool ok = (s0 + WAVES * u) * STEP + k < g.C;
#pragma unroll
            for (int e = 0; e < 4; ++e) { w[u][e] = ok ? w[u][e] : 0u; x[u][e] = ok ? x[u][e] : 0u; }
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_frag(w[u]), as_frag(x[u]), acc, 0, 0, 0);
        }
    }
    // feature row 4 (lane / 16) + r, row lane % 16 of X: those of one stretch, added up over the stretches
    const int m16 = lane & 15;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int n = 4 * (lane >> 4) + r;
        if constexpr (R == 16) {
            part[wave][n][m16] = acc[r];
        } else {
            // stretch t: features R t .. of rows R t ..; lanes of the same feature and row are R columns and R rows apart
            float v = n / R == m16 / R ? acc[r] : 0.f;
            if constexpr (R == 8) {
                v += __shfl_xor(v, 40, 64);                                   // (m ^ 8, n ^ 8)
            } else {
                v += __shfl_xor(v, 20, 64);                                   // (m ^ 4, n ^ 4)
                v += __shfl_xor(v, 40, 64);
            }
            if (n < R && m16 < R) part[wave][n][m16] = v;
        }
    }
    __syncthreads();
    if (!scatter) {
        if (!mine) return;
        float z = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) z += part[w][my_n][my_m];
        beside.finish(g.f, g.out, g.ldo, my_m, j0 + my_n, z);
        return;
    }
    // the workgroup owns the columns from its first kept one (0 for the first workgroup) to the next one's first
    const int start = j0 == 0 ? 0 : sidx[0];
    const int end = j0 + R >= g.J ? g.N : clamp_idx(g.rows[j0 + R], g.extent);
    const int owned = max(end - start, 0);
    for (int64_t u = tid; u < (int64_t)owned * g.M; u += NT) {
        const int m = (int)(u / owned), col = start + (int)(u - (int64_t)m * owned);
        Beside b;
        b.load(g.f, m, col);
        const int n = min(lower_bound_lds(sidx, features, col), features - 1);
        float z = 0.f;
        if (sidx[n] == col) {
#pragma unroll
            for (int w = 0; w < WAVES; ++w) z += part[w][n][m];
        }
        b.finish(g.f, g.out, g.ldo, m, col, z);
    }
}

// ---- W stored [K x N] ----
// ELEMS: X is read element by element (through the list, or where its rows are not 16-byte aligned); otherwise as it lies, also beside
// a list, which its columns have been picked by before.
template <bool ELEMS, int U>
__global__ __launch_bounds__(1024) void act_few_cols_kernel(const FewArgs g)
{
    constexpr int WAVES = 16, FEATURES = 32, TILES = 2, STEP = 32;
    constexpr int PITCH = 20;                               // words of a row of 32 features in LDS (16 and 4: rows on other banks)
    __shared__ __align__(16) float part[WAVES][FEATURES][17];
    __shared__ __align__(16) uint32_t turn[WAVES][STEP * PITCH];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lin = (int)((blockIdx.x % 8) * (gridDim.x / 8) + blockIdx.x / 8);           // (the grid is a multiple of 8)
    const int j0 = lin * FEATURES;
    if (j0 >= g.J) return;
    const int n16 = lane & 15, q = lane >> 4;               // row of a fragment, which eight of the 32 contraction indices

    Beside beside;
    const int my_m = tid / FEATURES, my_n = tid % FEATURES;
    const bool mine = my_m < g.M && j0 + my_n < g.J;
    if (mine) beside.load(g.f, my_m, j0 + my_n);

    f4 acc[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) acc[t] = f4{0.f, 0.f, 0.f, 0.f};
    const int steps = (g.C + STEP - 1) / STEP;
    const Bf* xrow = g.X + (size_t)min(n16, g.M - 1) * (size_t)g.ldx;
    const int from = min(j0 + 8 * (lane & 3), g.J - 8);     // (J is a multiple of 8: a chunk is within or past)
    uint32_t* mine_lds = turn[wave];
    for (int s0 = wave; s0 < steps; s0 += WAVES * U) {
        u4 w[U][2], x[U];
        int row[U][2];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) row[u][h] = min((s0 + WAVES * u) * STEP + (lane >> 2) + 16 * h, g.C - 1);
        if (g.rows) {
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int h = 0; h < 2; ++h) row[u][h] = g.rows[row[u][h]];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int h = 0; h < 2; ++h) row[u][h] = clamp_idx(row[u][h], g.extent);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) w[u][h] = *(const u4*)(g.W + (size_t)row[u][h] * (size_t)g.ldw + from);
        if constexpr (!ELEMS) {
#pragma unroll
            for (int u = 0; u < U; ++u) x[u] = *(const u4*)(xrow + min((s0 + WAVES * u) * STEP + 8 * q, g.x_extent - 8));       // (a multiple of 8)
        } else {
            int at[U][8];
            uint32_t h[U][8];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int e = 0; e < 8; ++e) at[u][e] = min((s0 + WAVES * u) * STEP + 8 * q + e, g.C - 1);
            if (g.rows) {
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int e = 0; e < 8; ++e) at[u][e] = g.rows[at[u][e]];
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int e = 0; e < 8; ++e) at[u][e] = clamp_idx(at[u][e], g.extent);
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int e = 0; e < 8; ++e) h[u][e] = xrow[at[u][e]];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e) x[u][e] = h[u][2 * e] | h[u][2 * e + 1] << 16;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c0 = (s0 + WAVES * u) * STEP;
            if (c0 >= g.C) break;
            // (past the end: zeros, of both, since what was read instead may be no number)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = (lane >> 2) + 16 * h;
                u4 v = w[u][h];
                const bool ok = c0 + r < g.C;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = ok ? v[e] : 0u;
                *(u4*)(mine_lds + r * PITCH + 4 * (lane & 3)) = v;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int c = c0 + 8 * q + 2 * e;
                x[u][e] = c + 1 < g.C ? x[u][e] : c < g.C ? x[u][e] & 0xffffu : 0u;
            }
            // (a wavefront's LDS operations are done in their order)
            __builtin_amdgcn_wave_barrier();
            union { v4i16 h[2]; u4 u; } f[TILES];
            typedef __attribute__((address_space(3))) v4i16* lp;
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                // a 16-lane group reads 4 contraction indices x 16 features; its lane n gets feature n's four
                const uint32_t* p = mine_lds + (8 * q + (n16 >> 2)) * PITCH + 8 * t + 2 * (n16 & 3);
                f[t].h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)p);
                f[t].h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(p + 4 * PITCH));
            }
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int t = 0; t < TILES; ++t)
                acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_frag(f[t].u), as_frag(x[u]), acc[t], 0, 0, 0);
        }
    }
    // feature 4 q + r of a tile, row n16
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) part[wave][16 * t + 4 * q + r][n16] = acc[t][r];
    __syncthreads();
    if (!mine) return;
    float z = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) z += part[w][my_n][my_m];
    beside.finish(g.f, g.out, g.ldo, my_m, j0 + my_n, z);
}

// ---- host side ----
// Steps that a wavefront requests together: all of its own, or equal shares of them.
int together(int steps, int waves, int most)
{
    const int each = (steps + waves - 1) / waves, rounds = (each + most - 1) / most;
    return (each + rounds - 1) / rounds;
}

template <class F> void pick(int u, F f)
{
    switch (u) {
        case 1: f(std::integral_constant<int, 1>()); break;
        case 2: f(std::integral_constant<int, 2>()); break;
        case 3: f(std::integral_constant<int, 3>()); break;
        case 4: f(std::integral_constant<int, 4>()); break;
        case 5: f(std::integral_constant<int, 5>()); break;
        case 6: f(std::integral_constant<int, 6>()); break;
        case 7: f(std::integral_constant<int, 7>()); break;
        default: f(std::integral_constant<int, 8>()); break;
    }
}

template <int R> int launch_rows(const FewArgs& a, hipStream_t stream)
{
    const int step = 32 * (16 / R), u = together((a.C + step - 1) / step, ROW_WAVES, 8);
    if (debug_names_wanted()) snprintf(g_debug.last_kernel, sizeof(g_debug.last_kernel), "act_few_rows_kernel<%d, %d>", R, u);
    pick(u, [&](auto un) {
        hipLaunchKernelGGL((act_few_rows_kernel<R, decltype(un)::value>), dim3((unsigned)((a.J + R - 1) / R)), dim3(64 * ROW_WAVES), 0, stream, a);
    });
    return hip_status(hipGetLastError());
}

template <bool ELEMS> int launch_cols(const FewArgs& a, hipStream_t stream)
{
    constexpr int MOST = ELEMS ? 3 : 6;
    const int u = together((a.C + 31) / 32, 16, MOST);
    if (debug_names_wanted()) snprintf(g_debug.last_kernel, sizeof(g_debug.last_kernel), "act_few_cols_kernel<%s, %d>", ELEMS ? "true" : "false", u);
    pick(u, [&](auto un) {
        constexpr int U = decltype(un)::value <= MOST ? decltype(un)::value : MOST;
        hipLaunchKernelGGL((act_few_cols_kernel<ELEMS, U>), dim3((unsigned)((a.J + 255) / 256 * 8)), dim3(1024), 0, stream, a);
    });
    return hip_status(hipGetLastError());
}

}  // namespace

// Returns -1 when the product is not for this kernel, else a zr_status.
int launch_act_few(const GemmDesc& d, hipStream_t stream)
{
    auto aligned = [](const Operand& o) { return (uintptr_t)o.base % 16 == 0 && o.ld % 8 == 0; };
    if (d.dtype != ZR_BF16 || d.I > ACT_FEW || !d.A.c_contig || d.B.map_contig || !aligned(d.B)) return -1;
    // (extracted columns have zeros behind them, to a multiple of 64)
    const int x_extent = d.A.zero_padded ? d.A.n_contig : d.C;
    const bool x_chunks = !d.A.map_contig && aligned(d.A) && x_extent % 8 == 0;
    FewArgs a;
    a.X = (const Bf*)d.A.base; a.ldx = d.A.ld; a.W = (const Bf*)d.B.base; a.ldw = d.B.ld;
    a.rows = d.B.map_strided; a.extent = d.B.n_strided;
    a.M = d.I; a.J = d.J; a.C = d.C; a.N = d.epilogue == EPI_COL_SCATTER ? d.out_full : d.J;
    a.out = (Bf*)d.out; a.ldo = d.ldo; a.f = *d.finish;
    a.x_extent = x_extent;
    if (d.B.c_contig) {
        if (!x_chunks || d.C % 8 != 0) return -1;
        // Features of a workgroup by measurement (us in a graph, 4 / 8 / 16 of them): one row, 2752 x 4096 7.0 / 8.1 / 7.5, 640 x 2560
        // 4.0 / 4.2 / 5.4, 11008 x 4096 17.3 / 19.0 / 20.0; four rows, 2752 x 4096 8.6 / 9.1 / 8.2, 1728 x 5120 7.7 / 6.8 / 9.5
        // (sixteen wavefronts in place of eight: as fast on 16, 4 to 35 % slower on 4)
        if (a.M == 1) return launch_rows<4>(a, stream);
        if (a.M <= 8 && a.J < 16 * 160) return launch_rows<8>(a, stream);
        return launch_rows<16>(a, stream);
    }
    if (d.J % 8 != 0 || d.epilogue != EPI_PLAIN) return -1;
    if (x_chunks) return launch_cols<false>(a, stream);
    // element by element through the list that picks rows of W, or where nothing is picked
    return d.A.map_contig == d.B.map_strided ? launch_cols<true>(a, stream) : -1;
}

}  // namespace zr
