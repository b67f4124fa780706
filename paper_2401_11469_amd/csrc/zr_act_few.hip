// Forward products of up to 16 rows with bias, activation, gate, dropout and residual (bf16, gfx950): a decoding step.
//
// The weight shard has to be read once, 2 bytes for 2 M FLOP, and nothing else counts but how soon its loads are under way and how
// the chip is filled: sixteen wavefronts share the 16 (or 32) features of a workgroup and take every sixteenth step of 32
// contraction indices each, eight steps requested together, so that a shard of 4096 x 2752 is in flight as a whole.  The partial
// sums meet in LDS; a thread has asked for the bias, gate and residual of its element before the loop.
//   W stored [N x K]  rows of W are rows of the 16 x 16 x 32 MFMA as they are: 16-byte loads, 1 KB of each row for the workgroup's
//                     sixteen steps.  A kept list picks rows.
//   W stored [K x N]  32 features, 64 bytes of 32 rows a step, through 2 KB of LDS of the wavefront's own and the transposing read.
//                     A kept list picks rows of W and elements of X.
#include "zr_act.h"

namespace zr {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short v4i16 __attribute__((ext_vector_type(4)));

constexpr int WAVES = 16, NT = 64 * WAVES, STEP = 32;

struct FewArgs {
    const Bf* X; int64_t ldx;
    const Bf* W; int64_t ldw;
    const int32_t* rows;        // [N x K]: the kept rows of W, or nullptr; [K x N]: the kept contraction indices, or nullptr
    int extent;                 // of the axis that they index
    int M, J, C;                // rows of X, features multiplied, contraction
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

// KN: W stored [K x N].  ELEMS: X is read element by element (through the list, or where its rows are not 16-byte aligned).
template <bool KN, bool ELEMS>
__global__ __launch_bounds__(NT) void act_few_kernel(const FewArgs g)
{
    constexpr int FEATURES = KN ? 32 : 16, TILES = FEATURES / 16, U = !KN ? 8 : ELEMS ? 2 : 4;
    constexpr int PITCH = 20;                               // words of a row of 32 features in LDS (16 and 4: rows on other banks)
    __shared__ __align__(16) float part[WAVES][FEATURES][16];
    __shared__ __align__(16) uint32_t turn[KN ? WAVES : 1][KN ? STEP * PITCH : 4];
    __shared__ int sidx[FEATURES];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int j0 = (int)blockIdx.x * FEATURES, features = min(FEATURES, g.J - j0);
    const int n16 = lane & 15, q = lane >> 4;               // row of a fragment, which eight of the 32 contraction indices
    const bool scatter = !KN && g.rows;

    // this thread's element of the output, and what lies there
    Beside beside;
    const int my_m = tid / FEATURES, my_n = tid % FEATURES;
    const bool mine = my_m < g.M && my_n < features;
    if (scatter) {
        if (tid < features) sidx[tid] = clamp_idx(g.rows[j0 + tid], g.extent);
    } else if (mine) {
        beside.load(g.f, my_m, j0 + my_n);
    }

    f4 acc[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) acc[t] = f4{0.f, 0.f, 0.f, 0.f};
    const int steps = (g.C + STEP - 1) / STEP;
    const Bf* xrow = g.X + (size_t)min(n16, g.M - 1) * (size_t)g.ldx;

    // eight contraction indices of a row of X from c on (0 past the end)
    auto x_frag = [&](int c) -> u4 {
        if constexpr (!ELEMS) {
            u4 v = *(const u4*)(xrow + min(c, g.C - 8));    // (C is a multiple of 8)
            const bool ok = c < g.C;
            v.x = ok ? v.x : 0u; v.y = ok ? v.y : 0u; v.z = ok ? v.z : 0u; v.w = ok ? v.w : 0u;
            return v;
        } else {
            int at[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) at[e] = min(c + e, g.C - 1);
            if (KN && g.rows) {
#pragma unroll
                for (int e = 0; e < 8; ++e) at[e] = g.rows[at[e]];
#pragma unroll
                for (int e = 0; e < 8; ++e) at[e] = clamp_idx(at[e], g.extent);
            }
            uint32_t h[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) h[e] = xrow[at[e]];
            u4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = (c + 2 * e < g.C ? h[2 * e] : 0u) | (c + 2 * e + 1 < g.C ? h[2 * e + 1] << 16 : 0u);
            return v;
        }
    };

    if constexpr (!KN) {
        int row = j0 + min(n16, features - 1);
        if (scatter) row = clamp_idx(g.rows[row], g.extent);
        const Bf* wrow = g.W + (size_t)row * (size_t)g.ldw;
        for (int s0 = wave; s0 < steps; s0 += WAVES * U) {
            u4 w[U], x[U];
#pragma unroll
            for (int u = 0; u < U; ++u) w[u] = __builtin_nontemporal_load((const u4*)(wrow + min((s0 + WAVES * u) * STEP + 8 * q, g.C - 8)));
#pragma unroll
            for (int u = 0; u < U; ++u) x[u] = x_frag((s0 + WAVES * u) * STEP + 8 * q);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                // (past the end x is 0, and so must W be: what was read instead may be no number)
                const bool ok = (s0 + WAVES * u) * STEP + 8 * q < g.C;
                w[u].x = ok ? w[u].x : 0u; w[u].y = ok ? w[u].y : 0u; w[u].z = ok ? w[u].z : 0u; w[u].w = ok ? w[u].w : 0u;
                acc[0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_frag(w[u]), as_frag(x[u]), acc[0], 0, 0, 0);
            }
        }
    } else {
        typedef __attribute__((address_space(3))) v4i16* lp;
        const int at = j0 + 8 * (lane & 3), from = min(at, g.J - 8);          // (J is a multiple of 8: a chunk is within or past)
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
                for (int h = 0; h < 2; ++h) w[u][h] = __builtin_nontemporal_load((const u4*)(g.W + (size_t)row[u][h] * (size_t)g.ldw + from));
#pragma unroll
            for (int u = 0; u < U; ++u) x[u] = x_frag((s0 + WAVES * u) * STEP + 8 * q);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int c0 = (s0 + WAVES * u) * STEP;
                if (c0 >= g.C) break;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int r = (lane >> 2) + 16 * h;
                    u4 v = w[u][h];
                    const bool ok = c0 + r < g.C;
                    v.x = ok ? v.x : 0u; v.y = ok ? v.y : 0u; v.z = ok ? v.z : 0u; v.w = ok ? v.w : 0u;
                    *(u4*)(mine_lds + r * PITCH + 4 * (lane & 3)) = v;
                }
                // (a wavefront's LDS operations are done in their order)
                __builtin_amdgcn_wave_barrier();
                union { v4i16 h[2]; u4 u; } f[TILES];
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
    }

    // sums of the wavefronts, in their order: feature 4 q + r of a tile, row n16
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) part[wave][16 * t + 4 * q + r][n16] = acc[t][r];
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
    const int end = j0 + FEATURES >= g.J ? g.N : clamp_idx(g.rows[j0 + FEATURES], g.extent);
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

template <bool KN, bool ELEMS> int launch(const FewArgs& a, hipStream_t stream)
{
    const int features = KN ? 32 : 16;
    if (debug_names_wanted())
        snprintf(g_debug.last_kernel, sizeof(g_debug.last_kernel), "act_few_kernel<%s, %s>", KN ? "true" : "false", ELEMS ? "true" : "false");
    hipLaunchKernelGGL((act_few_kernel<KN, ELEMS>), dim3((unsigned)((a.J + features - 1) / features)), dim3(NT), 0, stream, a);
    return hip_status(hipGetLastError());
}

}  // namespace

// Returns -1 when the product is not for this kernel, else a zr_status.
int launch_act_few(const GemmDesc& d, hipStream_t stream)
{
    auto aligned = [](const Operand& o) { return (uintptr_t)o.base % 16 == 0 && o.ld % 8 == 0; };
    if (d.dtype != ZR_BF16 || d.I > ACT_FEW || !d.A.c_contig || d.B.map_contig || !aligned(d.B)) return -1;
    const bool x_chunks = !d.A.map_contig && aligned(d.A) && d.C % 8 == 0;
    FewArgs a;
    a.X = (const Bf*)d.A.base; a.ldx = d.A.ld; a.W = (const Bf*)d.B.base; a.ldw = d.B.ld;
    a.rows = d.B.map_strided; a.extent = d.B.n_strided;
    a.M = d.I; a.J = d.J; a.C = d.C; a.N = d.epilogue == EPI_COL_SCATTER ? d.out_full : d.J;
    a.out = (Bf*)d.out; a.ldo = d.ldo; a.f = *d.finish;
    if (d.B.c_contig) return x_chunks ? launch<false, false>(a, stream) : -1;
    if (d.J % 8 != 0 || d.epilogue != EPI_PLAIN) return -1;
    // X through a list must be W's: one contraction for both
    if (d.A.map_contig != d.B.map_strided) return -1;
    return x_chunks ? launch<true, false>(a, stream) : launch<true, true>(a, stream);
}

}  // namespace zr
