// Forward products with bias, activation, gate, dropout and residual, of bf16 tensors with 16-byte aligned rows: the loops and tile
// shapes of zr_gemm_fast.h with finish_tile at their end.  MFMA bound up to there, then by the way of the end's tensors, which one of
// two tiles on a compute unit can overlap and a 256 x 256 one cannot: 8192 x 1024 x 1024 with bias, GELU and Z 24 to 26 us (the product alone 20),
// 8192 x 4096 x 2752 of 2064 kept with SiLU, gate and Z 146 to 167 (135 alone; 135 MB more to move, 25 us of HBM).
#include "zr_gemm_fast.h"

namespace zr {

namespace {

template <template <int, int> class LA, template <int, int> class LB, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void act_fast_kernel(const FinishFArgs g)
{
    extern __shared__ __align__(16) uint32_t smem[];
    fast_body<LA, LB, BM, BN, WM, WN, 0, PART_NONE>(g, smem, (int)((blockIdx.x % 8) * (gridDim.x / 8) + blockIdx.x / 8));
}

// First launch of a split contraction.
template <template <int, int> class LA, template <int, int> class LB>
__global__ __launch_bounds__(256) void act_slice_kernel(const FArgs g)
{
    extern __shared__ __align__(16) uint32_t smem[];
    fast_body<LA, LB, 128, 128, 2, 2, 1>(g, smem, (int)((blockIdx.x % 8) * (gridDim.x / 8) + blockIdx.x / 8));
}

// Second launch of a split contraction (128 x 128 tiles, four wavefronts): the slices' accumulators, as fast_body's first phase leaves
// them, are added in slice order.  Four workgroups to a tile, each with one 16-row strip of both wavefront rows.
__global__ __launch_bounds__(256) void act_reduce_kernel(const FinishFArgs g)
{
    constexpr int BN = 128, CP = BN + 4, NT = 256;
    __shared__ __align__(16) float Cs[32 * CP];
    __shared__ int sidx[BN];
    __shared__ __align__(16) int tab[FINISH_TAB];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int total = g.tiles_i * g.tiles_j, t = (int)blockIdx.x >> 2, strip = blockIdx.x & 3;
    int ti, tj;
    tile_at(g, t, ti, tj);
    const int i0 = g.i_base + ti * 128, j0 = g.j_base + tj * BN;
    const int cols = min(BN, g.J - j0);
    const bool scatter = g.epilogue == EPI_COL_SCATTER;
    if (scatter && tid < cols) sidx[tid] = clamp_idx(g.keep[j0 + tid], g.out_full);
    float4 sum[4];
    const float4* p = (const float4*)g.partial + (size_t)t * (size_t)(16 * NT) + strip * 4 * NT + tid;
    const size_t slice = (size_t)total * (size_t)(16 * NT);
#pragma unroll
    for (int b = 0; b < 4; ++b) sum[b] = p[b * NT];
    for (int z = 1; z < g.split; z += 2) {
        float4 x[2][4];
        const bool two = z + 1 < g.split;
        const float4* p1 = p + slice * (size_t)z;
        const float4* p2 = two ? p1 + slice : p1;
#pragma unroll
        for (int b = 0; b < 4; ++b) { x[0][b] = p1[b * NT]; x[1][b] = p2[b * NT]; }
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            sum[b].x += x[0][b].x; sum[b].y += x[0][b].y; sum[b].z += x[0][b].z; sum[b].w += x[0][b].w;
            if (two) { sum[b].x += x[1][b].x; sum[b].y += x[1][b].y; sum[b].z += x[1][b].z; sum[b].w += x[1][b].w; }
        }
    }
    const int r0 = (wave >> 1) * 16 + 4 * (lane >> 4), c0 = (wave & 1) * 64 + (lane & 15);
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        Cs[r0 * CP + c0 + 16 * b] = sum[b].x;
        Cs[(r0 + 1) * CP + c0 + 16 * b] = sum[b].y;
        Cs[(r0 + 2) * CP + c0 + 16 * b] = sum[b].z;
        Cs[(r0 + 3) * CP + c0 + 16 * b] = sum[b].w;
    }
    __syncthreads();
    const int start = !scatter || j0 == 0 ? 0 : sidx[0];
    const int end = !scatter ? 0 : j0 + BN >= g.J ? g.out_full : clamp_idx(g.keep[j0 + BN], g.out_full);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int row = i0 + 64 * h + 16 * strip;
        if (row < g.I) finish_tile<NT, BN, FINISH_TAB, 4>(g.f, g.out, g.ldo, Cs + 16 * h * CP, CP, row, min(16, g.I - row), j0, cols,
                                                       scatter ? sidx : nullptr, start, end, tab, tid);
    }
}

template <template <int, int> class LA, template <int, int> class LB, int BM, int BN, int WM, int WN>
int launch_inst(const FinishFArgs& a, int i_base, int i_end, int j_base, int j_end, hipStream_t stream)
{
    typedef LA<BM, 64 * WM * WN> A;
    typedef LB<BN, 64 * WM * WN> B;
    constexpr bool ring = A::RING;
    constexpr int list_bytes = [] { if constexpr (ring) return (A::MAPPED || B::MAPPED) ? ring_list_max<BM, BN>() * 4 : 0; else return 0; }();
    constexpr int loop_bytes = fast_smem_bytes<A::WORDS, B::WORDS, BM, BN, ring>() + list_bytes, end_bytes = finish_smem_bytes<BM, BN>();
    constexpr int smem = loop_bytes > end_bytes ? loop_bytes : end_bytes;
    static_assert(smem <= 160 * 1024, "LDS of a workgroup");
    auto fn = act_fast_kernel<LA, LB, BM, BN, WM, WN>;
    static AttrFlags attr_set;      // per instantiation and device
    if (!ensure_max_dynamic_lds((const void*)fn, smem, &attr_set)) return ZR_ERR_HIP;
    if (debug_names_wanted())
        snprintf(g_debug.last_kernel, sizeof(g_debug.last_kernel), "act_fast_kernel<%s, %s, %d, %d, %d, %d>", A::NAME, B::NAME, BM, BN, WM, WN);
    FinishFArgs k = a;
    k.i_base = i_base; k.i_end = i_end; k.j_base = j_base; k.j_end = j_end;
    k.tiles_i = (i_end - i_base + BM - 1) / BM;
    k.tiles_j = (j_end - j_base + BN - 1) / BN;
    const int64_t tiles = (int64_t)k.tiles_i * k.tiles_j;
    if (tiles > 0x7ffffff0) return ZR_ERR_LIMIT;
    k.split = 1; k.kt_per = 0;
    // few tiles and a long contraction: slices of it, as for the products without an end of their own
    if constexpr (!ring && BM == 128 && BN == 128) {
        const int sp = slices_for(a.C, tiles, a.partial, a.partial_bytes, false);
        if (sp >= 2) {
            const int KT = (a.C + BK - 1) / BK;
            k.kt_per = (KT + sp - 1) / sp;
            k.split = (KT + k.kt_per - 1) / k.kt_per;                      // no empty slice
            auto fn1 = act_slice_kernel<LA, LB>;
            static AttrFlags attr1;
            if (!ensure_max_dynamic_lds((const void*)fn1, loop_bytes, &attr1)) return ZR_ERR_HIP;
            hipLaunchKernelGGL(fn1, dim3((unsigned)((tiles * k.split + 7) / 8 * 8)), dim3(256), loop_bytes, stream, (const FArgs&)k);
            if (hipGetLastError() != hipSuccess) return ZR_ERR_HIP;
            hipLaunchKernelGGL(act_reduce_kernel, dim3((unsigned)(tiles * 4)), dim3(256), 0, stream, k);
            if (debug_names_wanted()) snprintf(g_debug.last_kernel, sizeof(g_debug.last_kernel), "act_slice_kernel<%s, %s> split %d", A::NAME, B::NAME, k.split);
            return hip_status(hipGetLastError());
        }
    }
    hipLaunchKernelGGL(fn, dim3((unsigned)((tiles + 7) / 8 * 8)), dim3(64 * WM * WN), smem, stream, k);
    return hip_status(hipGetLastError());
}

// LA, LB: the loaders of the 64-deep loop; the ring's take their place on tiles above 128 x 128 while a list fits LDS
template <template <int, int> class LA, template <int, int> class LB, template <int, int> class RA, template <int, int> class RB, int BM, int BN, int WM, int WN>
int launch_tile(const FinishFArgs& a, int i_base, int i_end, int j_base, int j_end, hipStream_t stream)
{
    if (i_end <= i_base || j_end <= j_base) return ZR_OK;
    if constexpr (BM * BN > 128 * 128) {
        typedef RB<BN, 64 * WM * WN> B;
        if (ring_enabled() && (!B::MAPPED || a.C <= ring_list_max<BM, BN>()))
            return launch_inst<RA, RB, BM, BN, WM, WN>(a, i_base, i_end, j_base, j_end, stream);
    }
    return launch_inst<LA, LB, BM, BN, WM, WN>(a, i_base, i_end, j_base, j_end, stream);
}

// Tile shapes as for the products without an end of their own (see launch_shape in zr_gemm_fast.hip).
template <template <int, int> class LA, template <int, int> class LB, template <int, int> class RA, template <int, int> class RB>
int launch_shape(const FinishFArgs& a, const GemmDesc& d, hipStream_t stream)
{
    constexpr bool rows_of_w = std::is_same<LB<128, 256>, DmaP<128, 256>>::value;
    if (const int f = forced_tiles()) {
        if (f == 2) return launch_tile<LA, LB, RA, RB, 192, 256, 2, 4>(a, 0, a.I, 0, a.J, stream);
        if (f == 3) return launch_tile<LA, LB, RA, RB, 256, 192, 4, 2>(a, 0, a.I, 0, a.J, stream);
        if constexpr (rows_of_w)
            if (f == 5) return launch_tile<LA, LB, RA, RB, 64, 128, 1, 4>(a, 0, a.I, 0, a.J, stream);
        if (f >= 4) return launch_tile<LA, LB, RA, RB, 128, 128, 2, 2>(a, 0, a.I, 0, a.J, stream);
        return launch_tile<LA, LB, RA, RB, 256, 256, 2, 4>(a, 0, a.I, 0, a.J, stream);
    }
    const Sched sc = plan_tiles(a.I, a.J);
    const int64_t tj = tiles_of(a.I, a.J, 256, 192), ti = tiles_of(a.I, a.J, 192, 256);
    const double cj = cost_192(tj), ci = cost_192(ti);
    if (std::min(cj, ci) < sc.cost - 1e-9) {
        if (cj < ci || (cj == ci && tj <= ti)) return launch_tile<LA, LB, RA, RB, 256, 192, 4, 2>(a, 0, a.I, 0, a.J, stream);
        return launch_tile<LA, LB, RA, RB, 192, 256, 2, 4>(a, 0, a.I, 0, a.J, stream);
    }
    if constexpr (rows_of_w) {
        const int64_t t = tiles_of(a.I, a.J, 128, 128);
        if (sc.big_i_end == 0 && (t <= 256 || (t <= 384 && a.C <= 1024)) && slices_for(a.C, t, a.partial, a.partial_bytes, false) < 2)
            return launch_tile<LA, LB, RA, RB, 64, 128, 1, 4>(a, 0, a.I, 0, a.J, stream);
    }
    if (sc.big_i_end == 0) return launch_tile<LA, LB, RA, RB, 128, 128, 2, 2>(a, 0, a.I, 0, a.J, stream);
    const int st = launch_tile<LA, LB, RA, RB, 256, 256, 2, 4>(a, 0, sc.big_i_end, 0, sc.big_j_end, stream);
    if (st != ZR_OK || (sc.big_i_end >= a.I && sc.big_j_end >= a.J)) return st;
    // A few columns behind the panel: 32 x 32 tiles that split each stage over their wavefronts, one to a compute unit, instead of 128 x 128
    // ones in slices (8192 x 4096, 16 columns behind 2048: 27 us in two launches, now 17).
    if (!sc.cut_rows && a.J - sc.big_j_end <= 64) {
        const int rest = launch_act_narrow(d, sc.big_j_end, stream);
        if (rest >= 0) return rest;
    }
    if (sc.cut_rows) return launch_tile<LA, LB, RA, RB, 128, 128, 2, 2>(a, sc.big_i_end, a.I, 0, a.J, stream);
    return launch_tile<LA, LB, RA, RB, 128, 128, 2, 2>(a, 0, a.I, sc.big_j_end, a.J, stream);
}

}  // namespace

// Returns -1 when the problem is not eligible, else a zr_status.
int launch_act_fast(const GemmDesc& d, hipStream_t stream)
{
    if (!gemm_fast_takes(d)) return -1;
    // a list on a contiguous axis is gathered by the kernel for any alignment, and so are contractions of less than three stages
    // that are no whole ones
    if (!d.A.c_contig || d.A.map_contig || d.B.map_contig) return -1;
    if (d.B.c_contig && d.C % BK != 0 && d.C < 3 * BK && !d.A.zero_padded) return -1;
    FinishFArgs a;
    (FArgs&)a = fargs_of(d);
    // (with SiLU and a bias, 1096 to 1336 deep, us in two slices and in one piece: rows of W, 72 tiles 18.4 / 13.1, 144 25 / 16.5 to 21.9, 216 26 to
    // 27.4 / 21.1 to 23.8; all of W, 168 tiles 24.3 / 20 to 23.3, 256 28 / 19.6 to 22.5)
    if (short_for_slices(d)) { a.partial = nullptr; a.partial_bytes = 0; }
    a.f = *d.finish;
    if (d.B.c_contig) return launch_shape<DmaP, DmaP, RingP, RingP>(a, d, stream);
    return d.B.map_strided ? launch_shape<DmaP, DmaQM, RingP, RingQM>(a, d, stream) : launch_shape<DmaP, DmaQ, RingP, RingQ>(a, d, stream);
}

}  // namespace zr
