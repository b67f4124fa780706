// Launches of the bf16 products of any alignment (the kernel stands in zr_gemm_any.h): tile shapes and loaders, dX and dW in one
// launch, and the choice between the paths.
#include "zr_gemm_any.h"

namespace zr {

namespace {

// A pair of loaders, as a type.
template <template <int, int, bool> class LA, bool AP, template <int, int, bool> class LB, bool BP> struct Loaders {
    template <int R> static __device__ __forceinline__ void run(const Args& g, uint32_t* smem, int lin)
    {
        gemm_body<LA, AP, LB, BP, R, 256, true>(g, smem, lin);
    }
};

// dX and dW of one backward call: the first per_w workgroups of every XCD are dW's, or with x_first the last ones.
template <class X, int XR, class W, int WR>
__global__ __launch_bounds__(256, 2) void gemm_pair_kernel(const Args gx, const Args gw, const int per_x, const int per_w, const int x_first)
{
    extern __shared__ __align__(16) uint32_t smem[];
    const int xcd = blockIdx.x % 8, q = blockIdx.x / 8;
    const int qx = x_first ? q : q - per_w, qw = x_first ? q - per_x : q;
    if (qw >= 0 && qw < per_w) W::template run<WR>(gw, smem, xcd * per_w + qw);
    else X::template run<XR>(gx, smem, xcd * per_x + qx);
}

// ---------------------------------------------------------------------------
// dX and dW in one launch
// ---------------------------------------------------------------------------
// The order in which a product is added up stays the one it has on its own (see adds_in_groups): 32 x 32
// tiles below 96 of 64 x 64, 64 x 64 ones with alternating sums where those of 512 threads would be used, and
// else 64 x 64 or 128 x 128, whichever the model of the schedule finds shorter (every XCD takes its tiles in
// order, each as soon as one of 64 halves of a unit is free; a tile takes a start and an end, and a time per
// stage, longer where kept columns are gathered).  Fitted to 16170 backward calls (32 to 16384 tokens, 64 to 5121
// wide), each in all forms and in two launches, for the time of what they pick: 0.766 of that of two launches on average (the
// best form of each would be 0.760), 90 of them more than 8 % slower than two launches.  Each of the 56 forms (seven pairs of tiles for eight
// of loaders) is picked, for 11 to 981 of the calls, and takes 0.69 to 0.90 of the time in two launches there.  us before, in two launches, and now: 985 x 1001 x 771
// 34 -> 25, 489 x 953 x 1073 30 -> 19, 2024 x 1024 x 1024 40 -> 30, 4095 x 2960 x 2304 64 for 130.
struct Plan { int xr, wr; bool x_first; };
struct Cost { double start, stage; };
constexpr Cost kCost32 = {6.0, 0.45}, kCost64 = {7.0, 1.17}, kCost128 = {11.0, 1.09};     // us, us per stage of 128, 128 and 64
constexpr double kGathered = 0.59, kHalfFree = 0.80, kPair = 2.0, kAlone = 1.0;           // per gathered operand; a unit to itself; a launch
constexpr double kWide = 0.80, kWideGathered = 0.84;                                      // the same for 512 threads on 64 x 64
constexpr double kLimit = 1.07;                                                           // two launches take this much more than the model of each says

int64_t tiles_of(const Args& a, int r) { return (int64_t)((a.I + r - 1) / r) * ((a.J + r - 1) / r); }

int tile_of(const Args& a, bool wide) { return tiles_of(a, 64) < 96 ? 32 : wide && !adds_in_groups(a.I, a.J, a.C) ? 128 : 64; }

double tile_us(const Args& a, int r, double f, double gathered = kGathered)
{
    const Cost c = r == 32 ? kCost32 : r == 64 ? kCost64 : kCost128;
    const int bk = r == 128 ? 64 : 128;
    return c.start + f * c.stage * ((a.C + bk - 1) / bk) * (1 + gathered * ((a.A.map_c != nullptr) + (a.B.map_c != nullptr)));
}

// Which tiles start first: dX's where they take clearly longer than dW's, gathers apart (those weigh less beside the other product's
// tiles than on their own).  43903 backward calls in both orders: 1.0073 of the better one on average, 1.0117 by the times with
// gathers, 1.032 with dW first always (2024 x 1024 x 1024 of 768 kept columns, [K x N], dX on 128 x 128 beside dW on 64 x 64: dW
// first 57.8 us, dX first 61.4; dX on 64 x 64 beside dW on 32 x 32, 2024 x 256 x 1024 of 192 kept rows: 33.2 and 31.0).
constexpr double kClearlyLonger = 1.15;
bool x_starts(const Args& x, int xr, const Args& w, int wr) { return tile_us(x, xr, 1.0, 0.0) > kClearlyLonger * tile_us(w, wr, 1.0, 0.0); }

double alone_us(const Args& a)
{
    double best = 1e30;
    for (bool wide : {false, true}) {
        const int r = tile_of(a, wide);
        const int64_t n = (tiles_of(a, r) + 7) / 8;
        const int g = (a.A.map_c != nullptr) + (a.B.map_c != nullptr);
        double f = n <= 32 ? kHalfFree : 1.0;
        if (r == 64 && adds_in_groups(a.I, a.J, a.C)) f *= kWide * (1 + kWideGathered * g) / (1 + kGathered * g);
        best = std::min(best, (double)((n + 63) / 64) * tile_us(a, r, f));
    }
    return best + kAlone;
}

// false: two launches (limit: what those take, on whichever kernels)
bool plan_pair(const Args& x, const Args& w, double limit, Plan& p)
{
    double best = limit;
    bool found = false;
    for (bool xwide : {false, true})
        for (bool wwide : {false, true}) {
            const int xr = tile_of(x, xwide), wr = tile_of(w, wwide);
            if (xr + wr == 160) continue;                   // (no kernel of 32 x 32 beside 128 x 128)
            const int64_t nx = (tiles_of(x, xr) + 7) / 8, nw = (tiles_of(w, wr) + 7) / 8;
            if (nx + nw > 1 << 20) continue;
            const double f = nx + nw <= 32 ? kHalfFree : 1.0, tx = tile_us(x, xr, f), tw = tile_us(w, wr, f);
            const double us = kPair + (tx > tw ? two_groups((int)nx, tx, (int)nw, tw, 64) : two_groups((int)nw, tw, (int)nx, tx, 64));
            if (us < best) { best = us; p = Plan{xr, wr, x_starts(x, xr, w, wr)}; found = true; }
        }
    return found;
}

template <class X, int XR, class W, int WR>
int launch_pair_inst(const Args& x, const Args& w, const char* name, bool x_first, hipStream_t stream)
{
    constexpr int words = Geo<XR, 256>::WORDS > Geo<WR, 256>::WORDS ? Geo<XR, 256>::WORDS : Geo<WR, 256>::WORDS;
    constexpr int smem = 2 * 2 * words * 4;
    auto fn = gemm_pair_kernel<X, XR, W, WR>;
    static AttrFlags attr_set;      // per instantiation and device
    if (!ensure_max_dynamic_lds((const void*)fn, smem, &attr_set)) return ZR_ERR_HIP;
    if (debug_names_wanted())
        snprintf(g_debug.last_kernel, sizeof(g_debug.last_kernel), "gemm_kernel<%s> beside each other, %d and %d", name, WR, XR);
    Args kx = x, kw = w;
    kx.tiles_i = (x.I + XR - 1) / XR; kx.tiles_j = (x.J + XR - 1) / XR;
    kw.tiles_i = (w.I + WR - 1) / WR; kw.tiles_j = (w.J + WR - 1) / WR;
    const int64_t px = ((int64_t)kx.tiles_i * kx.tiles_j + 7) / 8, pw = ((int64_t)kw.tiles_i * kw.tiles_j + 7) / 8;
    hipLaunchKernelGGL(fn, dim3((unsigned)(px + pw) * 8), dim3(256), smem, stream, kx, kw, (int)px, (int)pw, x_first ? 1 : 0);
    return hip_status(hipGetLastError());
}

template <class X, class W>
int launch_pair(const Args& x, const Args& w, const char* name, const Plan& p, hipStream_t stream)
{
    if (p.xr == 128 && p.wr == 128) return launch_pair_inst<X, 128, W, 128>(x, w, name, p.x_first, stream);
    if (p.xr == 128) return launch_pair_inst<X, 128, W, 64>(x, w, name, p.x_first, stream);
    if (p.wr == 128) return launch_pair_inst<X, 64, W, 128>(x, w, name, p.x_first, stream);
    if (p.xr == 64 && p.wr == 64) return launch_pair_inst<X, 64, W, 64>(x, w, name, p.x_first, stream);
    if (p.xr == 64) return launch_pair_inst<X, 64, W, 32>(x, w, name, p.x_first, stream);
    if (p.wr == 64) return launch_pair_inst<X, 32, W, 64>(x, w, name, p.x_first, stream);
    return launch_pair_inst<X, 32, W, 32>(x, w, name, p.x_first, stream);
}

int launch_gemm_any_pair(const GemmDesc& dx, const GemmDesc& dw, hipStream_t stream)
{
    if (forced_tiles() || !ring_enabled() || dx.I < 1 || dx.J < 1 || dx.C < 1 || dw.I < 1 || dw.J < 1 || dw.C < 1) return -1;
    for (const GemmDesc* d : {&dx, &dw})
        if (too_short(*d, d->A) || too_short(*d, d->B)) return -1;
    if (!dx.A.c_contig || dw.A.c_contig || dw.B.c_contig) return -1;
    Args x = args_of(dx), w = args_of(dw);
    Plan p;
    // a large dW with a gather in flight has its own kernel (4096 x 2752 x 4096 of 2064 kept rows 247 us in two launches, 262
    // in one; 2048 x 4096 x 4096, stored [N x K], 206 / 268; up to 256 tiles: 4096 x 2048 x 2048 of 1024 kept columns 251 / 121)
    const bool w_fast = gemm_fast_takes(dw);
    if (w_fast && tiles_of(w, 128) > 256) return -1;
    const bool x_fast = gemm_fast_takes(dx);
    double limit = kLimit * ((x_fast ? gemm_fast_us(dx) : alone_us(x)) + (w_fast ? gemm_fast_us(dw) : alone_us(w)));
    // A clearer gain where the models are the less certain: kept columns of a large [N x K] shard in both products (4832 x 2184 x 2840 of
    // 1249 193 us, 278 in one launch), and long contractions on 512 threads a tile.
    if (x_fast && w_fast && x.B.map_c && w.B.map_c && !dx.B.c_contig) limit *= 0.70;
    auto long_wide = [](const Args& a) { return a.C > 4096 && tiles_of(a, 64) >= 96 && adds_in_groups(a.I, a.J, a.C); };
    if (long_wide(x) || long_wide(w)) limit *= 0.95;
    if (!plan_pair(x, w, limit, p)) return -1;
    x.alternate = p.xr == 64 && adds_in_groups(x.I, x.J, x.C);
    w.alternate = p.wr == 64 && adds_in_groups(w.I, w.J, w.C);
    const bool xa = dx.A.map_contig, xb = dx.B.map_contig, wa = dw.A.map_contig, wb = dw.B.map_contig;
    typedef Loaders<Plain, false, Plain, false> WPlain;
    typedef Loaders<Gather, false, Plain, false> WGatherA;
    typedef Loaders<Plain, false, Gather, false> WGatherB;
    if (dx.B.c_contig) {                    // weight stored [K x N]
        if (xa && xb && !wa && wb) return launch_pair<Loaders<Gather, true, Gather, true>, WGatherB>(x, w, "Pg, Pg; Q, Qg", p, stream);
        if (xa || wb) return -1;
        if (xb) return wa ? -1 : launch_pair<Loaders<Plain, true, Gather, true>, WPlain>(x, w, "P, Pg; Q, Q", p, stream);
        if (wa) return launch_pair<Loaders<Plain, true, Plain, true>, WGatherA>(x, w, "P, P; Qg, Q", p, stream);
        return launch_pair<Loaders<Plain, true, Plain, true>, WPlain>(x, w, "P, P; Q, Q", p, stream);
    }
    if (xa && !xb && wa && !wb) return launch_pair<Loaders<Gather, true, Plain, false>, WGatherA>(x, w, "Pg, Q; Qg, Q", p, stream);
    if (xa || wa) return -1;
    if (xb && wb) return launch_pair<Loaders<Plain, true, Gather, false>, WGatherB>(x, w, "P, Qg; Q, Qg", p, stream);
    if (wb) return -1;
    if (xb) return launch_pair<Loaders<Plain, true, Gather, false>, WPlain>(x, w, "P, Qg; Q, Q", p, stream);
    return launch_pair<Loaders<Plain, true, Plain, false>, WPlain>(x, w, "P, Q; Q, Q", p, stream);
}

int launch_gemm_any(const GemmDesc& d, hipStream_t stream)
{
    if (d.I < 1 || d.J < 1 || d.C < 1) return ZR_ERR_SHAPE;
    const Args a = args_of(d);
    const bool ag = d.A.map_contig != nullptr, bg = d.B.map_contig != nullptr;
    const bool ap = d.A.c_contig, bp = d.B.c_contig;
    if (!ap && bp) return ZR_ERR_MODE;
    if (too_short(d, d.A) || too_short(d, d.B)) {
        if (ap) return bp ? launch_short<Any, true, Any, true>(a, "Pe, Pe", stream) : launch_short<Any, true, Any, false>(a, "Pe, Qe", stream);
        return launch_short<Any, false, Any, false>(a, "Qe, Qe", stream);
    }
    if (ap && !bp) {            // forward, weight stored [K x N]; dX, weight stored [N x K]
        if (ag) return bg ? ZR_ERR_MODE : launch_shape<Gather, true, Plain, false>(a, "Pg, Q", stream);
        return bg ? launch_shape<Plain, true, Gather, false>(a, "P, Qg", stream) : launch_shape<Plain, true, Plain, false>(a, "P, Q", stream);
    }
    if (ap && bp) {
        if (ag) return bg ? launch_shape<Gather, true, Gather, true>(a, "Pg, Pg", stream) : ZR_ERR_MODE;
        return bg ? launch_shape<Plain, true, Gather, true>(a, "P, Pg", stream) : launch_shape<Plain, true, Plain, true>(a, "P, P", stream);
    }
    // dW
    if (ag) return bg ? ZR_ERR_MODE : launch_shape<Gather, false, Plain, false>(a, "Qg, Q", stream);
    return bg ? launch_shape<Plain, false, Gather, false>(a, "Q, Qg", stream) : launch_shape<Plain, false, Plain, false>(a, "Q, Q", stream);
}

}  // namespace

thread_local DebugState g_debug;

bool ensure_max_dynamic_lds(const void* fn, int bytes, void* flags16)
{
    AttrFlags* f = (AttrFlags*)flags16;
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess) return false;
    if (dev < 0 || dev >= AttrFlags::MAX_DEVICES) {      // beyond the table: set it every time
        return hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) == hipSuccess;
    }
    if (f->done[dev].load(std::memory_order_acquire)) return true;
    if (hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) != hipSuccess) return false;
    f->done[dev].store(true, std::memory_order_release);
    return true;
}

static int launch_gemm_untimed(const GemmDesc& d, hipStream_t stream)
{
    if (d.finish) {
        int st = launch_act_few(d, stream);
        if (st < 0) st = launch_act_fast(d, stream);
        if (st >= 0) return st;
        return d.dtype == ZR_BF16 ? launch_act_any(d, stream) : d.dtype == ZR_F32 ? launch_act_f32(d, stream) : ZR_ERR_DTYPE;
    }
    const int fast = launch_gemm_fast(d, stream);   // bf16, 16-byte aligned rows
    if (fast >= 0) return fast;
    if (d.dtype == ZR_BF16) return launch_gemm_any(d, stream);
    if (d.dtype == ZR_F32) return launch_gemm_f32(d, stream);
    return ZR_ERR_DTYPE;
}

int launch_gemm(const GemmDesc& desc, hipStream_t stream)
{
    GemmDesc d = desc;
    if (d.with) {
        // (the measuring aid times products one by one)
        int st = -1;
        if (!g_debug.armed_once) {
            if (d.dtype == ZR_F32) st = launch_gemm_f32_pair(*d.with, d, stream);
            else if (d.dtype == ZR_BF16) {
                st = launch_gemm_pair(*d.with, d, stream);
                if (st < 0) st = launch_gemm_any_pair(*d.with, d, stream);
            }
        }
        if (st >= 0 || d.only_together) return st;
        st = launch_gemm(*d.with, stream);
        if (st != ZR_OK) return st;
        d.with = nullptr;
    }
    if (d.avg_partial) {
        const bool leaves = gemm_leaves_sums(d);
        if (d.sums_left) *d.sums_left = leaves;
        if (leaves) {
            const int extent = d.epilogue == EPI_COL_SCATTER ? d.J : d.I;
            const int st = launch_zero_f32(d.avg_partial, (size_t)((extent + 127) / 128) * (size_t)d.avg_len, stream);
            if (st != ZR_OK) return st;
        } else {
            d.avg_partial = nullptr;
        }
    }
    if (!g_debug.armed_once) return launch_gemm_untimed(d, stream);
    // measuring aid (zr_debug_time_next_product): events right around this product's own
    // launch(es), without a preceding extraction or a following imputation pass.  One shot.
    hipEvent_t e0 = g_debug.start, e1 = g_debug.stop;
    if (hipEventRecord(e0, stream) != hipSuccess) { g_debug.armed_once = false; return ZR_ERR_HIP; }
    const int st = launch_gemm_untimed(d, stream);
    g_debug.armed_once = false;
    g_debug.start = g_debug.stop = nullptr;
    if (hipEventRecord(e1, stream) != hipSuccess) return ZR_ERR_HIP;
    return st;
}

}  // namespace zr
