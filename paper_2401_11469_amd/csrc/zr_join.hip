// A block's output joins the residual stream and the next block's input leaves it (gfx950), forward and backward:
//   t = D(y + bias),  n = post(t),  x_out = x + scale gate n,  h = pre(x_out)
// with post and pre root-mean-square or layer norms over the features of a row.  HBM bound: every tensor once, a row in registers.
//
// NT threads take a row, NV groups of eight columns a thread; rows of up to 512 columns run on one wavefront without a barrier.
// The backward pass normalises again from y and x_out (a few instructions; kept statistics would be read and, of a stored
// x_out, be slightly off), and every thread adds up the gradients of the vectors for its columns over all rows of its workgroup;
// a second launch adds the workgroups' sums in their order.
#include <type_traits>

#include "zr_act.h"

namespace zr {

namespace {

constexpr int MAX_COLS = 16384;

// Sum over a wavefront, for all of its lanes: within rows of 16 lanes, then across the rows (no LDS: a shuffle takes ten times as long).
__device__ __forceinline__ float wave_sum(float v)
{
    auto step = [](float x, auto ctrl) {
        return x + __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(x), decltype(ctrl)::value, 0xf, 0xf, false));
    };
    v = step(v, std::integral_constant<int, 0x111>());      // row_shr 1, 2, 4, 8
    v = step(v, std::integral_constant<int, 0x112>());
    v = step(v, std::integral_constant<int, 0x114>());
    v = step(v, std::integral_constant<int, 0x118>());
    v = step(v, std::integral_constant<int, 0x142>());      // row_bcast 15, 31
    v = step(v, std::integral_constant<int, 0x143>());
    return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), 63));
}

// Sums over the NT threads of a row, for every one of them.  One barrier a call: consecutive calls use two places in turn.
template <int NT, int G> struct RowSums {
    static constexpr int WAVES = NT / 64;
    float (*part)[2][G * WAVES];            // [place][which][wavefront]
    int place = 0;
    __device__ __forceinline__ void two(float& a, float& b)
    {
        a = wave_sum(a);
        b = wave_sum(b);
        if constexpr (WAVES > 1) {
            const int wave = threadIdx.x >> 6, first = wave / WAVES * WAVES;
            if ((threadIdx.x & 63) == 0) { part[place][0][wave] = a; part[place][1][wave] = b; }
            __syncthreads();
            a = b = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) { a += part[place][0][first + w]; b += part[place][1][first + w]; }
            place ^= 1;
        }
    }
};

// rows that a workgroup takes at a time
template <int NT> constexpr int groups_of() { return NT < 256 ? 256 / NT : 1; }

// Where a thread's columns lie: groups of eight at col[k], of which hi[k] are within the row (negative or 0: none).
// Loads are unconditional (a load under a branch is waited for where the branch ends): a group past the end, or that reaches past
// it, is read from the row's last eight columns and moved into place.
template <int NT, int NV> struct Columns {
    int col[NV], hi[NV];
    uint32_t from[NV];
    bool ragged, narrow, edge;         // uniform: the last group is no whole one; rows of less than eight; threads without columns
    __device__ __forceinline__ Columns(int cols, int tid)
    {
        narrow = cols < 8;
        ragged = cols % 8 != 0 && !narrow;
        edge = cols % (8 * NT * NV) != 0;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            col[k] = 8 * (tid + NT * k);
            hi[k] = min(8, cols - col[k]);
            from[k] = (uint32_t)max(0, min(col[k], cols - 8));
        }
    }
    template <typename T> __device__ __forceinline__ void fetch(Raw8<T> (&r)[NV], const void* p, int64_t at) const
    {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if (narrow) {
                float x[8];
                load8((const T*)p + at, 0, max(hi[k], 0), x);
                r[k].take(x);
            } else {
                r[k].load((const T*)p + at + from[k]);
            }
        }
    }
    // the values, 0 past the row's end
    template <typename T> __device__ __forceinline__ void values(const Raw8<T> (&r)[NV], float (&x)[NV][8]) const
    {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            r[k].values(x[k]);
            if (ragged) {
                const int s = col[k] - (int)from[k];
#pragma unroll
                for (int bit = 1; bit < 8; bit *= 2)
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[k][e] = s & bit ? (e + bit < 8 ? x[k][e + bit] : 0.f) : x[k][e];
            }
            if (edge) {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[k][e] = e < hi[k] ? x[k][e] : 0.f;
            }
        }
    }
    template <typename T> __device__ __forceinline__ void put(void* p, int64_t at, const float (&x)[NV][8]) const
    {
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (hi[k] > 0) store8((T*)p + at + (uint32_t)col[k], 0, hi[k], x[k]);
    }
};

// A vector of the row's columns; one that is missing changes nothing.  In registers for all rows, or (LEAN: rows of more columns than
// the registers have room for) read again wherever it is used.
template <typename T, int NT, int NV, bool LEAN> struct Vector {
    Raw8<T> r[LEAN ? 1 : NV];
    const void* p;
    const Columns<NT, NV>& c;
    __device__ __forceinline__ Vector(const void* p_, const Columns<NT, NV>& c_) : p(p_), c(c_)
    {
        if constexpr (!LEAN) {
            if (p) {
                c.template fetch<T>(r, p, 0);
                float x[NV][8];
                c.template values<T>(r, x);
#pragma unroll
                for (int k = 0; k < NV; ++k) r[k].take(x[k]);
            }
        }
    }
    template <class F> __device__ __forceinline__ void with(float (&x)[NV][8], F f) const
    {
        if (!p) return;
        float v[NV][8];
        if constexpr (LEAN) {
            Raw8<T> now[NV];
            c.template fetch<T>(now, p, 0);
            c.template values<T>(now, v);
        } else {
#pragma unroll
            for (int k = 0; k < NV; ++k) r[k].values(v[k]);
        }
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) x[k][e] = f(x[k][e], v[k][e]);
    }
    __device__ __forceinline__ void times(float (&x)[NV][8]) const { with(x, [](float a, float b) { return a * b; }); }
    __device__ __forceinline__ void plus(float (&x)[NV][8]) const { with(x, [](float a, float b) { return a + b; }); }
};

// v <- (v - mean) r for both of two rows' worth of values (TWO), or the first alone; r for each
template <int NV, bool TWO, class S>
__device__ __forceinline__ void normalise(float (&u)[NV][8], float (&v)[NV][8], float& ru, float& rv, const int (&hi)[NV], int cols,
                                          int layer, float eps, S& sums)
{
    const float inv = 1.f / (float)cols;
    if (layer) {
        float a = 0.f, b = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) { a += u[k][e]; if constexpr (TWO) b += v[k][e]; }
        sums.two(a, b);
        a *= inv; b *= inv;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                u[k][e] = e < hi[k] ? u[k][e] - a : 0.f;
                if constexpr (TWO) v[k][e] = e < hi[k] ? v[k][e] - b : 0.f;
            }
    }
    float a = 0.f, b = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            a = fmaf(u[k][e], u[k][e], a);
            if constexpr (TWO) b = fmaf(v[k][e], v[k][e], b);
        }
    sums.two(a, b);
    ru = 1.f / sqrtf(a * inv + eps);
    rv = 1.f / sqrtf(b * inv + eps);
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) { u[k][e] *= ru; if constexpr (TWO) v[k][e] *= rv; }
}

template <typename T, int NT, int NV, bool POST, bool PRE>
__global__ __launch_bounds__(NT * groups_of<NT>(), 4) void join_kernel(const Join j)
{
    constexpr int G = groups_of<NT>();
    __shared__ __align__(16) float part[2][2][NT * G / 64];
    RowSums<NT, G> sums{part};
    const Columns<NT, NV> c(j.cols, threadIdx.x % NT);
    const int mine = G == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / NT);        // (a row is a wavefront's or more: scalar addresses)
    constexpr bool LEAN = NT * NV > 1024;
    typedef Vector<T, NT, NV, LEAN> V;
    const V bias(j.bias, c), gate(j.gate, c), post_w(POST ? j.post_w : nullptr, c), post_b(POST ? j.post_b : nullptr, c);
    const V pre_w(PRE ? j.pre_w : nullptr, c), pre_b(PRE ? j.pre_b : nullptr, c);
    uint64_t seed = 0, offset = 0;
    if (j.drop) { seed = j.rng[0]; offset = j.rng[1]; }
    const int64_t step = (int64_t)gridDim.x * G;
    int64_t base = (int64_t)blockIdx.x * G;
    Raw8<T> ry[NV], rx[NV];
    auto fetch = [&](int64_t from) {
        const int64_t row = min(from + mine, (int64_t)j.rows - 1);
        c.template fetch<T>(ry, j.y, row * j.ldy);
        c.template fetch<T>(rx, j.x, row * j.ldx);
    };
    if constexpr (!LEAN) fetch(base);
    for (; base < j.rows; base += step) {
        if constexpr (LEAN) fetch(base);
        const int64_t row = base + mine;
        const bool on = row < j.rows;
        float t[NV][8], x[NV][8], r, unused;
        c.template values<T>(ry, t);
        c.template values<T>(rx, x);
        // the next row's values travel while this one's are used (past the last row: the last one's again)
        if constexpr (!LEAN) fetch(base + step);
        bias.plus(t);
        if (j.drop) {
#pragma unroll
            for (int k = 0; k < NV; ++k) Draw(seed, offset, (uint32_t)row, (uint32_t)c.col[k] >> 3).apply(t[k], j.drop, j.factor);
        }
        if constexpr (POST) {
            normalise<NV, false>(t, t, r, unused, c.hi, j.cols, j.layer, j.eps, sums);
            post_w.times(t);
            post_b.plus(t);
        }
        gate.times(t);
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) x[k][e] = fmaf(j.scale, t[k][e], x[k][e]);
        if (on) c.template put<T>(j.x_out, row * j.ldxo, x);
        if constexpr (PRE) {
            // (of the sums as they are, before they are rounded into x_out; columns past the end are zeros all the way)
            normalise<NV, false>(x, x, r, unused, c.hi, j.cols, j.layer, j.eps, sums);
            pre_w.times(x);
            pre_b.plus(x);
            if (on) c.template put<T>(j.h, row * j.ldh, x);
        }
    }
}

// The gradient at the values of a norm: g <- r (g - hat mean(g hat) [- mean(g)]); 0 past the row's end, where g and hat are
template <int NV, class S>
__device__ __forceinline__ void norm_back(float (&g)[NV][8], const float (&hat)[NV][8], float r, const int (&hi)[NV], int cols, int layer, S& sums)
{
    float a = 0.f, b = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) { a = fmaf(g[k][e], hat[k][e], a); b += g[k][e]; }
    sums.two(a, b);
    a /= (float)cols;
    b = layer ? b / (float)cols : 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) g[k][e] = e < hi[k] ? r * (g[k][e] - b - hat[k][e] * a) : 0.f;
}

template <int NV> __device__ __forceinline__ void add_product(float (&total)[NV][8], const float (&a)[NV][8], const float (&b)[NV][8])
{
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) total[k][e] = fmaf(a[k][e], b[k][e], total[k][e]);
}
template <int NV> __device__ __forceinline__ void add(float (&total)[NV][8], const float (&a)[NV][8])
{
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) total[k][e] += a[k][e];
}

// wavefronts to a SIMD that the registers have to leave room for
template <typename T, int NT, bool POST, bool PRE, bool BIASES> constexpr int back_waves()
{
    return NT > 640 ? 4 : NT > 512 ? 3 : NT == 512 || BIASES || (POST && PRE && sizeof(T) == 4) ? 2 : 3;
}

// BIASES: gradients of bias, post_b or pre_b are wanted (without them a third of the registers for sums goes, and two rows of up to
// 4096 columns fit a compute unit at a time)
template <typename T, int NT, int NV, bool POST, bool PRE, bool BIASES>
__global__ __launch_bounds__(NT * groups_of<NT>(), (back_waves<T, NT, POST, PRE, BIASES>())) void join_back_kernel(const Join j)
{
    constexpr int G = groups_of<NT>(), BLOCK = NT * G;
    __shared__ __align__(16) float part[2][2][BLOCK / 64];
    RowSums<NT, G> sums{part};
    const Columns<NT, NV> c(j.cols, threadIdx.x % NT);
    const int mine = G == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / NT);        // (a row is a wavefront's or more: scalar addresses)
    constexpr bool LEAN = NT * NV > 640 || (NT == 640 && sizeof(T) == 4);
    typedef Vector<T, NT, NV, LEAN> V;
    const V bias(j.bias, c), gate(j.gate, c), post_w(POST ? j.post_w : nullptr, c), post_b(POST ? j.post_b : nullptr, c);
    const V pre_w(PRE ? j.pre_w : nullptr, c);
    uint64_t seed = 0, offset = 0;
    if (j.drop) { seed = j.rng[0]; offset = j.rng[1]; }
    // gradients of the vectors, where their sums lie in j.partial: bias, gate, weight and bias of the post norm, of the pre norm
    // (IN_LDS: those of the biases of wide rows lie in LDS, four columns of every thread side by side)
    constexpr bool IN_LDS = BIASES && NT > 512 && NV == 1;
    extern __shared__ __align__(16) float biases[];
    auto add_bias = [&](int s, float (&sum)[NV][8], const float (&v)[NV][8]) {
        if constexpr (!IN_LDS) {
            add<NV>(sum, v);
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                f4* at = (f4*)(biases + ((s * 2 + h) * NT + threadIdx.x) * 4);
                f4 old = *at;
#pragma unroll
                for (int e = 0; e < 4; ++e) old[e] += v[0][4 * h + e];
                *at = old;
            }
        }
    };
    if constexpr (IN_LDS) {
#pragma unroll
        for (int q = 0; q < 6; ++q) *(f4*)(biases + (q * NT + threadIdx.x) * 4) = f4{0.f, 0.f, 0.f, 0.f};
    }
    float total[6][NV][8];
#pragma unroll
    for (int s = 0; s < 6; ++s)
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) total[s][k][e] = 0.f;

    const int64_t step = (int64_t)gridDim.x * G;
    int64_t base = (int64_t)blockIdx.x * G;
    Raw8<T> rd[NV], rh[NV], rx[NV], ry[NV];
    auto fetch = [&](int64_t from) {
        const int64_t row = min(from + mine, (int64_t)j.rows - 1);
        if (j.dx_out) c.template fetch<T>(rd, j.dx_out, row * j.lddxo);
        if constexpr (PRE) {
            c.template fetch<T>(rh, j.dh, row * j.lddh);
            c.template fetch<T>(rx, j.x, row * j.ldx);
        }
        if (j.y) c.template fetch<T>(ry, j.y, row * j.ldy);
    };
#pragma unroll
    for (int k = 0; k < NV; ++k) { rd[k].clear(); ry[k].clear(); }
    if constexpr (!LEAN) fetch(base);
    for (; base < j.rows; base += step) {
        if constexpr (LEAN) fetch(base);
        const int64_t row = base + mine;
        const bool on = row < j.rows;
        float t[NV][8], x[NV][8], d[NV][8], g[NV][8], rt = 0.f, rr = 0.f;
        c.template values<T>(rd, d);
        if constexpr (PRE) {
            c.template values<T>(rh, g);
            c.template values<T>(rx, x);
        }
        c.template values<T>(ry, t);
        if constexpr (!LEAN) fetch(base + step);
        if constexpr (G > 1) {
            // (a group of threads behind the last row has that row's values again, and adds nothing)
            if (!on) {
#pragma unroll
                for (int k = 0; k < NV; ++k)
#pragma unroll
                    for (int e = 0; e < 8; ++e) { d[k][e] = 0.f; g[k][e] = 0.f; }
            }
        }
        bias.plus(t);
        uint32_t kept[NV];
        auto drop = [&](float (&v)[NV][8]) {
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[k][e] = kept[k] >> e & 1 ? v[k][e] * j.factor : 0.f;
        };
        if (j.drop) {
#pragma unroll
            for (int k = 0; k < NV; ++k) kept[k] = Draw(seed, offset, (uint32_t)row, (uint32_t)c.col[k] >> 3).bits(j.drop);
            drop(t);
        }
        if constexpr (POST && PRE) normalise<NV, true>(x, t, rr, rt, c.hi, j.cols, j.layer, j.eps, sums);
        else if constexpr (PRE) normalise<NV, false>(x, x, rr, rt, c.hi, j.cols, j.layer, j.eps, sums);
        else if constexpr (POST) normalise<NV, false>(t, t, rt, rr, c.hi, j.cols, j.layer, j.eps, sums);
        if constexpr (PRE) {
            add_product<NV>(total[4], g, x);
            if constexpr (BIASES) add_bias(2, total[5], g);
            pre_w.times(g);
            norm_back<NV>(g, x, rr, c.hi, j.cols, j.layer, sums);
            add<NV>(d, g);
        }
        // d: the gradient at x_out and at x; t: D(y + bias), or what the post norm makes of it before its weight
        if (j.dx && on) c.template put<T>(j.dx, row * j.lddx, d);
        float n[NV][8];
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) { d[k][e] *= j.scale; n[k][e] = t[k][e]; }
        if constexpr (POST) {
            post_w.times(n);
            post_b.plus(n);
        }
        add_product<NV>(total[1], d, n);
        gate.times(d);
        if constexpr (POST) {
            add_product<NV>(total[2], d, t);
            if constexpr (BIASES) add_bias(1, total[3], d);
            post_w.times(d);
            norm_back<NV>(d, t, rt, c.hi, j.cols, j.layer, sums);
        }
        if (j.drop) drop(d);
        if constexpr (BIASES) add_bias(0, total[0], d);
        if (j.dy && on) c.template put<T>(j.dy, row * j.lddy, d);
    }

    if (!j.partial) return;
    if constexpr (IN_LDS) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                total[0][0][4 * h + e] = biases[(h * NT + threadIdx.x) * 4 + e];
                total[3][0][4 * h + e] = biases[((2 + h) * NT + threadIdx.x) * 4 + e];
                total[5][0][4 * h + e] = biases[((4 + h) * NT + threadIdx.x) * 4 + e];
            }
    }
    // the G rows' sums of a workgroup, in their order
    __shared__ __align__(16) float all[G > 1 ? BLOCK * 8 : 4];
#pragma unroll
    for (int s = 0; s < 6; ++s) {
        if constexpr (!BIASES) { if (s == 0 || s == 3 || s == 5) continue; }
        if ((s == 2 || s == 3) && !POST) continue;
        if (s >= 4 && !PRE) continue;
        float* dst = j.partial + ((size_t)s * (size_t)j.slabs + blockIdx.x) * (size_t)j.cols;
        if constexpr (G > 1) {
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                __syncthreads();
                store8(all + threadIdx.x * 8, 0, 8, total[s][k]);
                __syncthreads();
                if (threadIdx.x < NT)
#pragma unroll
                    for (int q = 1; q < G; ++q)
#pragma unroll
                        for (int e = 0; e < 8; ++e) total[s][k][e] += all[(threadIdx.x + NT * q) * 8 + e];
            }
            if (threadIdx.x >= NT) continue;
        }
        c.template put<float>(dst, 0, total[s]);
    }
}

template <typename T, int NT, int NV, bool BACK>
int launch_shape(const Join& j, int blocks, hipStream_t stream)
{
    constexpr int threads = NT * groups_of<NT>();
    bool ok = true;
    auto go = [&](auto post, auto pre, auto biases) {
        constexpr bool POST = decltype(post)::value, PRE = decltype(pre)::value, BIASES = decltype(biases)::value;
        if constexpr (BACK) {
            constexpr int lds = BIASES && NT > 512 && NV == 1 ? 6 * NT * 16 : 0;
            const auto fn = join_back_kernel<T, NT, NV, POST, PRE, BIASES>;
            if constexpr (lds > 0) {
                static AttrFlags attr_set;
                if (!ensure_max_dynamic_lds((const void*)fn, lds, &attr_set)) { ok = false; return; }
            }
            hipLaunchKernelGGL(fn, dim3((unsigned)blocks), dim3(threads), lds, stream, j);
        }
        else hipLaunchKernelGGL((join_kernel<T, NT, NV, POST, PRE>), dim3((unsigned)blocks), dim3(threads), 0, stream, j);
    };
    const std::true_type yes;
    const std::false_type no;
    auto norms = [&](auto biases) {
        if (j.post && j.pre) go(yes, yes, biases);
        else if (j.post) go(yes, no, biases);
        else if (j.pre) go(no, yes, biases);
        else go(no, no, biases);
    };
    if constexpr (!BACK) norms(no);
    else if constexpr (NT * NV == 1024) { if (j.biases == (NT == 512)) norms(std::integral_constant<bool, NT == 512>()); else return ZR_ERR_SHAPE; }
    else if (j.biases) norms(yes);
    else norms(no);
    if (!ok) return ZR_ERR_HIP;
    return hip_status(hipGetLastError());
}

// Threads to a row (a group of eight columns each, two in the widest rows), rows that a workgroup takes at a time, and workgroups to a
// compute unit, which is how many of them its registers hold: a launch is that many, each with its share of the rows.  (Backward, 8192 x 4096, two norms, us by wavefronts to a unit: 8
// 98, 12 127, 16 105, 24 112; 12608 x 1024: 43, 42, 50, 48.)
struct Shape { int threads, rows_at_once, per_unit; };
Shape shape_of(int cols)
{
    const int nt = cols <= 512 ? 64 : cols <= 1024 ? 128 : cols <= 2048 ? 256 : cols <= 4096 ? 512 : cols <= 5120 ? 640 : 1024;
    return Shape{nt, nt < 256 ? 256 / nt : 1, nt <= 256 ? 4 : nt <= 640 ? 2 : 1};
}
Shape back_shape_of(const Join& j)
{
    Shape s = shape_of(j.cols);
    if (s.threads <= 256) s.per_unit = j.biases ? 2 : 3;
    else if (s.threads == 512) s.per_unit = j.biases || (j.post && j.pre) ? 1 : 2;
    else s.per_unit = 1;
    // six vectors' sums: two groups of columns to a thread of twice the registers (4096 x 8192, layer norms, dropout, all gradients:
    // 171 us, 204 on 1024 threads with three of the sums in LDS; 8192 x 5120 on 640 threads 288 and 218)
    if (j.biases && j.cols > 5120 && j.cols <= 8192) s.threads = 512;
    return s;
}
int blocks_of(int rows, const Shape& s)
{
    return (int)std::min<int64_t>(((int64_t)rows + s.rows_at_once - 1) / s.rows_at_once, 256 * s.per_unit);
}

template <bool BACK, typename T>
int launch_any(const Join& j, const Shape& s, int blocks, hipStream_t stream)
{
    switch (s.threads) {
        case 64: return launch_shape<T, 64, 1, BACK>(j, blocks, stream);
        case 128: return launch_shape<T, 128, 1, BACK>(j, blocks, stream);
        case 256: return launch_shape<T, 256, 1, BACK>(j, blocks, stream);
        case 512:
            if constexpr (BACK)
                if (j.cols > 4096) return launch_shape<T, 512, 2, true>(j, blocks, stream);
            return launch_shape<T, 512, 1, BACK>(j, blocks, stream);
        case 640: return launch_shape<T, 640, 1, BACK>(j, blocks, stream);
        default: return j.cols <= 8192 ? launch_shape<T, 1024, 1, BACK>(j, blocks, stream) : launch_shape<T, 1024, 2, BACK>(j, blocks, stream);
    }
}

}  // namespace

int join_max_cols() { return MAX_COLS; }

int join_most_slabs(int rows, int cols) { return blocks_of(rows, shape_of(cols)); }
int join_slabs(const Join& j) { return blocks_of(j.rows, back_shape_of(j)); }

int launch_join(const Join& j, int dtype, hipStream_t stream)
{
    const Shape s = shape_of(j.cols);
    const int blocks = blocks_of(j.rows, s);
    return dtype == ZR_BF16 ? launch_any<false, Bf>(j, s, blocks, stream) : launch_any<false, float>(j, s, blocks, stream);
}

int launch_join_back(const Join& j, int dtype, hipStream_t stream)
{
    const Shape s = back_shape_of(j);
    return dtype == ZR_BF16 ? launch_any<true, Bf>(j, s, j.slabs, stream) : launch_any<true, float>(j, s, j.slabs, stream);
}

}  // namespace zr
