// A block's output joins the residual stream and the next block's input leaves it (gfx950), forward and backward:
//   t = D(y + bias),  n = post(t),  x_out = x + scale gate n,  h = pre(x_out)
// with post and pre root-mean-square or layer norms over the features of a row.  HBM bound: every tensor once, a row in registers.
//
// NT threads take a row, NV groups of eight columns a thread; rows of up to 512 columns run on one wavefront without a barrier.
// The backward pass normalises again from y and x_out (a few instructions; kept statistics would be read and, of a stored
// x_out, be slightly off), and every thread adds up the gradients of the vectors for its columns over all rows of its workgroup;
// a second launch adds the workgroups' sums in their order and makes the vectors' gradients of them.
// Measured, bf16, as called: 12608 x 1024, layer norm, dropout, bias and gate 22 us (4.7 TB/s); backward, 8192 x 4096, two RMS norms 81 us
// (5.0 TB/s; under a profiler 84 to 89 and 5 for the second launch), two layer norms with every gradient 109.
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
    __device__ __forceinline__ void one(float& a)
    {
        a = wave_sum(a);
        if constexpr (WAVES > 1) {
            const int wave = threadIdx.x >> 6, first = wave / WAVES * WAVES;
            if ((threadIdx.x & 63) == 0) part[place][0][wave] = a;
            __syncthreads();
            a = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) a += part[place][0][first + w];
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

// 0 past the row's end
template <int NV, class C> __device__ __forceinline__ void mask(float (&x)[NV][8], const C& c)
{
    if (!c.edge) return;
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) x[k][e] = e < c.hi[k] ? x[k][e] : 0.f;
}

// v <- (v - mean) r for both of two rows' worth of values (TWO), or the first alone; r for each
template <int NV, bool TWO, class C, class S>
__device__ __forceinline__ void normalise(float (&u)[NV][8], float (&v)[NV][8], float& ru, float& rv, const C& c, int cols,
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
                u[k][e] -= a;
                if constexpr (TWO) v[k][e] -= b;
            }
        mask<NV>(u, c);
        if constexpr (TWO) mask<NV>(v, c);
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
            normalise<NV, false>(t, t, r, unused, c, j.cols, j.layer, j.eps, sums);
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
            normalise<NV, false>(x, x, r, unused, c, j.cols, j.layer, j.eps, sums);
            pre_w.times(x);
            pre_b.plus(x);
            if (on) c.template put<T>(j.h, row * j.ldh, x);
        }
    }
}

// With a = mean(g hat) and b = mean(g) (layer norms; else 0), the gradient at the values of a norm is r (g - b - hat a) =
// r g - (b r) - hat (a r).  a r and b r:
template <int NV, bool LAYER, class S>
__device__ __forceinline__ void norm_back(const float (&g)[NV][8], const float (&hat)[NV][8], float r, int cols, float& ar, float& br, S& sums)
{
    float a = 0.f, b = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            a = fmaf(g[k][e], hat[k][e], a);
            if constexpr (LAYER) b += g[k][e];
        }
    if constexpr (LAYER) sums.two(a, b);
    else sums.one(a);
    ar = a / (float)cols * r;
    br = b / (float)cols * r;
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

// A vector's values, `other` where it is missing
template <typename T, int NV, class C> __device__ __forceinline__ void vector_of(float (&x)[NV][8], const void* p, float other, const C& c)
{
    if (p) {
        Raw8<T> r[NV];
        c.template fetch<T>(r, p, 0);
        c.template values<T>(r, x);
    } else {
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) x[k][e] = other;
    }
}

// wavefronts to a SIMD that the registers have to leave room for
template <typename T, int NT, bool BIASES> constexpr int back_waves()
{
    return NT > 640 ? 4 : NT > 512 ? 3 : NT == 512 || BIASES ? 2 : 3;
}

// With d the gradient at x_out, which is the one at x, and t = D(y + bias) or, behind a post norm, its normalised value:
//   dgate = scale (post_w A + post_b B),  dpost_w = scale gate A,  dpost_b = scale gate B,   A = sum d t,  B = sum d  over the rows,
// and what the post norm passes back is scale times its gradient for d gate post_w: two sums and one product for an element where
// the formulas have three and four.
// BIASES: B, or a gradient of bias or pre_b, is wanted.
template <typename T, int NT, int NV, bool POST, bool PRE, bool LAYER, bool BIASES>
__global__ __launch_bounds__(NT * groups_of<NT>(), (back_waves<T, NT, BIASES>())) void join_back_kernel(const Join j)
{
    constexpr int G = groups_of<NT>(), BLOCK = NT * G;
    __shared__ __align__(16) float part[2][2][BLOCK / 64];
    RowSums<NT, G> sums{part};
    const Columns<NT, NV> c(j.cols, threadIdx.x % NT);
    const int mine = G == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / NT);        // (a row is a wavefront's or more: scalar addresses)
    // vectors in registers for all rows; rows of 1024 threads have no room for them and read them again
    constexpr bool LEAN = NT > 640;
    float bias[LEAN ? 1 : NV][8], gw[LEAN ? 1 : NV][8], pw[LEAN ? 1 : NV][8];
    auto gate_and_weight = [&](float (&x)[NV][8]) {
        vector_of<T, NV>(x, j.gate, 1.f, c);
        if constexpr (POST) {
            if (j.post_w) {
                float w[NV][8];
                vector_of<T, NV>(w, j.post_w, 1.f, c);
#pragma unroll
                for (int k = 0; k < NV; ++k)
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[k][e] *= w[k][e];
            }
        }
    };
    if constexpr (!LEAN) {
        vector_of<T, NV>(bias, j.bias, 0.f, c);
        gate_and_weight(gw);
        if constexpr (PRE) vector_of<T, NV>(pw, j.pre_w, 1.f, c);
    }
    auto times = [&](float (&x)[NV][8], const auto& held, auto read) {
        if constexpr (LEAN) {
            float v[NV][8];
            read(v);
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) x[k][e] *= v[k][e];
        } else {
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) x[k][e] *= held[k][e];
        }
    };
    uint64_t seed = 0, offset = 0;
    if (j.drop) { seed = j.rng[0]; offset = j.rng[1]; }
    // sums over the rows: d t, dh times the pre norm's value; d, dh, dy
    float A[NV][8], P[NV][8], B[NV][8], Q[NV][8], D[NV][8];
    auto zero = [](float (&x)[NV][8]) {
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) x[k][e] = 0.f;
    };
    zero(A); zero(P); zero(B); zero(Q); zero(D);

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
        float t[NV][8], x[NV][8], d[NV][8], g[NV][8], rt = 0.f, rr = 0.f, ar, br;
        c.template values<T>(rd, d);
        if constexpr (PRE) {
            c.template values<T>(rh, g);
            c.template values<T>(rx, x);
        }
        c.template values<T>(ry, t);
        // the next row's values travel while this one's are used (past the last row: the last one's again)
        if constexpr (!LEAN) fetch(base + step);
        if constexpr (G > 1) {
            // (a group of threads behind the last row has that row's values again, and adds nothing: see below)
            if (!on) { zero(d); zero(g); }
        }
        if (j.bias) {
            if constexpr (LEAN) {
                float v[NV][8];
                vector_of<T, NV>(v, j.bias, 0.f, c);
                add<NV>(t, v);
            } else {
                add<NV>(t, bias);
            }
        }
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
        if constexpr (POST && PRE) normalise<NV, true>(x, t, rr, rt, c, j.cols, LAYER, j.eps, sums);
        else if constexpr (PRE) normalise<NV, false>(x, x, rr, rt, c, j.cols, LAYER, j.eps, sums);
        else if constexpr (POST) normalise<NV, false>(t, t, rt, rr, c, j.cols, LAYER, j.eps, sums);
        if constexpr (G > 1) {
            // (its draws are those of a row that there is not: values that the last row drops, whatever they are, may be kept in t, and
            // zeros have no deviation with eps 0; 0 times either is no 0)
            if (!on) {
                zero(t);
                if constexpr (PRE) zero(x);
                rt = rr = 0.f;
            }
        }
        if constexpr (PRE) {
            add_product<NV>(P, g, x);
            if constexpr (BIASES) add<NV>(Q, g);
            times(g, pw, [&](float (&v)[NV][8]) { vector_of<T, NV>(v, j.pre_w, 1.f, c); });
            norm_back<NV, LAYER>(g, x, rr, j.cols, ar, br, sums);
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    d[k][e] = fmaf(-ar, x[k][e], fmaf(rr, g[k][e], d[k][e]));
                    if constexpr (LAYER) d[k][e] -= br;
                }
            if constexpr (LAYER) mask<NV>(d, c);
            if constexpr (G > 1) { if (!on) zero(d); }
        }
        if (j.dx && on) c.template put<T>(j.dx, row * j.lddx, d);
        add_product<NV>(A, d, t);
        if constexpr (BIASES) add<NV>(B, d);
        times(d, gw, gate_and_weight);
        if constexpr (POST) {
            norm_back<NV, LAYER>(d, t, rt, j.cols, ar, br, sums);
            ar *= j.scale; br *= j.scale;
            const float r = rt * j.scale;
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if constexpr (LAYER) d[k][e] = fmaf(-ar, t[k][e], fmaf(r, d[k][e], -br));
                    else d[k][e] = fmaf(-ar, t[k][e], r * d[k][e]);
                }
            if constexpr (LAYER) mask<NV>(d, c);
        } else {
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) d[k][e] *= j.scale;
        }
        if (j.drop) drop(d);
        if constexpr (BIASES) {
            if constexpr (G > 1) { if (!on) zero(d); }          // (0 times a gate or weight that is no number)
            add<NV>(D, d);
        }
        if (j.dy && on) c.template put<T>(j.dy, row * j.lddy, d);
    }

    if (!j.partial) return;
    const int64_t size = (int64_t)j.slabs * j.cols;
    float* dst = j.partial + (int64_t)blockIdx.x * j.cols;
    if constexpr (G == 1) {
        c.template put<float>(dst, SUM_DT * size, A);
        if constexpr (PRE) c.template put<float>(dst, SUM_HAT * size, P);
        if constexpr (BIASES) {
            c.template put<float>(dst, SUM_D * size, B);
            c.template put<float>(dst, SUM_DY * size, D);
            if constexpr (PRE) c.template put<float>(dst, SUM_DH * size, Q);
        }
    } else {
        // the sums of the G rows that a workgroup takes at a time, added up in their order
        static_assert(NV == 1, "a group of eight columns a thread");
        constexpr int COUNT = BIASES ? JOIN_SUMS : 2, WIDTH = NT * 8;
        __shared__ __align__(16) float all[COUNT][BLOCK * 8];
        auto keep = [&](int which, const float (&x)[NV][8]) { store8(all[which] + threadIdx.x * 8, 0, 8, x[0]); };
        keep(SUM_DT, A);
        keep(SUM_HAT, P);
        if constexpr (BIASES) {
            keep(SUM_D, B);
            keep(SUM_DY, D);
            keep(SUM_DH, Q);
        }
        __syncthreads();
        for (int i = threadIdx.x; i < COUNT * (WIDTH / 4); i += BLOCK) {
            const int which = i / (WIDTH / 4), col = i % (WIDTH / 4) * 4;
            f4 v = *(const f4*)(all[which] + col);
#pragma unroll
            for (int q = 1; q < G; ++q) v += *(const f4*)(all[which] + WIDTH * q + col);
            float* p = dst + which * size + col;
            if (col + 4 <= j.cols) {
                *(f4_any*)p = v;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (col + e < j.cols) p[e] = v[e];
            }
        }
    }
}

template <typename T, int NT, int NV, bool BACK>
int launch_shape(const Join& j, int blocks, hipStream_t stream)
{
    constexpr int threads = NT * groups_of<NT>();
    const std::true_type yes;
    const std::false_type no;
    auto both = [&](bool a, bool b, auto f) {
        if (a && b) f(yes, yes);
        else if (a) f(yes, no);
        else if (b) f(no, yes);
        else f(no, no);
    };
    both(j.post, j.pre, [&](auto post, auto pre) {
        constexpr bool POST = decltype(post)::value, PRE = decltype(pre)::value;
        if constexpr (BACK) {
            // (without a norm there is no kind of norm)
            both((POST || PRE) && j.layer, j.biases, [&](auto layer, auto biases) {
                constexpr bool LAYER = decltype(layer)::value && (POST || PRE);
                hipLaunchKernelGGL((join_back_kernel<T, NT, NV, POST, PRE, LAYER, decltype(biases)::value>), dim3((unsigned)blocks), dim3(threads), 0, stream, j);
            });
        } else {
            hipLaunchKernelGGL((join_kernel<T, NT, NV, POST, PRE>), dim3((unsigned)blocks), dim3(threads), 0, stream, j);
        }
    });
    return hip_status(hipGetLastError());
}

// Threads to a row (a group of eight columns each, two in the widest rows), rows that a workgroup takes at a time, and workgroups to a
// compute unit: a launch is that many, each with its share of the rows, and their number is that of the sums to be added up in the
// end.  (Backward, two norms, bf16, us with 1 / 2 / 3 workgroups to a unit: 8192 x 4096 83 / 90 / -, 8192 x 2048 62 / 47 / 50, 12608 x 1024
// 52 / 39 / 40, 8192 x 768 36 / 27 / 24, 8192 x 5120 100 / 112 / -.)
// Above 5120 columns 1024 threads leave 128 registers each, and rows and sums spill in the backward kernels: 8192 x 8192 forward 99 us (5.4 TB/s),
// backward 187 (4.3), with layer norms and every gradient 420 (1.9); 4096 x 16384 115 (4.7), 415 (1.9), 897 (0.9).
struct Shape { int threads, rows_at_once, per_unit; };
Shape shape_of(int cols)
{
    const int nt = cols <= 512 ? 64 : cols <= 1024 ? 128 : cols <= 2048 ? 256 : cols <= 4096 ? 512 : cols <= 5120 ? 640 : 1024;
    return Shape{nt, nt < 256 ? 256 / nt : 1, nt <= 256 ? 4 : nt <= 640 ? 2 : 1};
}
Shape back_shape_of(const Join& j)
{
    Shape s = shape_of(j.cols);
    s.per_unit = s.threads > 256 ? 1 : s.threads == 256 || j.biases ? 2 : 3;
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
        case 512: return launch_shape<T, 512, 1, BACK>(j, blocks, stream);
        case 640: return launch_shape<T, 640, 1, BACK>(j, blocks, stream);
        default: return j.cols <= 8192 ? launch_shape<T, 1024, 1, BACK>(j, blocks, stream) : launch_shape<T, 1024, 2, BACK>(j, blocks, stream);
    }
}

}  // namespace

int join_max_cols() { return MAX_COLS; }

int join_most_slabs(int rows, int cols) { return blocks_of(rows, shape_of(cols)); }
int join_slabs(const Join& j)
{
    // (two turns at least where there are sums: those of a workgroup with one are as much to write and read as its rows; 985 x 1023
    // in fp32, all gradients, with 1 / 2 / 3 / 4: 20.2, 19.7, 22.3, 24.6 us)
    const Shape s = back_shape_of(j);
    const int64_t turns = ((int64_t)j.rows + s.rows_at_once - 1) / s.rows_at_once;
    const int64_t most = std::min<int64_t>(blocks_of(j.rows, s), join_most_slabs(j.rows, j.cols));
    return (int)(j.partial ? std::min(most, (turns + 1) / 2) : most);
}

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
