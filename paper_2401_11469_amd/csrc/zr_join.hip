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

// Sums over the NT threads of a row, for every one of them.  One barrier a call: consecutive calls use two places in turn.
template <int NT, int G> struct RowSums {
    static constexpr int WAVES = NT / 64;
    float (*part)[2][G * WAVES];            // [place][which][wavefront]
    int place = 0;
    __device__ __forceinline__ void two(float& a, float& b)
    {
#pragma unroll
        for (int off = 32; off; off >>= 1) {
            a += __shfl_xor(a, off, 64);
            b += __shfl_xor(b, off, 64);
        }
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

template <int NT> constexpr int groups_of() { return NT < 256 ? 256 / NT : 1; }

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

// x <- x * v[col ..] (add: + v), with a vector that may be missing
template <typename T> __device__ __forceinline__ void times(float (&x)[8], const void* v, int col, int hi)
{
    if (!v || hi <= 0) return;
    float w[8];
    load8((const T*)v + col, 0, hi, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= w[e];
}
template <typename T> __device__ __forceinline__ void plus(float (&x)[8], const void* v, int col, int hi)
{
    if (!v || hi <= 0) return;
    float w[8];
    load8((const T*)v + col, 0, hi, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] += w[e];
}
template <typename T> __device__ __forceinline__ void row8(const void* p, int64_t ld, int64_t row, int col, int hi, float (&x)[8])
{
    if (p && hi > 0) load8((const T*)p + row * ld + col, 0, hi, x);
    else
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = 0.f;
}

template <typename T, int NT, int NV, bool POST, bool PRE>
__global__ __launch_bounds__(NT * groups_of<NT>()) void join_kernel(const Join j)
{
    constexpr int G = groups_of<NT>();
    __shared__ float part[2][2][NT * G / 64];
    RowSums<NT, G> sums{part};
    const int tid = threadIdx.x % NT;
    int col[NV], hi[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) { col[k] = 8 * (tid + NT * k); hi[k] = min(8, j.cols - col[k]); }
    uint64_t seed = 0, offset = 0;
    if (j.drop) { seed = j.rng[0]; offset = j.rng[1]; }
    for (int64_t base = (int64_t)blockIdx.x * G; base < j.rows; base += (int64_t)gridDim.x * G) {
        const int64_t row = base + threadIdx.x / NT;
        const bool on = row < j.rows;
        float t[NV][8], x[NV][8], r, unused;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int h = on ? hi[k] : 0;
            row8<T>(j.y, j.ldy, row, col[k], h, t[k]);
            row8<T>(j.x, j.ldx, row, col[k], h, x[k]);
            plus<T>(t[k], j.bias, col[k], h);
            if (j.drop) Draw(seed, offset, (uint32_t)row, (uint32_t)col[k] >> 3).apply(t[k], j.drop, j.factor);
        }
        if constexpr (POST) {
            normalise<NV, false>(t, t, r, unused, hi, j.cols, j.layer, j.eps, sums);
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                times<T>(t[k], j.post_w, col[k], hi[k]);
                plus<T>(t[k], j.post_b, col[k], hi[k]);
            }
        }
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            times<T>(t[k], j.gate, col[k], hi[k]);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[k][e] = fmaf(j.scale, t[k][e], x[k][e]);
            if (on && hi[k] > 0) store8((T*)j.x_out + row * j.ldxo + col[k], 0, hi[k], x[k]);
        }
        if constexpr (PRE) {
            // (of the sums as they are, before they are rounded into x_out; columns past the end are zeros all the way)
            normalise<NV, false>(x, x, r, unused, hi, j.cols, j.layer, j.eps, sums);
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                times<T>(x[k], j.pre_w, col[k], hi[k]);
                plus<T>(x[k], j.pre_b, col[k], hi[k]);
                if (on && hi[k] > 0) store8((T*)j.h + row * j.ldh + col[k], 0, hi[k], x[k]);
            }
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

template <typename T, int NT, int NV, bool POST, bool PRE>
__global__ __launch_bounds__(NT * groups_of<NT>()) void join_back_kernel(const Join j)
{
    constexpr int G = groups_of<NT>(), BLOCK = NT * G;
    __shared__ float part[2][2][BLOCK / 64];
    RowSums<NT, G> sums{part};
    const int tid = threadIdx.x % NT;
    int col[NV], hi[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) { col[k] = 8 * (tid + NT * k); hi[k] = min(8, j.cols - col[k]); }
    uint64_t seed = 0, offset = 0;
    if (j.drop) { seed = j.rng[0]; offset = j.rng[1]; }
    // gradients of the vectors: bias, gate, weight and bias of the post norm, of the pre norm
    constexpr int SETS = 2 + (POST ? 2 : 0) + (PRE ? 2 : 0), AT_POST = 2, AT_PRE = POST ? 4 : 2;
    float total[SETS][NV][8];
#pragma unroll
    for (int s = 0; s < SETS; ++s)
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) total[s][k][e] = 0.f;

    for (int64_t base = (int64_t)blockIdx.x * G; base < j.rows; base += (int64_t)gridDim.x * G) {
        const int64_t row = base + threadIdx.x / NT;
        const bool on = row < j.rows;
        float t[NV][8], x[NV][8], d[NV][8], g[NV][8], rt = 0.f, rx = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int h = on ? hi[k] : 0;
            row8<T>(j.dx_out, j.lddxo, row, col[k], h, d[k]);
            if constexpr (PRE) {
                row8<T>(j.x, j.ldx, row, col[k], h, x[k]);
                row8<T>(j.dh, j.lddh, row, col[k], h, g[k]);
            }
            row8<T>(j.y, j.ldy, row, col[k], h, t[k]);
            plus<T>(t[k], j.bias, col[k], h);
            if (j.drop) Draw(seed, offset, (uint32_t)row, (uint32_t)col[k] >> 3).apply(t[k], j.drop, j.factor);
        }
        if constexpr (POST && PRE) normalise<NV, true>(x, t, rx, rt, hi, j.cols, j.layer, j.eps, sums);
        else if constexpr (PRE) normalise<NV, false>(x, x, rx, rt, hi, j.cols, j.layer, j.eps, sums);
        else if constexpr (POST) normalise<NV, false>(t, t, rt, rx, hi, j.cols, j.layer, j.eps, sums);
        if constexpr (PRE) {
#pragma unroll
            for (int k = 0; k < NV; ++k) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    total[AT_PRE][k][e] = on ? fmaf(g[k][e], x[k][e], total[AT_PRE][k][e]) : total[AT_PRE][k][e];
                    total[AT_PRE + 1][k][e] += g[k][e];
                }
                times<T>(g[k], j.pre_w, col[k], hi[k]);
            }
            norm_back<NV>(g, x, rx, hi, j.cols, j.layer, sums);
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) d[k][e] += g[k][e];
        }
        // d: the gradient at x_out and at x; t: D(y + bias), or what the post norm makes of it before its weight
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if (on && hi[k] > 0 && j.dx) store8((T*)j.dx + row * j.lddx + col[k], 0, hi[k], d[k]);
            float n[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) { d[k][e] = on ? j.scale * d[k][e] : 0.f; n[e] = t[k][e]; }
            if constexpr (POST) {
                times<T>(n, j.post_w, col[k], hi[k]);
                plus<T>(n, j.post_b, col[k], hi[k]);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) total[1][k][e] = on ? fmaf(d[k][e], n[e], total[1][k][e]) : total[1][k][e];
            times<T>(d[k], j.gate, col[k], hi[k]);
            if constexpr (POST) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    total[AT_POST][k][e] = on ? fmaf(d[k][e], t[k][e], total[AT_POST][k][e]) : total[AT_POST][k][e];
                    total[AT_POST + 1][k][e] += d[k][e];
                }
                times<T>(d[k], j.post_w, col[k], hi[k]);
            }
        }
        if constexpr (POST) norm_back<NV>(d, t, rt, hi, j.cols, j.layer, sums);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if (j.drop) Draw(seed, offset, (uint32_t)row, (uint32_t)col[k] >> 3).apply(d[k], j.drop, j.factor);
#pragma unroll
            for (int e = 0; e < 8; ++e) total[0][k][e] += on ? d[k][e] : 0.f;
            if (on && hi[k] > 0 && j.dy) store8((T*)j.dy + row * j.lddy + col[k], 0, hi[k], d[k]);
        }
    }

    if (!j.partial) return;
    // the G rows' sums of a workgroup, in their order
    __shared__ float all[G > 1 ? BLOCK * 8 : 1];
#pragma unroll
    for (int s = 0; s < SETS; ++s) {
        const int at = s < 2 ? s : POST && s < 4 ? s : 4 + (s & 1);
        float* dst = j.partial + ((size_t)at * (size_t)j.slabs + blockIdx.x) * (size_t)j.cols;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = total[s][k][e];
            if constexpr (G > 1) {
                __syncthreads();
                store8(all + threadIdx.x * 8, 0, 8, v);
                __syncthreads();
                if (threadIdx.x >= NT) continue;
#pragma unroll
                for (int q = 1; q < G; ++q)
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] += all[(threadIdx.x + NT * q) * 8 + e];
            }
            if (hi[k] > 0) store8(dst + col[k], 0, hi[k], v);
        }
    }
}

template <typename T, int NT, int NV, bool BACK>
int launch_shape(const Join& j, int blocks, hipStream_t stream)
{
    constexpr int threads = NT * groups_of<NT>();
    auto go = [&](auto post, auto pre) {
        constexpr bool POST = decltype(post)::value, PRE = decltype(pre)::value;
        if constexpr (BACK) hipLaunchKernelGGL((join_back_kernel<T, NT, NV, POST, PRE>), dim3((unsigned)blocks), dim3(threads), 0, stream, j);
        else hipLaunchKernelGGL((join_kernel<T, NT, NV, POST, PRE>), dim3((unsigned)blocks), dim3(threads), 0, stream, j);
    };
    const std::true_type yes;
    const std::false_type no;
    if (j.post && j.pre) go(yes, yes);
    else if (j.post) go(yes, no);
    else if (j.pre) go(no, yes);
    else go(no, no);
    return hip_status(hipGetLastError());
}

// workgroups of a launch for rows of `cols` columns, `rows_at_once` rows each at a time
struct Shape { int threads, rows_at_once; };
Shape shape_of(int cols)
{
    const int nt = cols <= 1024 ? 64 : cols <= 2048 ? 128 : cols <= 4096 ? 256 : cols <= 8192 ? 512 : 1024;
    return Shape{nt, nt < 256 ? 256 / nt : 1};
}

template <bool BACK, typename T>
int launch_any(const Join& j, int blocks, hipStream_t stream)
{
    if (j.cols <= 512) return launch_shape<T, 64, 1, BACK>(j, blocks, stream);
    if (j.cols <= 1024) return launch_shape<T, 64, 2, BACK>(j, blocks, stream);
    if (j.cols <= 2048) return launch_shape<T, 128, 2, BACK>(j, blocks, stream);
    if (j.cols <= 4096) return launch_shape<T, 256, 2, BACK>(j, blocks, stream);
    if (j.cols <= 8192) return launch_shape<T, 512, 2, BACK>(j, blocks, stream);
    return launch_shape<T, 1024, 2, BACK>(j, blocks, stream);
}

}  // namespace

int join_max_cols() { return MAX_COLS; }

int join_slabs(int rows, int cols)
{
    const Shape s = shape_of(cols);
    const int64_t all = ((int64_t)rows + s.rows_at_once - 1) / s.rows_at_once;
    return (int)std::min<int64_t>(all, s.threads <= 256 ? 512 : 256);
}

int launch_join(const Join& j, int dtype, hipStream_t stream)
{
    const Shape s = shape_of(j.cols);
    const int blocks = (int)std::min<int64_t>(((int64_t)j.rows + s.rows_at_once - 1) / s.rows_at_once, 2048);
    return dtype == ZR_BF16 ? launch_any<false, Bf>(j, blocks, stream) : launch_any<false, float>(j, blocks, stream);
}

int launch_join_back(const Join& j, int dtype, hipStream_t stream)
{
    return dtype == ZR_BF16 ? launch_any<true, Bf>(j, j.slabs, stream) : launch_any<true, float>(j, j.slabs, stream);
}

}  // namespace zr
