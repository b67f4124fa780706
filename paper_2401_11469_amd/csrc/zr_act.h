// What stands around the products of the layer: bias, activation, gate, dropout and residual, as device functions on
// eight neighbouring columns of a row, and the launchers of the kernels that use them.
//
// Columns are taken in aligned groups of eight everywhere (columns 8 g .. 8 g + 7 of the whole row), because one call of the
// generator gives the eight halves of a group: no element's draw depends on which kernel, tile or thread visits it.
#pragma once

#include "zr_common.h"

namespace zr {

// Applied to the result of a forward product before it is stored:
//   z = sum + bias;  Z <- z;  out <- residual + D(act(z) * gate)
struct Finish {
    const void* bias;        // [N] or nullptr
    const void* gate;        // [M x N] or nullptr
    int64_t ldg;
    const void* residual;    // [M x N] or nullptr
    int64_t ldr;
    void* Z;                 // [M x N] or nullptr
    int64_t ldz;
    const uint64_t* rng;     // seed, offset
    uint32_t drop;           // an element is dropped where its half is below this; 0: none
    float factor;            // what the others are multiplied by
    int act;
};

// Probability to halves: round(65536 p), at most 65535, and the factor that keeps the mean.
inline uint32_t drop_below(double p) { return (uint32_t)std::min(65535.0, std::floor(p * 65536.0 + 0.5)); }
inline float kept_factor(uint32_t q) { return (float)(65536.0 / (65536.0 - (double)q)); }

// ---- launchers ----------------------------------------------------------------
// act_dz: what the backward pass of a Finish does to dY before the products, T = D(dY):
//   dgate <- T act(Z);  dz <- T gate act'(Z);  partial[slab] <- column sums of dz over the slab's rows
struct ActBack {
    const void* dY; int64_t lddy;
    const void* Z; int64_t ldz;            // nullptr: no activation and no gate gradient
    const void* gate; int64_t ldg;
    void* dgate; int64_t lddg;
    void* dz; int64_t lddz;                // nullptr: not wanted
    float* partial;                        // [slabs x N] or nullptr
    const uint64_t* rng; uint32_t drop; float factor; int act;
    int M, N;
    // bf16, N above 256: dz receives these columns side by side, [M x width] with zeros behind the last (nullptr: all, in their places)
    const int32_t* keep; int n_keep; int width;
};
constexpr int ACT_KEPT_ABOVE = 256;        // (a wavefront has a row then)
int act_slabs(int M, int N);
int launch_act_back(const ActBack& a, int dtype, hipStream_t stream);
// out[c] = sum over slabs of partial[slab * n + c], in slab order
int launch_sum_slabs(const float* partial, int slabs, int n, void* out, int dtype, hipStream_t stream);
int launch_dropout(const void* x, int64_t ldx, void* out, int64_t ldo, int rows, int cols, const uint64_t* rng, uint32_t drop,
                   float factor, int dtype, hipStream_t stream);

// A block's output joins the residual stream: t = D(y + bias), n = post(t), x_out = x + scale gate n, h = pre(x_out).
struct Join {
    const void* y; int64_t ldy;
    const void* x; int64_t ldx;            // forward: the stream before; backward: behind the block (what h is the norm of)
    void* x_out; int64_t ldxo;
    void* h; int64_t ldh;
    const void *bias, *gate, *post_w, *post_b, *pre_w, *pre_b;      // [cols] or nullptr
    float scale, eps;
    int post, pre, layer;                  // which norms there are; layer norms (else root mean square)
    const uint64_t* rng; uint32_t drop; float factor;
    int rows, cols;
    // backward
    const void* dx_out; int64_t lddxo;     // nullptr: zeros
    const void* dh; int64_t lddh;
    void* dx; int64_t lddx;
    void* dy; int64_t lddy;
    float* partial;                        // [sums x slabs x cols], the sums below; without `biases` the first two
    int slabs;
    void* vectors[6];                      // gradients of bias, gate, post_w, post_b, pre_w, pre_b; each may be nullptr
    int biases;                            // sums of d, dh or dy are wanted: a gradient of bias, post_b or pre_b, or of the gate beside a post_b
};
enum { SUM_DT, SUM_HAT, SUM_D, SUM_DY, SUM_DH, JOIN_SUMS };     // over the rows: of d t, dh times the pre norm's value, d, dy, dh
int join_max_cols();
int join_most_slabs(int rows, int cols);                // of any backward call of this size
int join_slabs(const Join& j);                          // of this one
int launch_join(const Join& j, int dtype, hipStream_t stream);
int launch_join_back(const Join& j, int dtype, hipStream_t stream);
int launch_join_sums(const Join& j, int dtype, hipStream_t stream);

// products with a Finish (GemmDesc::finish set): any alignment, and fp32
constexpr int ACT_FEW = 16;     // rows of X up to which launch_act_few takes a product
constexpr int ACT_FEW_GATHERED = 4;     // and up to which it is left to gather the kept columns of X
int launch_act_few(const GemmDesc& d, hipStream_t stream);      // bf16, few rows; -1: not taken
int launch_act_any(const GemmDesc& d, hipStream_t stream);
int launch_act_narrow(const GemmDesc& d, int j_base, hipStream_t stream);      // columns j_base .. of a product without lists on a contiguous axis, on 32 x 32 tiles; -1: not taken
int launch_act_fast(const GemmDesc& d, hipStream_t stream);     // bf16, 16-byte aligned rows; -1: not taken
int launch_act_f32(const GemmDesc& d, hipStream_t stream);

// ---- device functions -----------------------------------------------------------
namespace {

typedef uint16_t Bf;
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4_any __attribute__((ext_vector_type(4), aligned(2)));       // 16 bytes at any bf16 element
typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f4_any __attribute__((ext_vector_type(4), aligned(4)));

// round to nearest, ties to even (v_cvt_pk_bf16_f32)
__device__ __forceinline__ uint32_t round_two(float a, float b)
{
    union { __bf16 h[2]; uint32_t u; } x;
    x.h[0] = (__bf16)a;
    x.h[1] = (__bf16)b;
    return x.u;
}

__device__ __forceinline__ float one_of(const Bf* p) { return bf16_bits_to_f32(*p); }
__device__ __forceinline__ float one_of(const float* p) { return *p; }
__device__ __forceinline__ void put_one(Bf* p, float v) { *p = (Bf)round_two(v, 0.f); }
__device__ __forceinline__ void put_one(float* p, float v) { *p = v; }

// Eight values as they lie in memory, at any element address.
template <typename T> struct Raw8;
template <> struct Raw8<Bf> {
    u4 v;
    __device__ __forceinline__ void load(const Bf* p) { v = *(const u4_any*)p; }
    __device__ __forceinline__ void values(float (&x)[8]) const
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[2 * e] = __uint_as_float(v[e] << 16);
            x[2 * e + 1] = __uint_as_float(v[e] & 0xffff0000u);
        }
    }
    __device__ __forceinline__ void take(const float (&x)[8])
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = round_two(x[2 * e], x[2 * e + 1]);
    }
    __device__ __forceinline__ void store(Bf* p) const { *(u4_any*)p = v; }
    __device__ __forceinline__ void clear() { v = u4{0u, 0u, 0u, 0u}; }
};
template <> struct Raw8<float> {
    f4 v[2];
    __device__ __forceinline__ void load(const float* p) { v[0] = *(const f4_any*)p; v[1] = *(const f4_any*)(p + 4); }
    __device__ __forceinline__ void values(float (&x)[8]) const
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = v[e >> 2][e & 3];
    }
    __device__ __forceinline__ void take(const float (&x)[8])
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e >> 2][e & 3] = x[e];
    }
    __device__ __forceinline__ void store(float* p) const { *(f4_any*)p = v[0]; *(f4_any*)(p + 4) = v[1]; }
    __device__ __forceinline__ void clear() { v[0] = v[1] = f4{0.f, 0.f, 0.f, 0.f}; }
};

// Elements lo .. hi - 1 of the eight at p (the others: 0, and left as they are)
template <typename T> __device__ __forceinline__ void load8(const T* p, int lo, int hi, float (&x)[8])
{
    if (lo == 0 && hi == 8) {
        Raw8<T> r;
        r.load(p);
        r.values(x);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = e >= lo && e < hi ? one_of(p + e) : 0.f;
    }
}
template <typename T> __device__ __forceinline__ void store8(T* p, int lo, int hi, const float (&x)[8])
{
    if (lo == 0 && hi == 8) {
        Raw8<T> r;
        r.take(x);
        r.store(p);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e >= lo && e < hi) put_one(p + e, x[e]);
    }
}

// Philox 4 x 32 of 7 rounds (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011: the fewest that
// passed all their tests), key = seed, counter = (group of eight columns, row, offset): eight halves for the group.
// 14 products of 32 x 32 bits for eight elements, at a quarter of the rate of an addition.
struct Draw {
    uint32_t w[4];
    __device__ __forceinline__ Draw(uint64_t seed, uint64_t offset, uint32_t row, uint32_t group)
    {
        uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
        uint32_t c0 = group, c1 = row, c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
#pragma unroll
        for (int i = 0; i < 7; ++i) {
            const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
            c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
            c1 = (uint32_t)b;
            c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
            c3 = (uint32_t)a;
            k0 += 0x9E3779B9u;
            k1 += 0xBB67AE85u;
        }
        w[0] = c0; w[1] = c1; w[2] = c2; w[3] = c3;
    }
    __device__ __forceinline__ bool kept(int e, uint32_t drop) const
    {
        return (e & 1 ? w[e >> 1] >> 16 : w[e >> 1] & 0xffffu) >= drop;
    }
    // (the same for an e that is not known at compile time: no indexed registers)
    __device__ __forceinline__ bool kept_at(int e, uint32_t drop) const
    {
        const uint64_t low = w[0] | (uint64_t)w[1] << 32, high = w[2] | (uint64_t)w[3] << 32;
        return (uint32_t)((e < 4 ? low : high) >> 16 * (e & 3) & 0xffffu) >= drop;
    }
    // bit e: element e is kept
    __device__ __forceinline__ uint32_t bits(uint32_t drop) const
    {
        uint32_t b = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) b |= kept(e, drop) ? 1u << e : 0u;
        return b;
    }
    // a dropped element is +0 whatever it was
    __device__ __forceinline__ void apply(float (&x)[8], uint32_t drop, float factor) const
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = kept(e, drop) ? x[e] * factor : 0.f;
    }
};

// e^x: bf16 results take the hardware's power of two (off by about |x| 2^-24 in all), fp32 ones the library's
template <bool EXACT> __device__ __forceinline__ float exp_of(float x)
{
    if constexpr (EXACT) return expf(x);
    else return __builtin_amdgcn_exp2f(x * 1.44269504f);
}
template <bool EXACT> __device__ __forceinline__ float recip(float x)
{
    if constexpr (EXACT) return 1.f / x;
    else return __builtin_amdgcn_rcpf(x);
}
template <bool EXACT> __device__ __forceinline__ float sigmoid_of(float x) { return recip<EXACT>(1.f + exp_of<EXACT>(-x)); }

// z Phi(z) and Phi(z) + z phi(z), Phi the normal distribution function and phi its density, by the tail T = Phi(-|z|):
//   z Phi(z) = max(z, 0) - |z| T
// bf16 results: T = t P(t) e^(-z^2 / 2) with t = 1 / (1 + 0.285 |z|), which goes to 0 as T e^(z^2 / 2) does (as 1 / |z|), and P of fifth
// degree, fitted for the smallest largest error where 7e-8 counts as much as 4.5e-4 of T: off by 6e-8 and by 2.5e-4 of T at most, before
// the roundings of fp32, where a bf16 result is off by 2^-9 of itself.  So small results keep their size, down to 1e-37 (one degree less: 3.5e-7
// at these tails).  fp32 results: the library's erfc.
template <bool EXACT, bool SLOPE> __device__ __forceinline__ void gelu_of(float z, float& a, float& s)
{
    if constexpr (EXACT) {
        const float cdf = 0.5f * erfcf(-0.70710678f * z);
        a = z * cdf;
        if constexpr (SLOPE) s = fmaf(z, 0.39894228f * expf(-0.5f * z * z), cdf);
    } else {
        const float e = __builtin_amdgcn_exp2f(z * (z * -0.72134752f));            // e^(-z^2 / 2)
        const float t = __builtin_amdgcn_rcpf(fmaf(0.285f, fabsf(z), 1.f));
        float p = -0.09544432f;
        p = fmaf(p, t, 0.32764384f);
        p = fmaf(p, t, -0.14764132f);
        p = fmaf(p, t, 0.20968573f);
        p = fmaf(p, t, 0.0899962f);
        p = fmaf(p, t, 0.115759924f);
        const float tail = p * t * e;
        // (not fmaxf: NaN stays NaN; an infinite z has no tail to be multiplied by)
        a = fmaf(-fminf(fabsf(z), 3e38f), tail, z < 0.f ? 0.f : z);
        if constexpr (SLOPE) s = fmaf(z, 0.39894228f * e, z > 0.f ? 1.f - tail : tail);
    }
}

// a = act(z), s = act'(z) (SLOPE)
template <bool EXACT, bool SLOPE> __device__ __forceinline__ void act_one(int act, float z, float& a, float& s)
{
    if (act == ZR_ACT_RELU) {
        a = z < 0.f ? 0.f : z;          // (NaN stays NaN)
        s = z > 0.f ? 1.f : 0.f;
    } else if (act == ZR_ACT_GELU) {
        gelu_of<EXACT, SLOPE>(z, a, s);
    } else if (act == ZR_ACT_GELU_TANH) {
        // (1 + tanh u) / 2 is the sigmoid of 2 u, u = sqrt(2 / pi) (z + 0.044715 z^3)
        const float zz = z * z, t = sigmoid_of<EXACT>(1.59576912f * z * fmaf(0.044715f, zz, 1.f));
        a = z * t;
        // (1 - t = 0 or t = 0 long before z^2 is held at 1e12: no infinity to be multiplied by)
        if constexpr (SLOPE) s = fmaf(z * t * (1.f - t), 1.59576912f * fmaf(0.134145f, fminf(zz, 1e12f), 1.f), t);
    } else if (act == ZR_ACT_SILU) {
        const float t = sigmoid_of<EXACT>(z);
        a = z * t;
        if constexpr (SLOPE) s = t * fmaf(z, 1.f - t, 1.f);
    } else {
        a = z;
        s = 1.f;
    }
}
// (the choice outside the loop: one uniform branch for eight elements)
template <bool EXACT, bool SLOPE> __device__ __forceinline__ void act8(int act, const float (&z)[8], float (&a)[8], float (&s)[8])
{
    auto all = [&](int which) {
#pragma unroll
        for (int e = 0; e < 8; ++e) act_one<EXACT, SLOPE>(which, z[e], a[e], s[e]);
    };
    switch (act) {
        case ZR_ACT_RELU: all(ZR_ACT_RELU); break;
        case ZR_ACT_GELU: all(ZR_ACT_GELU); break;
        case ZR_ACT_GELU_TANH: all(ZR_ACT_GELU_TANH); break;
        case ZR_ACT_SILU: all(ZR_ACT_SILU); break;
        default: all(ZR_ACT_NONE); break;
    }
}

// The group of eight columns at col (a multiple of 8) of one row of a product: z holds the sums; bias, gate, residual what lies
// there, requested before.
template <typename T>
__device__ __forceinline__ void finish8(const Finish& f, T* out, int64_t ldo, int row, int col, float (&z)[8], const Raw8<T>& bias,
                                        const Raw8<T>& gate, const Raw8<T>& residual)
{
    constexpr bool EXACT = sizeof(T) == 4;
    float x[8], a[8], unused[8];
    if (f.bias) {
        bias.values(x);
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] += x[e];
    }
    if (f.Z) store8((T*)f.Z + (size_t)row * (size_t)f.ldz + col, 0, 8, z);
    act8<EXACT, false>(f.act, z, a, unused);
    if (f.gate) {
        gate.values(x);
#pragma unroll
        for (int e = 0; e < 8; ++e) a[e] *= x[e];
    }
    if (f.drop) Draw(f.rng[0], f.rng[1], (uint32_t)row, (uint32_t)col >> 3).apply(a, f.drop, f.factor);
    if (f.residual) {
        residual.values(x);
#pragma unroll
        for (int e = 0; e < 8; ++e) a[e] += x[e];
    }
    store8(out + (size_t)row * (size_t)ldo + col, 0, 8, a);
}

// One element, the same way.
template <typename T>
__device__ __forceinline__ void finish1(const Finish& f, T* out, int64_t ldo, int row, int col, float z)
{
    float a, unused;
    if (f.bias) z += one_of((const T*)f.bias + col);
    if (f.Z) put_one((T*)f.Z + (size_t)row * (size_t)f.ldz + col, z);
    act_one<sizeof(T) == 4, false>(f.act, z, a, unused);
    if (f.gate) a *= one_of((const T*)f.gate + (size_t)row * (size_t)f.ldg + col);
    if (f.drop) a = Draw(f.rng[0], f.rng[1], (uint32_t)row, (uint32_t)col >> 3).kept_at(col & 7, f.drop) ? a * f.factor : 0.f;
    if (f.residual) a += one_of((const T*)f.residual + (size_t)row * (size_t)f.ldr + col);
    put_one(out + (size_t)row * (size_t)ldo + col, a);
}

// Rows row0 .. row0 + rows - 1 of a tile of R columns whose sums lie in LDS (Cs, pitch CP floats), NT threads.
// sidx == nullptr: the tile's columns are col0 .. col0 + cols - 1 (col0 a multiple of 8).  Otherwise sidx[j] is the original
// column of the tile's column j, ascending, and the tile owns the original columns start .. end - 1: those without an entry have
// the sum 0.  tab: TAB words of LDS, 16-byte aligned.  Every thread of the workgroup calls it; LDS is free again after a barrier.
// Whole groups of eight leave as such, a thread requesting what it needs of U of them together; the elements of the groups that a
// tile shares with its neighbours, or at the end of a row, go out one by one in a pass of their own (as a branch among the groups
// they are in every wavefront's way: 8192 x 4096 x 2752 of 2064 kept, gated 170 us without the remainder panel's split, now 144 with).
template <int NT, int R, int TAB, int U, typename T>
__device__ __forceinline__ void finish_tile(const Finish& f, T* out, int64_t ldo, const float* Cs, int CP, int row0, int rows, int col0,
                                            int cols, const int* sidx, int start, int end, int* tab, int tid)
{
    static_assert(TAB % 8 == 0, "whole groups");
    // `count` whole groups, sums(r, col, z) gives those of row r; where(i, r, col) says where group i lies
    auto whole = [&](int count, auto where, auto sums) {
        for (int i0 = tid; i0 < count; i0 += NT * U) {
            Raw8<T> b[U], g[U], r[U];
            int at[U], col[U];
#pragma unroll
            for (int i = 0; i < U; ++i) where(min(i0 + NT * i, count - 1), at[i], col[i]);        // (past the end: the last one, not stored)
            if (f.bias) {
#pragma unroll
                for (int i = 0; i < U; ++i) b[i].load((const T*)f.bias + col[i]);
            }
            if (f.gate) {
#pragma unroll
                for (int i = 0; i < U; ++i) g[i].load((const T*)f.gate + (size_t)(row0 + at[i]) * (size_t)f.ldg + col[i]);
            }
            if (f.residual) {
#pragma unroll
                for (int i = 0; i < U; ++i) r[i].load((const T*)f.residual + (size_t)(row0 + at[i]) * (size_t)f.ldr + col[i]);
            }
#pragma unroll
            for (int i = 0; i < U; ++i) {
                if (i0 + NT * i >= count) break;
                float z[8];
                sums(at[i], col[i], z);
                finish8(f, out, ldo, row0 + at[i], col[i], z, b[i], g[i], r[i]);
            }
        }
    };
    // elements [lo1, hi1) and [lo2, hi2) of every row
    auto single = [&](int lo1, int hi1, int lo2, int hi2, auto sum) {
        const int n1 = max(hi1 - lo1, 0), n = n1 + max(hi2 - lo2, 0);
        for (int u = tid; u < rows * n; u += NT) {
            const int r = u / n, e = u - r * n, col = e < n1 ? lo1 + e : lo2 + (e - n1);
            finish1(f, out, ldo, row0 + r, col, sum(r, col));
        }
    };
    if (!sidx) {
        constexpr int GROUPS = R / 8;
        auto sums = [&](int r, int col, float (&z)[8]) {
            const float* c = Cs + r * CP + col - col0;
            const f4 z0 = *(const f4*)c, z1 = *(const f4*)(c + 4);
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] = e < 4 ? z0[e & 3] : z1[e & 3];
        };
        const int groups = cols >> 3;
        if (groups == GROUPS) whole(rows * GROUPS, [&](int i, int& r, int& col) { r = i / GROUPS; col = col0 + 8 * (i % GROUPS); }, sums);
        else whole(rows * groups, [&](int i, int& r, int& col) { r = i / groups; col = col0 + 8 * (i - r * groups); }, sums);
        single(col0 + 8 * groups, col0 + cols, 0, 0, [&](int r, int col) { return Cs[r * CP + col - col0]; });
        return;
    }
    for (int base = start & ~7; base < end; base += TAB) {
        const int lo = max(start, base), hi = min(end, base + TAB);
        for (int q = tid; q < TAB; q += NT) tab[q] = -1;
        __syncthreads();
        for (int q = tid; q < cols; q += NT) {
            const int p = sidx[q] - base;
            if (p >= 0 && p < TAB) tab[p] = q;
        }
        __syncthreads();
        const int first = (lo + 7) & ~7, last = hi & ~7, groups = max(last - first, 0) >> 3;
        // (count below 2^23, so the quotient is exact but for a last bit that the half step covers)
        const float inv = 1.f / (float)max(groups, 1);
        whole(rows * groups,
              [&](int i, int& r, int& col) {
                  r = (int)(((float)i + 0.5f) * inv);
                  col = first + 8 * (i - r * groups);
              },
              [&](int r, int col, float (&z)[8]) {
                  typedef int i4 __attribute__((ext_vector_type(4)));
                  const i4 j0 = *(const i4*)(tab + col - base), j1 = *(const i4*)(tab + col - base + 4);
#pragma unroll
                  for (int e = 0; e < 8; ++e) {
                      const int j = e < 4 ? j0[e & 3] : j1[e & 3];
                      const float v = Cs[r * CP + max(j, 0)];
                      z[e] = j >= 0 ? v : 0.f;
                  }
              });
        const int mid = min(first, hi);
        single(lo, mid, max(last, mid), hi, [&](int r, int col) { const int j = tab[col - base]; return j >= 0 ? Cs[r * CP + j] : 0.f; });
        __syncthreads();
    }
}

}  // namespace

}  // namespace zr
