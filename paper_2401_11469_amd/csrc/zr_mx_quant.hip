// Tensors into blocks of 32 with a power of two each, and back (zr_mx.h has the format).  All of it is bound by memory:
// every value is read once, its block's largest magnitude is found among the few lanes (or in the one thread) that hold
// the block, and the elements leave in the same pass.
#include "zr_mx.h"

namespace zr {

namespace {

constexpr int SEG = 512;        // values of a row that a wavefront handles at a time: 8 a lane, one group of scales

__device__ __forceinline__ float as_float(uint16_t v) { return bf16_bits_to_f32(v); }
__device__ __forceinline__ float as_float(float v) { return v; }

// eight neighbouring values, 16-byte aligned
__device__ __forceinline__ void load8(const uint16_t* p, float (&x)[8])
{
    const uint4 v = *(const uint4*)p;
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ void load8(const float* p, float (&x)[8])
{
    const float4 a = *(const float4*)p, b = *(const float4*)(p + 4);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}

// One row's values seg * 512 + 8 * lane .. + 7 (zeros from n on) into the row's elements and scales.  Four lanes hold a
// block.  Called by whole wavefronts.
template <int FMT>
__device__ __forceinline__ void store_seg(const float (&x)[8], uint8_t* __restrict__ q, uint8_t* __restrict__ s, int n, int seg, int lane)
{
    uint32_t a = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) a = max(a, __float_as_uint(x[i]) & 0x7fffffffu);
    a = max(a, (uint32_t)__shfl_xor((int)a, 1, 64));
    a = max(a, (uint32_t)__shfl_xor((int)a, 2, 64));
    const int c = mx_code<FMT>(a);
    const int at = seg * SEG + 8 * lane;
    if (at < (n + 127) / 128 * 128) {
        const uint2 e = mx_encode8<FMT>(x, c == 255 ? 0.f : mx_inv(c));
        if constexpr (FMT == ZR_MX_E2M1) *(uint32_t*)(q + at / 2) = e.x;
        else *(uint2*)(q + at) = e;
    }
    if ((lane & 3) == 0) s[mx_scale_at(seg * 16 + (lane >> 2))] = at < n ? c : 0;
}

// Rows of 16-byte loads, nothing gathered: a wavefront takes a segment of four rows, all requested together.
template <class T, int FMT>
__global__ __launch_bounds__(256) void mx_rows_kernel(const T* __restrict__ src, int64_t ld, int rows, int n, int segs,
                                                      uint8_t* __restrict__ q, int64_t ldq, uint8_t* __restrict__ s, int64_t lds)
{
    constexpr int RB = 4;
    const int lane = threadIdx.x & 63;
    const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int r0 = (int)(item / segs) * RB, seg = (int)(item % segs);
    if (r0 >= rows) return;
    const int at = seg * SEG + 8 * lane;
    float x[RB][8];
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        const T* p = src + (size_t)min(r0 + r, rows - 1) * (size_t)ld;
        if (at + 8 <= n) load8(p + at, x[r]);
        else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[r][i] = at + i < n ? as_float(p[at + i]) : 0.f;
        }
    }
#pragma unroll
    for (int r = 0; r < RB; ++r)
        if (r0 + r < rows) store_seg<FMT>(x[r], q + (size_t)(r0 + r) * (size_t)ldq, s + (size_t)(r0 + r) * (size_t)lds, n, seg, lane);
}

// Rows of any alignment, and gathered columns: RB whole rows come into LDS in aligned 16-byte chunks (the chunks at a row's
// ends by elements), and are picked from there.
template <class T, int FMT>
__global__ __launch_bounds__(256) void mx_gather_kernel(const T* __restrict__ src, int64_t ld, int rows, int cols, const int32_t* __restrict__ keep,
                                                        int n, int segs, int rb, int pitch, uint8_t* __restrict__ q, int64_t ldq,
                                                        uint8_t* __restrict__ s, int64_t lds)
{
    extern __shared__ __align__(16) uint8_t stage[];
    constexpr int ES = sizeof(T), PER = 16 / ES;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int r0 = blockIdx.x * rb, nr = min(rb, rows - r0);
    for (int r = 0; r < nr; ++r) {
        const T* row = src + (size_t)(r0 + r) * (size_t)ld;
        const int off = (int)((uintptr_t)row & 15) / ES;         // elements between the aligned address and the row
        const int chunks = (off + cols + PER - 1) / PER;
        uint8_t* dst = stage + r * pitch;
        for (int c0 = 0; c0 < chunks; c0 += 1024) {
            uint4 v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int c = c0 + u * 256 + tid, e = c * PER - off;
                if (e >= 0 && e + PER <= cols) v[u] = *(const uint4*)(row + e);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int c = c0 + u * 256 + tid, e = c * PER - off;
                if (e >= 0 && e + PER <= cols) *(uint4*)(dst + c * 16) = v[u];
                else if (c < chunks) {
                    for (int i = max(e, 0); i < min(e + PER, cols); ++i) *(T*)(dst + (off + i) * ES) = row[i];
                }
            }
        }
    }
    __syncthreads();
    for (int seg = wave; seg < segs; seg += 4) {
        const int at = seg * SEG + 8 * lane;
        int pick[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) pick[i] = keep ? clamp_idx(keep[min(at + i, n - 1)], cols) : min(at + i, n - 1);
        for (int r = 0; r < nr; ++r) {
            const size_t row = (size_t)(r0 + r);
            const T* d = (const T*)(stage + r * pitch) + (int)((uintptr_t)(src + row * (size_t)ld) & 15) / ES;
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) { const float v = as_float(d[pick[i]]); x[i] = at + i < n ? v : 0.f; }
            store_seg<FMT>(x, q + row * (size_t)ldq, s + row * (size_t)lds, n, seg, lane);
        }
    }
}

// Rows too long for LDS that are gathered or of any alignment: element by element.
template <class T, int FMT>
__global__ __launch_bounds__(256) void mx_long_kernel(const T* __restrict__ src, int64_t ld, int rows, int cols, const int32_t* __restrict__ keep,
                                                      int n, int segs, uint8_t* __restrict__ q, int64_t ldq, uint8_t* __restrict__ s, int64_t lds)
{
    const int lane = threadIdx.x & 63;
    const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int r = (int)(item / segs), seg = (int)(item % segs);
    if (r >= rows) return;
    const int at = seg * SEG + 8 * lane;
    const T* p = src + (size_t)r * (size_t)ld;
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int k = min(at + i, n - 1);
        const float v = as_float(p[keep ? clamp_idx(keep[k], cols) : k]);
        x[i] = at + i < n ? v : 0.f;
    }
    store_seg<FMT>(x, q + (size_t)r * (size_t)ldq, s + (size_t)r * (size_t)lds, n, seg, lane);
}

// Blocks along the strided axis: a tile of 128 (kept) rows x 64 columns comes into LDS; each thread then takes one block of
// one column (its lanes 64 neighbouring columns: no bank conflicts, no exchange between lanes), and the elements go through
// LDS once more, so that each column's 64 or 128 bytes leave together.
template <class T, int FMT, bool VEC>
__global__ __launch_bounds__(256) void mx_cols_kernel(const T* __restrict__ src, int64_t ld, int rows, int cols, const int32_t* __restrict__ keep,
                                                      int n, uint8_t* __restrict__ q, int64_t ldq, uint8_t* __restrict__ s, int64_t lds)
{
    constexpr int KT = 128, CT = 64, PITCH = CT + 16 / (int)sizeof(T);
    constexpr int OB = FMT == ZR_MX_E2M1 ? 64 : 128, OP = OB + 16;       // bytes of a column's elements in a tile
    __shared__ __align__(16) T tile[KT * PITCH];
    __shared__ __align__(16) uint8_t outs[CT * OP];
    const int tid = threadIdx.x;
    const int c0 = blockIdx.x * CT, k0 = blockIdx.y * KT;
    if constexpr (VEC) {
        constexpr int PER = 16 / sizeof(T), LPR = CT / PER, RPP = 256 / LPR, PASSES = KT / RPP;
        uint4 v[PASSES];
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            const int k = min(k0 + p * RPP + tid / LPR, n - 1), c = c0 + tid % LPR * PER;
            const int row = keep ? clamp_idx(keep[k], rows) : k;
            v[p] = *(const uint4*)(src + (size_t)row * (size_t)ld + min(c, cols - PER));     // cols is a multiple of PER here
        }
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            const int k = p * RPP + tid / LPR;
            *(uint4*)(tile + k * PITCH + tid % LPR * PER) = k0 + k < n ? v[p] : make_uint4(0u, 0u, 0u, 0u);
        }
    } else {
        const int c = min(c0 + (tid & 63), cols - 1);
        for (int i0 = 0; i0 < KT / 4; i0 += 8) {
            T v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int k = min(k0 + (i0 + i) * 4 + (tid >> 6), n - 1);
                v[i] = src[(size_t)(keep ? clamp_idx(keep[k], rows) : k) * (size_t)ld + c];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int k = (i0 + i) * 4 + (tid >> 6);
                tile[k * PITCH + (tid & 63)] = k0 + k < n ? v[i] : T(0);
            }
        }
    }
    __syncthreads();
    const int col = tid & 63, blk = tid >> 6;
    float x[4][8];
    uint32_t a = 0;
#pragma unroll
    for (int o = 0; o < 4; ++o)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[o][i] = as_float(tile[(blk * 32 + o * 8 + i) * PITCH + col]);
            a = max(a, __float_as_uint(x[o][i]) & 0x7fffffffu);
        }
    const int code = mx_code<FMT>(a);
    const float inv = code == 255 ? 0.f : mx_inv(code);
#pragma unroll
    for (int o = 0; o < 4; ++o) {
        const uint2 e = mx_encode8<FMT>(x[o], inv);
        if constexpr (FMT == ZR_MX_E2M1) *(uint32_t*)(outs + col * OP + blk * 16 + o * 4) = e.x;
        else *(uint2*)(outs + col * OP + blk * 32 + o * 8) = e;
    }
    if (c0 + col < cols) {
        uint8_t* row = s + (size_t)(c0 + col) * (size_t)lds;
        const int b = k0 / 32 + blk;
        row[mx_scale_at(b)] = b * 32 < n ? code : 0;
        // behind the last tile: the rest of its group of 16
        if (k0 + KT >= n)
            for (int z = b + 4; z < (k0 / 512 + 1) * 16; z += 4) row[mx_scale_at(z)] = 0;
    }
    __syncthreads();
    constexpr int LPC = OB / 16;
    for (int u = tid; u < CT * LPC; u += 256) {
        const int c = u / LPC, o = u % LPC * 16;
        if (c0 + c < cols) *(uint4*)(q + (size_t)(c0 + c) * (size_t)ldq + (FMT == ZR_MX_E2M1 ? k0 / 2 : k0) + o) = *(const uint4*)(outs + c * OP + o);
    }
}

__device__ __forceinline__ void put8(uint16_t* p, const float (&x)[8])
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = f32_to_bf16_bits(x[2 * i]) | f32_to_bf16_bits(x[2 * i + 1]) << 16;
    *(uint4*)p = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void put8(float* p, const float (&x)[8])
{
    *(float4*)p = make_float4(x[0], x[1], x[2], x[3]);
    *(float4*)(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void put1(uint16_t* p, float v) { *p = (uint16_t)f32_to_bf16_bits(v); }
__device__ __forceinline__ void put1(float* p, float v) { *p = v; }

// Blocks back into values.  A wavefront takes a segment of four rows; VEC: 16-byte stores.
template <class T, int FMT, bool VEC>
__global__ __launch_bounds__(256) void mx_values_kernel(const uint8_t* __restrict__ q, int64_t ldq, const uint8_t* __restrict__ s, int64_t lds,
                                                        int rows, int n, int segs, T* __restrict__ out, int64_t ldo, int width)
{
    constexpr int RB = 4;
    const int lane = threadIdx.x & 63;
    const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int r0 = (int)(item / segs) * RB, seg = (int)(item % segs);
    if (r0 >= rows) return;
    const int at = seg * SEG + 8 * lane;
    if (at >= width) return;
    uint2 e[RB];
    int c[RB];
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        const size_t row = (size_t)min(r0 + r, rows - 1);
        if constexpr (FMT == ZR_MX_E2M1) e[r] = make_uint2(*(const uint32_t*)(q + row * (size_t)ldq + at / 2), 0u);
        else e[r] = *(const uint2*)(q + row * (size_t)ldq + at);
        c[r] = s[row * (size_t)lds + mx_scale_at(seg * 16 + (lane >> 2))];
    }
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        if (r0 + r >= rows) break;
        float x[8];
        mx_decode8<FMT>(e[r], mx_scale(c[r]), x);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = at + i < n ? x[i] : 0.f;
        T* o = out + (size_t)(r0 + r) * (size_t)ldo + at;
        if (VEC && at + 8 <= width) put8(o, x);
        else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (at + i < width) put1(o + i, x[i]);
        }
    }
}

template <class T, int FMT>
int quantize_rows(const T* src, int64_t ld, int rows, int cols, const int32_t* keep, int n, uint8_t* q, int64_t ldq, uint8_t* s, int64_t lds, hipStream_t stream)
{
    const int segs = (n + SEG - 1) / SEG;
    const int es = (int)sizeof(T);
    if (!keep && (uintptr_t)src % 16 == 0 && ld * es % 16 == 0) {
        const int64_t waves = (int64_t)((rows + 3) / 4) * segs;
        hipLaunchKernelGGL((mx_rows_kernel<T, FMT>), dim3((uint32_t)((waves + 3) / 4)), dim3(256), 0, stream, src, ld, rows, n, segs, q, ldq, s, lds);
        return hip_status(hipGetLastError());
    }
    const int pitch = (cols * es + 15 + 15) / 16 * 16;
    if (pitch <= 64 * 1024) {
        const int rb = std::max(1, std::min(4, 32 * 1024 / pitch));
        hipLaunchKernelGGL((mx_gather_kernel<T, FMT>), dim3((rows + rb - 1) / rb), dim3(256), (size_t)rb * pitch, stream, src, ld, rows, cols, keep, n, segs, rb,
                           pitch, q, ldq, s, lds);
        return hip_status(hipGetLastError());
    }
    const int64_t waves = (int64_t)rows * segs;
    hipLaunchKernelGGL((mx_long_kernel<T, FMT>), dim3((uint32_t)((waves + 3) / 4)), dim3(256), 0, stream, src, ld, rows, cols, keep, n, segs, q, ldq, s, lds);
    return hip_status(hipGetLastError());
}

template <class T, int FMT>
int quantize_cols(const T* src, int64_t ld, int rows, int cols, const int32_t* keep, int n, uint8_t* q, int64_t ldq, uint8_t* s, int64_t lds, hipStream_t stream)
{
    constexpr int PER = 16 / (int)sizeof(T);
    const dim3 grid((cols + 63) / 64, (n + 127) / 128);
    if ((uintptr_t)src % 16 == 0 && ld % PER == 0 && cols % PER == 0)
        hipLaunchKernelGGL((mx_cols_kernel<T, FMT, true>), grid, dim3(256), 0, stream, src, ld, rows, cols, keep, n, q, ldq, s, lds);
    else
        hipLaunchKernelGGL((mx_cols_kernel<T, FMT, false>), grid, dim3(256), 0, stream, src, ld, rows, cols, keep, n, q, ldq, s, lds);
    return hip_status(hipGetLastError());
}

template <class T, int FMT>
int dequantize(const MxArg& x, int rows, int n, T* out, int64_t ldo, int width, hipStream_t stream)
{
    const int segs = (width + SEG - 1) / SEG;
    const int64_t waves = (int64_t)((rows + 3) / 4) * segs;
    const dim3 grid((uint32_t)((waves + 3) / 4));
    if ((uintptr_t)out % 16 == 0 && ldo * (int64_t)sizeof(T) % 16 == 0)
        hipLaunchKernelGGL((mx_values_kernel<T, FMT, true>), grid, dim3(256), 0, stream, x.q, x.ldq, x.s, x.lds, rows, n, segs, out, ldo, width);
    else
        hipLaunchKernelGGL((mx_values_kernel<T, FMT, false>), grid, dim3(256), 0, stream, x.q, x.ldq, x.s, x.lds, rows, n, segs, out, ldo, width);
    return hip_status(hipGetLastError());
}

#define ZR_MX_EACH(CALL, T)                                    \
    switch (fmt) {                                             \
        case ZR_MX_E4M3: return CALL(T, ZR_MX_E4M3);           \
        case ZR_MX_E2M1: return CALL(T, ZR_MX_E2M1);           \
        default: return CALL(T, ZR_MX_INT8);                   \
    }

}  // namespace

int launch_mx_quantize_rows(const void* src, int64_t ld, int rows, int cols, const int32_t* keep, int n, int dtype, int fmt,
                            uint8_t* q, int64_t ldq, uint8_t* s, int64_t lds, hipStream_t stream)
{
#define ZR_CALL(T, F) quantize_rows<T, F>((const T*)src, ld, rows, cols, keep, n, q, ldq, s, lds, stream)
    if (dtype == ZR_BF16) { ZR_MX_EACH(ZR_CALL, uint16_t) }
    ZR_MX_EACH(ZR_CALL, float)
#undef ZR_CALL
}

int launch_mx_quantize_cols(const void* src, int64_t ld, int rows, int cols, const int32_t* keep, int n, int dtype, int fmt,
                            uint8_t* q, int64_t ldq, uint8_t* s, int64_t lds, hipStream_t stream)
{
#define ZR_CALL(T, F) quantize_cols<T, F>((const T*)src, ld, rows, cols, keep, n, q, ldq, s, lds, stream)
    if (dtype == ZR_BF16) { ZR_MX_EACH(ZR_CALL, uint16_t) }
    ZR_MX_EACH(ZR_CALL, float)
#undef ZR_CALL
}

int launch_mx_dequantize(const MxArg& x, int rows, int n, void* out, int64_t ldo, int width, int dtype, hipStream_t stream)
{
    const int fmt = x.fmt;
#define ZR_CALL(T, F) dequantize<T, F>(x, rows, n, (T*)out, ldo, width, stream)
    if (dtype == ZR_BF16) { ZR_MX_EACH(ZR_CALL, uint16_t) }
    ZR_MX_EACH(ZR_CALL, float)
#undef ZR_CALL
}

}  // namespace zr
