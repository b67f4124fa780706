// Values in blocks of 32 with a power of two each (E4M3, E2M1 or 8-bit integers in 64ths): what the
// translation units of the block-scaled operators share.
//
// Block b of a row holds the values 32 b .. 32 b + 31 along the contraction.  With a = max |x| over the block
//     e = the smallest integer with a <= top * 2^e, within [-127, 127];  held: rne(x * 2^-e) and e + 127
// so no value is clipped (unless e is), and each is off by at most half a step of the element's grid.  A block with
// a NaN or an infinity in it holds e + 127 = 255 and zeros: every value of it stands for NaN.
//
// A row of n values takes ceil(n / 128) * 128 elements and ceil(n / 512) * 16 scale bytes, zeros behind the n-th: whole
// steps of the matrix instruction (128 deep) and of four of them, so that no product has a tail to mask.  Block b of 16
// has its scale at byte 4 (b % 4) + b / 4: lane group g of the matrix instruction scales block g of each step, and finds
// its four scales of four successive steps in ONE dword, one byte per step, which the instruction itself picks.
#pragma once

#include "zr_common.h"

namespace zr {

struct MxArg {                  // one matrix in blocks, as the kernels take it
    const uint8_t* q;           // elements, 16-byte aligned rows
    int64_t ldq;                // bytes
    const uint8_t* s;           // scales
    int64_t lds;                // bytes
    int fmt;                    // zr_mx_format
};

inline int mx_bits(int fmt) { return fmt == ZR_MX_E2M1 ? 4 : 8; }
inline int64_t mx_row_bytes(int64_t n, int fmt) { return (n + 127) / 128 * 16 * mx_bits(fmt); }
inline int64_t mx_scale_bytes(int64_t n) { return (n + 511) / 512 * 16; }

struct MxProduct {
    MxArg X, W;                 // [M x C], [rows of W x C]
    const int32_t* w_rows;      // rows of W that are multiplied, or nullptr: all
    int w_extent;               // rows W has
    int M, J, C;                // J: rows multiplied
    void* Y;
    int64_t ldy;
    int N;                      // columns of Y (J of them results if w_rows is set)
    int dtype;                  // of Y, and of raw
    const void* prev;           // Same imputation: laid out like Y, or nullptr: +0
    // X as it arrives, quantised inside the product (few rows only), or nullptr
    const void* raw;
    int64_t ldraw;
    const int32_t* raw_cols;    // kept list on its columns, or nullptr
    int raw_extent;             // columns it has
};

int launch_mx_quantize_rows(const void* src, int64_t ld, int rows, int cols, const int32_t* keep, int n, int dtype, int fmt,
                            uint8_t* q, int64_t ldq, uint8_t* s, int64_t lds, hipStream_t stream);
int launch_mx_quantize_cols(const void* src, int64_t ld, int rows, int cols, const int32_t* keep, int n, int dtype, int fmt,
                            uint8_t* q, int64_t ldq, uint8_t* s, int64_t lds, hipStream_t stream);
// out[rows x width]: the values of each row, zeros from n to width (width <= whole steps of 128)
int launch_mx_dequantize(const MxArg& x, int rows, int n, void* out, int64_t ldo, int width, int dtype, hipStream_t stream);
int launch_mx_product(const MxProduct& p, hipStream_t stream);
constexpr int MX_FEW = 16;      // rows of X that a product quantises on its own

#ifdef __HIPCC__
// ---- device side -------------------------------------------------------------
typedef float mx_f2 __attribute__((ext_vector_type(2)));

// e + 127 for a block whose largest |x| has these bits; 255: not finite
template <int FMT> __device__ __forceinline__ int mx_code(uint32_t abits)
{
    constexpr int EMAX = FMT == ZR_MX_E4M3 ? 8 : FMT == ZR_MX_E2M1 ? 2 : 0;
    constexpr uint32_t TOP = FMT == ZR_MX_E4M3 ? 0x600000u : FMT == ZR_MX_E2M1 ? 0x400000u : 0x7e0000u;   // fraction of the largest value
    int c = (int)(abits >> 23) - EMAX + ((abits & 0x7fffffu) > TOP ? 1 : 0);
    if ((abits >> 23) == 0) c = FMT == ZR_MX_INT8 && abits > 0x7f0000u ? 1 : 0;      // subnormal a: 127/64 * 2^-127 is 0x7f0000
    c = min(max(c, 0), 254);
    return abits >= 0x7f800000u ? 255 : c;
}

// 2^-(code - 127), for codes up to 254; 2^-127 is subnormal
__device__ __forceinline__ float mx_inv(int code)
{
    return __uint_as_float(code >= 254 ? 0x00400000u : (uint32_t)(254 - code) << 23);
}

// 2^(code - 127); NaN for 255
__device__ __forceinline__ float mx_scale(int code)
{
    return __uint_as_float(code == 0 ? 0x00400000u : code == 255 ? 0x7fc00000u : (uint32_t)code << 23);
}

// Eight values of a block with this code, on the format's grid: 8 bytes, or 4 in .x
// (the conversions round to nearest even; nothing is beyond the largest value; zeros if the block is not finite)
template <int FMT> __device__ __forceinline__ uint2 mx_encode8(const float (&x)[8], int code)
{
    const float inv = mx_inv(code);
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = x[i] * inv;
    uint2 r = make_uint2(0u, 0u);
    if constexpr (FMT == ZR_MX_E4M3) {
        r.x = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
        r.x = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], r.x, true);
        r.y = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], 0, false);
        r.y = __builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], r.y, true);
    } else if constexpr (FMT == ZR_MX_E2M1) {
        r.x = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r.x, y[0], y[1], 1.f, 0);
        r.x = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r.x, y[2], y[3], 1.f, 1);
        r.x = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r.x, y[4], y[5], 1.f, 2);
        r.x = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r.x, y[6], y[7], 1.f, 3);
    } else {
        int v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = min(max((int)__builtin_rintf(y[i] * 64.f), -127), 127);
        r.x = (v[0] & 255) | (v[1] & 255) << 8 | (v[2] & 255) << 16 | (uint32_t)v[3] << 24;
        r.y = (v[4] & 255) | (v[5] & 255) << 8 | (v[6] & 255) << 16 | (uint32_t)v[7] << 24;
    }
    return code == 255 ? make_uint2(0u, 0u) : r;
}

// The eight values that mx_encode8's bytes stand for
template <int FMT> __device__ __forceinline__ void mx_decode8(uint2 r, float scale, float (&x)[8])
{
    if constexpr (FMT == ZR_MX_E4M3) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t w = h ? r.y : r.x;
            const mx_f2 a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
            x[4 * h] = a.x; x[4 * h + 1] = a.y; x[4 * h + 2] = b.x; x[4 * h + 3] = b.y;
        }
    } else if constexpr (FMT == ZR_MX_E2M1) {
        const mx_f2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(r.x, 1.f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(r.x, 1.f, 1);
        const mx_f2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(r.x, 1.f, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(r.x, 1.f, 3);
        x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y; x[4] = c.x; x[5] = c.y; x[6] = d.x; x[7] = d.y;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (float)((int)((i < 4 ? r.x : r.y) << (24 - 8 * (i & 3))) >> 24) * (1.f / 64.f);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] *= scale;
}

// the largest of four neighbouring lanes' values
__device__ __forceinline__ uint32_t mx_max4(uint32_t a)
{
    a = max(a, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)a, 0xb1, 0xf, 0xf, true));       // lanes 1 0 3 2
    return max(a, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)a, 0x4e, 0xf, 0xf, true));    // lanes 2 3 0 1
}

// What a lane reads that puts elements at .. at + PER - 1 of a row of `width` back into values (width: n, or up to the whole groups of
// 128 that the row's storage holds).  Every read lies in the row's storage, whatever `at` is: chunks that begin before the row read
// from its first element, chunks that lie behind it (the idle lanes of a row's last wavefront) from inside its last group.
// VEC: `at` is a multiple of PER.
struct MxRead {
    int e;          // the first element that is in the row
    int b;          // the byte from which PER elements' worth are read
    int more;       // (elements from odd places, 4 bits) a byte more, from here
};
template <int FMT, int PER, bool VEC> __host__ __device__ __forceinline__ MxRead mx_read_at(int at, int n, int width)
{
    const int held = (n + 127) / 128 * 128, last = VEC ? held - PER : width - 1;
    const int e = at < 0 ? 0 : at < last ? at : last;
    if constexpr (FMT == ZR_MX_E2M1) {
        const int top = (held - PER) / 2, b = e / 2 < top ? e / 2 : top, next = held / 2 - 1 - b;
        return MxRead{e, b, b + (PER / 2 < next ? PER / 2 : next)};
    }
    return MxRead{e, e < held - PER ? e : held - PER, 0};
}
// their bits from `row`, element e's first
template <int FMT, int PER, bool VEC> __host__ __device__ __forceinline__ uint2 mx_read(const uint8_t* row, MxRead a)
{
    const uint8_t* p = row + a.b;
    if constexpr (FMT == ZR_MX_E2M1) {
        uint32_t w;
        if constexpr (PER == 8) __builtin_memcpy(&w, p, 4);
        else { uint16_t h; __builtin_memcpy(&h, p, 2); w = h; }
        if constexpr (!VEC) w = (uint32_t)((w | (uint64_t)row[a.more] << (4 * PER)) >> (4 * (a.e - 2 * a.b)));     // an odd place: half a byte more
        return uint2{w, 0u};
    } else {
        uint64_t w = 0;
        __builtin_memcpy(&w, p, PER);
        if constexpr (!VEC) w >>= 8 * (a.e - a.b);
        return uint2{(uint32_t)w, (uint32_t)(w >> 32)};
    }
}
// wavefronts of 64 chunks to a row; rows that are not aligned may begin inside a chunk and so take one more
__host__ __device__ inline int mx_value_segs(int width, int per, bool vec) { return ((width + per - 1) / per + (vec ? 0 : 1) + 63) / 64; }

// byte of block b's scale in its row
__device__ __forceinline__ int mx_scale_at(int b) { return (b & ~15) + 4 * (b & 3) + ((b >> 2) & 3); }
#endif

}  // namespace zr
