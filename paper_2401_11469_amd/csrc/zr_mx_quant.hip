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
    const int c = mx_code<FMT>(mx_max4(a));
    const int at = seg * SEG + 8 * lane;
    if (at < (n + 127) / 128 * 128) {
        const uint2 e = mx_encode8<FMT>(x, c);
        if constexpr (FMT == ZR_MX_E2M1) *(uint32_t*)(q + at / 2) = e.x;
        else *(uint2*)(q + at) = e;
    }
    if ((lane & 3) == 0) s[mx_scale_at(seg * 16 + (lane >> 2))] = at < n ? c : 0;
}

// Rows of 16-byte loads, nothing gathered: a wavefront takes a segment of four rows, all requested together.
// (bf16 8192 x 4096 into 8 bits 19.4 us, 5.2 TB/s of what is read and written, the rate of a copy; into 4 bits 17.7)
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

// Rows of any alignment, and gathered columns: up to RB whole rows come into LDS in aligned 16-byte chunks, KL to a thread
// (what lies before the first and behind the last whole chunk of a row by elements, one to a thread), the list beside them in 16
// bits; all of it is requested at once.  The wavefronts then share out the segments of all rows.  ODD: some row does not begin and
// end on 16-byte addresses (false is a variant for speed alone: 17.4 us against 19.6 at the size below).
// (bf16 8192 x 2752, 2064 kept, into 8 bits: 17.4 us, 3.6 TB/s; 46 with the list read from memory by every lane.  A copy would
// take 12; bound by the vector instructions, 200 for 8 values of a lane, and the 2-byte LDS reads, half of them bank conflicts)
template <class T, int FMT, int KL, int RB, bool ODD>
__global__ __launch_bounds__(256) void mx_gather_kernel(const T* __restrict__ src, int64_t ld, int rows, int cols, const int32_t* __restrict__ keep,
                                                        int n, int segs, int rb, int pitch, uint8_t* __restrict__ q, int64_t ldq,
                                                        uint8_t* __restrict__ s, int64_t lds)
{
    extern __shared__ __align__(16) uint8_t stage[];
    constexpr int ES = sizeof(T), PER = 16 / ES;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int r0 = blockIdx.x * rb, nr = min(rb, rows - r0);
    uint16_t* list = (uint16_t*)(stage + rb * pitch);
    auto offset = [&](int r) { return ODD ? (int)((uintptr_t)(src + (size_t)(r0 + r) * (size_t)ld) & 15) / ES : 0; };    // elements behind an aligned address
    uint4 v[RB][KL];
    T edge[RB];
    // threads 0 .. PER - 1: the elements before the first whole chunk; PER .. 2 PER - 1: behind the last
    auto edge_at = [&](int off) {
        const int head = min(off ? PER - off : 0, cols), tail = head + (cols - head) / PER * PER;
        const int e = tid < PER ? tid : tail + tid - PER;
        return tid < PER ? (e < head ? e : -1) : (tid < 2 * PER && e < cols ? e : -1);
    };
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        const T* row = src + (size_t)(r0 + min(r, nr - 1)) * (size_t)ld;
        const int off = offset(min(r, nr - 1));
#pragma unroll
        for (int k = 0; k < KL; ++k) {
            const int e = (tid + 256 * k) * PER - off;
            v[r][k] = make_uint4(0u, 0u, 0u, 0u);
            if (r < nr && e >= 0 && e + PER <= cols) v[r][k] = *(const uint4*)(row + e);
        }
        if constexpr (ODD) {
            const int e = edge_at(off);
            edge[r] = T(0);
            if (r < nr && e >= 0) edge[r] = row[e];
        }
    }
    if (keep)
        for (int i0 = 0; i0 < n; i0 += 1024) {
            int k[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) k[u] = keep[min(i0 + u * 256 + tid, n - 1)];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (i0 + u * 256 + tid < ((n + 7) & ~7)) list[i0 + u * 256 + tid] = (uint16_t)clamp_idx(k[u], cols);
        }
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        uint8_t* dst = stage + r * pitch;
        const int off = offset(min(r, nr - 1));
#pragma unroll
        for (int k = 0; k < KL; ++k) {
            const int e = (tid + 256 * k) * PER - off;
            if (r < nr && e >= 0 && e + PER <= cols) *(uint4*)(dst + (tid + 256 * k) * 16) = v[r][k];
        }
        if constexpr (ODD) {
            const int e = edge_at(off);
            if (r < nr && e >= 0) *(T*)(dst + (off + e) * ES) = edge[r];
        }
    }
    __syncthreads();
    // items (segment, row) in this order, a quarter to each wavefront: where a lane finds its 8 values is looked up once a segment
    const int items = nr * segs, lo = items * wave / 4, hi = items * (wave + 1) / 4;
    int seg = lo / nr, r = lo - seg * nr;
    int pick[8];
    for (int it = lo; it < hi; ++it) {
        const int at = seg * SEG + 8 * lane;
        if (it == lo || r == 0) {
            if (keep) {
                const uint4 p = *(const uint4*)(list + min(at, (n - 1) & ~7));
                const uint32_t w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
                for (int i = 0; i < 8; ++i) pick[i] = (w[i >> 1] >> (16 * (i & 1))) & 0xffffu;
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) pick[i] = min(at + i, n - 1);
            }
        }
        const size_t row = (size_t)(r0 + r);
        const T* d = (const T*)(stage + r * pitch) + offset(r);
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = as_float(d[pick[i]]);
        if (at + 8 > n) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = at + i < n ? x[i] : 0.f;
        }
        store_seg<FMT>(x, q + row * (size_t)ldq, s + row * (size_t)lds, n, seg, lane);
        if (++r == nr) { r = 0; ++seg; }
    }
}

// Rows too long for LDS that are gathered or of any alignment: element by element, a segment of a row at a time.  The one kernel here
// whose lanes can outnumber what a launch can have (32 bits of them: 34 G values, 69 GB; the others' 4 rows a wavefront would be
// 275 GB): the wavefronts of at most LONG_BLOCKS workgroups take turns.
constexpr int64_t LONG_BLOCKS = 1 << 22;
template <class T, int FMT>
__global__ __launch_bounds__(256) void mx_long_kernel(const T* __restrict__ src, int64_t ld, int rows, int cols, const int32_t* __restrict__ keep,
                                                      int n, int segs, uint8_t* __restrict__ q, int64_t ldq, uint8_t* __restrict__ s, int64_t lds)
{
    const int lane = threadIdx.x & 63;
    const int64_t items = (int64_t)rows * segs;
    for (int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); item < items; item += (int64_t)gridDim.x * 4) {
        const int r = (int)(item / segs), seg = (int)(item % segs);
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
}

// Blocks along the strided axis: a tile of 128 (kept) rows x 64 columns comes into LDS; each thread then takes one block of
// one column (its lanes 64 neighbouring columns: no bank conflicts, no exchange between lanes), and the elements go through
// LDS once more, so that each column's 64 or 128 bytes leave together.
// (bf16 2752 x 4096, 2064 rows kept, into 8 bits 7.2 us, 3.6 TB/s; fp32 4096 x 11008 36.4 us, 6.2 TB/s.  Rows of 4097 12.4 us: 64 columns lie
// in nine chunks of two cache lines and not in eight of one, 45 % more requests and 1.8 times the vector instructions; wavefronts wait for memory
// 72 % of the time, 67 where rows are aligned.)
template <class T, int FMT, bool VEC>
__global__ __launch_bounds__(256) void mx_cols_kernel(const T* __restrict__ src, int64_t ld, int rows, int cols, const int32_t* __restrict__ keep,
                                                      int n, uint8_t* __restrict__ q, int64_t ldq, uint8_t* __restrict__ s, int64_t lds)
{
    // (rows of any alignment: one chunk more of each, whose column c lies `shift` of its row further on)
    constexpr int KT = 128, CT = 64, PER = 16 / (int)sizeof(T), PITCH = CT + PER * (VEC ? 1 : 2);
    constexpr int OB = FMT == ZR_MX_E2M1 ? 64 : 128, OP = OB + 16;       // bytes of a column's elements in a tile
    __shared__ __align__(16) T tile[KT * PITCH];
    __shared__ __align__(16) uint8_t outs[CT * OP];
    __shared__ uint8_t shift[VEC ? 1 : KT];
    const int tid = threadIdx.x;
    const int c0 = blockIdx.x * CT, k0 = blockIdx.y * KT;
    auto row_at = [&](int k) {
        k = min(k, n - 1);
        return src + (size_t)(keep ? clamp_idx(keep[k], rows) : k) * (size_t)ld;
    };
    if constexpr (VEC) {
        constexpr int LPR = CT / PER, RPP = 256 / LPR, PASSES = KT / RPP;
        uint4 v[PASSES];
#pragma unroll
        for (int p = 0; p < PASSES; ++p)
            v[p] = *(const uint4*)(row_at(k0 + p * RPP + tid / LPR) + min(c0 + tid % LPR * PER, cols - PER));     // cols is a multiple of PER here
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            const int k = p * RPP + tid / LPR;
            *(uint4*)(tile + k * PITCH + tid % LPR * PER) = k0 + k < n ? v[p] : make_uint4(0u, 0u, 0u, 0u);
        }
    } else {
        constexpr int CH = CT / PER + 1, PASSES = (KT * CH + 255) / 256;
        uint4 v[PASSES];
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            const int u = p * 256 + tid, k = min(u / CH, KT - 1);
            const T* row = row_at(k0 + k) + c0;
            const int off = (int)((uintptr_t)row & 15) / (int)sizeof(T), e = u % CH * PER - off;       // columns c0 + e ..
            v[p] = make_uint4(0u, 0u, 0u, 0u);
            if (c0 + e >= 0 && c0 + e + PER <= cols) v[p] = *(const uint4*)(row + e);
            else {                                                    // a row's first or last columns
                union { uint4 w; T t[PER]; } x;
                x.w = v[p];
#pragma unroll
                for (int i = 0; i < PER; ++i)
                    if (c0 + e + i >= 0 && c0 + e + i < cols) x.t[i] = row[e + i];
                v[p] = x.w;
            }
            if (u % CH == 0) shift[k] = (uint8_t)off;
        }
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            const int u = p * 256 + tid, k = u / CH;
            if (k < KT) *(uint4*)(tile + k * PITCH + u % CH * PER) = k0 + k < n ? v[p] : make_uint4(0u, 0u, 0u, 0u);
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
            x[o][i] = as_float(tile[(blk * 32 + o * 8 + i) * PITCH + (VEC ? 0 : shift[VEC ? 0 : blk * 32 + o * 8 + i]) + col]);
            a = max(a, __float_as_uint(x[o][i]) & 0x7fffffffu);
        }
    const int code = mx_code<FMT>(a);
#pragma unroll
    for (int o = 0; o < 4; ++o) {
        const uint2 e = mx_encode8<FMT>(x[o], code);
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

__device__ __forceinline__ uint32_t out_bits(float v, uint16_t) { return f32_to_bf16_bits(v); }
__device__ __forceinline__ uint32_t out_bits(float v, float) { return __float_as_uint(v); }

// Blocks back into values.  A lane stores an aligned chunk of 16 bytes of a row, of four rows at a time; in a row that does not
// begin on such an address, it is the elements that are read from odd places (a chunk may then lie in two blocks).
// (8192 x 4096 into bf16 18 us, 5.6 TB/s; 16384 x 12288 from 4 bits into fp32 167 us, 5.5 TB/s; rows of 2751 21 us)
template <class T, int FMT, bool VEC>
__global__ __launch_bounds__(256) void mx_values_kernel(const uint8_t* __restrict__ q, int64_t ldq, const uint8_t* __restrict__ s, int64_t lds,
                                                        int rows, int n, int segs, T* __restrict__ out, int64_t ldo, int width)
{
    constexpr int RB = 4, PER = 16 / (int)sizeof(T);
    const int lane = threadIdx.x & 63;
    const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int r0 = (int)(item / segs) * RB, chunk = (int)(item % segs) * 64 + lane;
    if (r0 >= rows) return;
    uint2 raw[RB];
    int c0[RB], c1[RB], at[RB];
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        const size_t row = (size_t)min(r0 + r, rows - 1);
        const int off = VEC ? 0 : (int)((uintptr_t)(out + row * (size_t)ldo) & 15) / (int)sizeof(T);
        at[r] = chunk * PER - off;
        const MxRead a = mx_read_at<FMT, PER, VEC>(at[r], n, width);
        const int e = a.e;
        raw[r] = mx_read<FMT, PER, VEC>(q + row * (size_t)ldq, a);
        const uint8_t* sr = s + row * (size_t)lds;
        c0[r] = sr[mx_scale_at(e >> 5)];
        c1[r] = VEC ? c0[r] : sr[mx_scale_at(min(e + PER - 1, width - 1) >> 5)];
    }
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        if (r0 + r >= rows) break;
        const int e = mx_read_at<FMT, PER, VEC>(at[r], n, width).e;
        float x[8];
        mx_decode8<FMT>(raw[r], 1.f, x);        // (PER of them)
        T* o = out + (size_t)(r0 + r) * (size_t)ldo;
        uint32_t w[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const float v = x[i] * mx_scale(VEC || (e & 31) + i < 32 ? c0[r] : c1[r]);
            w[i] = out_bits(e + i < n ? v : 0.f, T());
        }
        if (at[r] >= 0 && at[r] + PER <= width) {
            if constexpr (PER == 8) *(uint4*)(o + at[r]) = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
            else *(uint4*)(o + at[r]) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if (e + i >= at[r] && e + i < min(at[r] + PER, width)) {
                    if constexpr (PER == 8) o[e + i] = (uint16_t)w[i];
                    else o[e + i] = __uint_as_float(w[i]);
                }
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
    const bool odd = (uintptr_t)src % 16 != 0 || ld * es % 16 != 0 || cols * es % 16 != 0;
    const int pitch = odd ? (cols * es + 15 + 15) / 16 * 16 : cols * es, chunks = pitch / 16, list = keep ? (n + 7) / 8 * 16 : 0;
    if (pitch + list <= 64 * 1024) {
        // Rows to a workgroup: short ones up to four, where a thousand workgroups remain; long ones alone, of which the LDS holds more
        // workgroups.  bf16 into 8 bits, one row to a workgroup and four: 8192 x 1000, 750 kept, 9.7 and 7.0 us; 4096 x 2752 of 2064 11.5 and
        // 9.5; 197 x 256 of 192 2.7 and 2.9; 1500 x 1000 of 750 3.7 and 3.7.  One and two: 8192 x 8000 of 6000 45 and 50, 2048 x 8000 15.1 and
        // 16.7, 8192 x 11008 of 8256 73 and 87 (the least to gain: fp32 2048 x 4000 of 3000 10.5 and 9.5).  Chunks a thread: as few as hold the row (8192 x 2752 in two 17.6, in four 18.2; 8192 x 8000
        // in four 45.3, in eight 46.1; 8192 x 11008 in eight 72.9, in sixteen 74.8); single short rows in two (2.5 us in one, 2.7).
        const int rb = std::max(1, std::min({chunks <= 512 ? 4 : 1, (64 * 1024 - list) / pitch, rows / 1024}));
#define ZR_GATHER_AS(KL, RB, ODD)                                                                                                              \
        hipLaunchKernelGGL((mx_gather_kernel<T, FMT, KL, RB, ODD>), dim3((rows + rb - 1) / rb), dim3(256), (size_t)rb * pitch + list, stream, src, ld, rows, \
                           cols, keep, n, segs, rb, pitch, q, ldq, s, lds)
#define ZR_GATHER(KL, RB) do { if (odd) ZR_GATHER_AS(KL, RB, true); else ZR_GATHER_AS(KL, RB, false); } while (0)
        if (chunks <= 512) {
            if (rb == 1) ZR_GATHER(2, 1); else if (chunks <= 256) ZR_GATHER(1, 4); else ZR_GATHER(2, 4);
        } else if (chunks <= 1024) ZR_GATHER(4, 1); else if (chunks <= 2048) ZR_GATHER(8, 1); else ZR_GATHER(16, 1);
#undef ZR_GATHER_AS
#undef ZR_GATHER
        return hip_status(hipGetLastError());
    }
    const int64_t waves = (int64_t)rows * segs;
    hipLaunchKernelGGL((mx_long_kernel<T, FMT>), dim3((uint32_t)std::min((waves + 3) / 4, LONG_BLOCKS)), dim3(256), 0, stream, src, ld, rows, cols, keep, n, segs, q, ldq, s, lds);
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
    constexpr int PER = 16 / (int)sizeof(T);
    const bool vec = (uintptr_t)out % 16 == 0 && ldo % PER == 0;
    const int segs = mx_value_segs(width, PER, vec);
    const int64_t waves = (int64_t)((rows + 3) / 4) * segs;
    const dim3 grid((uint32_t)((waves + 3) / 4));
    if (vec) hipLaunchKernelGGL((mx_values_kernel<T, FMT, true>), grid, dim3(256), 0, stream, x.q, x.ldq, x.s, x.lds, rows, n, segs, out, ldo, width);
    else hipLaunchKernelGGL((mx_values_kernel<T, FMT, false>), grid, dim3(256), 0, stream, x.q, x.ldq, x.s, x.lds, rows, n, segs, out, ldo, width);
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
