// Passes over [tokens x features] around the products (gfx950): dropout, what the backward pass of a product with an activation
// does to dY before the products, and the sums over tokens that belong to both it and the norms.  HBM bound.
#include "zr_act.h"

namespace zr {

namespace {

// Threads of a workgroup over groups of eight columns and rows: `across` (a power of two) neighbours along a row.
constexpr int BACK_BLOCKS = 1024;          // workgroups of act_back_kernel, four to a compute unit
inline int lanes_across(int cols)
{
    int w = 1;
    while (w < 64 && w * 8 < cols) w *= 2;
    return w;
}

// ---------------------------------------------------------------------------
// Dropout: out = D(x).  One read, one write, one draw for eight elements: HBM bound (8192 x 4096 in bf16 25 us, 5.3 TB/s; the draws
// keep the vector units busy for 0.4 of that).
// ---------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(256) void dropout_kernel(const T* x, int64_t ldx, T* out, int64_t ldo, int rows, int cols,
                                                      const uint64_t* rng, uint32_t drop, float factor, int across, int rows_each)
{
    const int lane = threadIdx.x & (across - 1), sub = threadIdx.x / across, down = 256 / across;
    const int group = (int)blockIdx.x * across + lane, col = 8 * group;
    if (col >= cols) return;
    uint64_t seed = 0, offset = 0;
    if (drop) { seed = rng[0]; offset = rng[1]; }          // (no generator where nothing is dropped)
    const int hi = min(8, cols - col);
    const int64_t first = (int64_t)blockIdx.y * rows_each, last = min((int64_t)rows, first + rows_each);
    for (int64_t r = first + sub; r < last; r += down) {
        float v[8];
        load8(x + r * ldx + col, 0, hi, v);
        if (drop) Draw(seed, offset, (uint32_t)r, (uint32_t)group).apply(v, drop, factor);
        store8(out + r * ldo + col, 0, hi, v);
    }
}

// ---------------------------------------------------------------------------
// dZ = D(dY) gate act'(Z), dgate = D(dY) act(Z), and the column sums of dZ
// ---------------------------------------------------------------------------
// A workgroup has a panel of columns and rows_each rows; a thread's next row is on its way while it works on one.  What bounds it is
// HBM and, with an activation, the vector instructions as much: 12608 x 2048, 1638 kept, GELU, 40 to 45 us, where its 145 MB alone take 27 and
// its 36 instructions an element, two of them at a quarter of the rate, 28.
// KEPT (bf16): only the kept columns of dZ are written, side by side: a wavefront has a row's 512 columns, puts the kept
// ones into LDS at their places and stores 16 bytes a lane; the chunks that panels share go out element by element.
template <typename T, bool KEPT>
__global__ __launch_bounds__(256, 4) void act_back_kernel(const ActBack a, int across, int rows_each)
{
    constexpr int PANEL = 512, SLOTS = PANEL + 8 + 64;       // a row's panel, its place in a chunk, the zeros behind the last column
    __shared__ float sums[256 * 8];
    __shared__ uint32_t mask[KEPT ? 64 : 1];
    __shared__ __align__(16) Bf turn[KEPT ? 4 : 1][KEPT ? SLOTS + 8 : 8];
    constexpr bool EXACT = sizeof(T) == 4;
    const int lane = threadIdx.x & (across - 1), sub = threadIdx.x / across, down = 256 / across;
    const int group = (int)blockIdx.x * across + lane, col = 8 * group;
    const int hi = min(8, a.N - col);
    const int64_t first = (int64_t)blockIdx.y * rows_each, last = min((int64_t)a.M, first + rows_each);
    uint64_t seed = 0, offset = 0;
    if (a.drop) { seed = a.rng[0]; offset = a.rng[1]; }

    // KEPT: kept columns before the panel and behind it, and where this thread's eight go
    int begin = 0, end = 0, fill = 0, at[8];
    if constexpr (KEPT) {
        const int panel = (int)blockIdx.x * PANEL;
        begin = lower_bound_wave(a.keep, a.n_keep, panel, threadIdx.x & 63);
        end = panel + PANEL >= a.N ? a.n_keep : lower_bound_wave(a.keep, a.n_keep, panel + PANEL, threadIdx.x & 63);
        fill = panel + PANEL >= a.N ? a.width : end;         // (zeros behind the last kept column, to the end of the row)
        if (threadIdx.x < 64) mask[threadIdx.x] = 0u;
        __syncthreads();
        // (a list that is not ascending gives other columns, but none past the panel)
        for (int q = begin + (int)threadIdx.x; q < min(end, begin + PANEL); q += 256) {
            const int c = min(max(a.keep[q] - panel, 0), PANEL - 1);
            atomicOr(&mask[c >> 3], 1u << (c & 7));
        }
        __syncthreads();
        const uint32_t m = mask[lane];
        int before = __popc(m);
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int x = __shfl_up(before, off, 64);
            before += lane >= off ? x : 0;
        }
        before -= __popc(m);
#pragma unroll
        for (int e = 0; e < 8; ++e) at[e] = m >> e & 1 ? (begin & 7) + before + __popc(m & ((1u << e) - 1u)) : SLOTS;
        // (a slot that no column fills stays as it is: zeros)
        for (int q = (int)threadIdx.x; q < 4 * (SLOTS + 8); q += 256) turn[q / (SLOTS + 8)][q % (SLOTS + 8)] = 0;
        __syncthreads();
    }

    float total[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) total[e] = 0.f;
    const bool whole = hi == 8;
    Raw8<T> rt, rz, rg;
    rt.clear(); rz.clear(); rg.clear();
    auto fetch = [&](int64_t row) {
        const int64_t r = min(row, (int64_t)a.M - 1);
        auto one = [&](Raw8<T>& raw, const void* p, int64_t ld) {
            if (whole) {
                raw.load((const T*)p + r * ld + col);
            } else {
                float x[8];
                load8((const T*)p + r * ld + col, 0, max(hi, 0), x);
                raw.take(x);
            }
        };
        one(rt, a.dY, a.lddy);
        if (a.Z) one(rz, a.Z, a.ldz);
        if (a.gate) one(rg, a.gate, a.ldg);
    };
    if (first + sub < last) fetch(first + sub);
    for (int64_t r = first + sub; r < last; r += down) {
        float t[8], z[8], v[8], s[8], g[8];
        rt.values(t);
        if (a.Z) rz.values(z);
        if (a.gate) rg.values(g);
        fetch(r + down);
        // (the dropped ones become 0 last: nothing of dY, Z or gate at their places reaches a gradient)
        uint32_t kept = 0xffu;
        if (a.drop) {
            kept = Draw(seed, offset, (uint32_t)r, (uint32_t)group).bits(a.drop);
#pragma unroll
            for (int e = 0; e < 8; ++e) t[e] *= a.factor;
        }
        auto drop = [&](float (&x)[8]) {
            if (!a.drop) return;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = kept >> e & 1 ? x[e] : 0.f;
        };
        if (a.Z) {
            act8<EXACT, true>(a.act, z, v, s);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) { v[e] = 0.f; s[e] = 1.f; }
        }
        if (a.gate) {
#pragma unroll
            for (int e = 0; e < 8; ++e) s[e] *= g[e];
        }
        if (a.dgate && hi > 0) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] *= t[e];
            drop(v);
            store8((T*)a.dgate + r * a.lddg + col, 0, hi, v);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] *= s[e];
        drop(t);
#pragma unroll
        for (int e = 0; e < 8; ++e) total[e] += t[e];
        if constexpr (KEPT) {
            Bf* slots = turn[sub];
            Bf* row = (Bf*)a.dz + r * a.lddz + (begin & ~7);
            Raw8<Bf> raw;
            raw.take(t);
#pragma unroll
            for (int e = 0; e < 8; ++e) slots[at[e]] = (Bf)(e & 1 ? raw.v[e >> 1] >> 16 : raw.v[e >> 1]);
            // (a wavefront's LDS operations are done in their order)
            __builtin_amdgcn_wave_barrier();
            // whole chunks from the first slot on; slot 0 is column begin & ~7
            const int lo = begin & 7, top = min(fill - (begin & ~7), SLOTS);
            for (int c = (lo + 7) / 8 + lane; c < top / 8; c += 64) *(u4*)(row + 8 * c) = *(const u4*)(slots + 8 * c);
            const int part = lane < 8 ? lane : top / 8 * 8 + (lane - 8);
            const bool in_first = lane < 8 && part >= lo && part < top && lo > 0;
            const bool in_last = lane >= 8 && lane < 16 && part < top && (top / 8 > 0 || lo == 0);
            if (in_first || in_last) row[part] = slots[part];
            __builtin_amdgcn_wave_barrier();
        } else {
            if (a.dz && hi > 0) store8((T*)a.dz + r * a.lddz + col, 0, hi, t);
        }
    }
    if (!a.partial) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[(sub * across + lane) * 8 + e] = total[e];
    __syncthreads();
    float* dst = a.partial + (size_t)blockIdx.y * (size_t)a.N;
    for (int q = threadIdx.x; q < across * 8; q += 256) {
        const int c = (int)blockIdx.x * across * 8 + q;
        if (c >= a.N) continue;
        float v = 0.f;
        for (int i = 0; i < down; ++i) v += sums[i * across * 8 + q];
        dst[c] = v;
    }
}

// ---------------------------------------------------------------------------
// Sums over slabs: 64 columns to a workgroup, sixteen wavefronts along the slabs, eight loads of each on their way, added in a fixed
// order.  Latency bound: 2.4 to 5 us.
// ---------------------------------------------------------------------------
constexpr int SLAB_WAVES = 16;
// of this wavefront's slabs; column c below n
__device__ __forceinline__ float slab_sum(const float* p, int slabs, int n, int c, int wave)
{
    constexpr int W = SLAB_WAVES, U = 8;
    float v = 0.f;
    for (int s = wave; s < slabs; s += W * U) {
        float x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = p[(size_t)min(s + W * u, slabs - 1) * (size_t)n + c];
#pragma unroll
        for (int u = 0; u < U; ++u) v += s + W * u < slabs ? x[u] : 0.f;
    }
    return v;
}

template <typename T>
__global__ __launch_bounds__(1024) void sum_slabs_kernel(const float* partial, int slabs, int n, T* out)
{
    __shared__ float part[SLAB_WAVES][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = (int)blockIdx.x * 64 + lane;
    part[wave][lane] = slab_sum(partial, slabs, n, min(c, n - 1), wave);
    __syncthreads();
    if (wave == 0 && c < n) {
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < SLAB_WAVES; ++w) sum += part[w][lane];
        put_one(out + c, sum);
    }
}

// The gradients of a join's vectors, one to a row of the grid: one of the sums, or of SUM_DT and SUM_D with scale and
//   dgate = scale (post_w sum d t + post_b sum d),  dpost_w = scale gate sum d t,  dpost_b = scale gate sum d
template <typename T>
__global__ __launch_bounds__(1024) void join_sums_kernel(const Join j)
{
    __shared__ float part[2][SLAB_WAVES][64];
    const int which = blockIdx.y;
    void* out = j.vectors[0];
    int first = SUM_DY;
    const void* weight = nullptr;
    if (which == 1) { out = j.vectors[1]; first = SUM_DT; weight = j.post ? j.post_w : nullptr; }
    if (which == 2) { out = j.vectors[2]; first = SUM_DT; weight = j.gate; }
    if (which == 3) { out = j.vectors[3]; first = SUM_D; weight = j.gate; }
    if (which == 4) { out = j.vectors[4]; first = SUM_HAT; }
    if (which == 5) { out = j.vectors[5]; first = SUM_DH; }
    if (!out) return;
    const bool both = which == 1 && j.post && j.post_b;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = (int)blockIdx.x * 64 + lane, at = min(c, j.cols - 1);
    const size_t size = (size_t)j.slabs * (size_t)j.cols;
    float w = which >= 1 && which <= 3 ? j.scale : 1.f, w2 = j.scale;
    if (weight) w *= one_of((const T*)weight + at);
    if (both) w2 *= one_of((const T*)j.post_b + at);
    part[0][wave][lane] = slab_sum(j.partial + size * (size_t)first, j.slabs, j.cols, at, wave);
    if (both) part[1][wave][lane] = slab_sum(j.partial + size * (size_t)SUM_D, j.slabs, j.cols, at, wave);
    __syncthreads();
    if (wave == 0 && c < j.cols) {
        float sum = 0.f, sum2 = 0.f;
#pragma unroll
        for (int i = 0; i < SLAB_WAVES; ++i) {
            sum += part[0][i][lane];
            if (both) sum2 += part[1][i][lane];
        }
        sum *= w;
        if (both) sum = fmaf(w2, sum2, sum);
        put_one((T*)out + c, sum);
    }
}

}  // namespace

int launch_dropout(const void* x, int64_t ldx, void* out, int64_t ldo, int rows, int cols, const uint64_t* rng, uint32_t drop,
                   float factor, int dtype, hipStream_t stream)
{
    const int across = lanes_across(cols), down = 256 / across;
    const int wide = (cols + 8 * across - 1) / (8 * across);
    // 2048 workgroups and more where there is work for them, at least one row a thread
    const int64_t most = std::max<int64_t>(1, 4096 / wide);
    const int rows_each = (int)std::max<int64_t>(down, (rows + most - 1) / most);
    const dim3 grid((unsigned)wide, (unsigned)((rows + (int64_t)rows_each - 1) / rows_each));
    if (dtype == ZR_BF16)
        hipLaunchKernelGGL(dropout_kernel<Bf>, grid, dim3(256), 0, stream, (const Bf*)x, ldx, (Bf*)out, ldo, rows, cols, rng, drop, factor, across, rows_each);
    else
        hipLaunchKernelGGL(dropout_kernel<float>, grid, dim3(256), 0, stream, (const float*)x, ldx, (float*)out, ldo, rows, cols, rng, drop, factor, across, rows_each);
    return hip_status(hipGetLastError());
}

// rows that a workgroup of act_back_kernel takes
static int back_rows_each(int M, int N)
{
    const int across = lanes_across(N), down = 256 / across;
    const int wide = (N + 8 * across - 1) / (8 * across);
    const int most = std::max(1, std::min(512, BACK_BLOCKS / wide));
    return std::max(down, (M + most - 1) / most);
}
int act_slabs(int M, int N)
{
    const int each = back_rows_each(M, N);
    return (int)(((int64_t)M + each - 1) / each);
}

int launch_act_back(const ActBack& a, int dtype, hipStream_t stream)
{
    const int across = lanes_across(a.N);
    const dim3 grid((unsigned)((a.N + 8 * across - 1) / (8 * across)), (unsigned)act_slabs(a.M, a.N));
    const int each = back_rows_each(a.M, a.N);
    if (dtype == ZR_F32) hipLaunchKernelGGL((act_back_kernel<float, false>), grid, dim3(256), 0, stream, a, across, each);
    else if (a.keep) hipLaunchKernelGGL((act_back_kernel<Bf, true>), grid, dim3(256), 0, stream, a, across, each);
    else hipLaunchKernelGGL((act_back_kernel<Bf, false>), grid, dim3(256), 0, stream, a, across, each);
    return hip_status(hipGetLastError());
}

int launch_sum_slabs(const float* partial, int slabs, int n, void* out, int dtype, hipStream_t stream)
{
    const dim3 grid((unsigned)((n + 63) / 64));
    if (dtype == ZR_BF16) hipLaunchKernelGGL(sum_slabs_kernel<Bf>, grid, dim3(64 * SLAB_WAVES), 0, stream, partial, slabs, n, (Bf*)out);
    else hipLaunchKernelGGL(sum_slabs_kernel<float>, grid, dim3(64 * SLAB_WAVES), 0, stream, partial, slabs, n, (float*)out);
    return hip_status(hipGetLastError());
}

int launch_join_sums(const Join& j, int dtype, hipStream_t stream)
{
    const dim3 grid((unsigned)((j.cols + 63) / 64), 6);
    if (dtype == ZR_BF16) hipLaunchKernelGGL(join_sums_kernel<Bf>, grid, dim3(64 * SLAB_WAVES), 0, stream, j);
    else hipLaunchKernelGGL(join_sums_kernel<float>, grid, dim3(64 * SLAB_WAVES), 0, stream, j);
    return hip_status(hipGetLastError());
}

}  // namespace zr
