// Drives the C entry points of the block-scaled operators (zr_mx_api.hip, with zr_api.hip for the backward products) on the
// CPU under AddressSanitizer and UndefinedBehaviorSanitizer.  The launchers are stand-ins that check what the kernels
// rely on, among it that nothing they are handed reaches past the buffers of the call.
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "zr_mx.h"

namespace zr {
extern int g_launches;
extern const char* g_ws_begin;
extern const char* g_ws_end;

static void require(bool ok, const char* what)
{
    if (!ok) { fprintf(stderr, "mx stub invariant violated: %s\n", what); abort(); }
}
// where the call under test may write elements / scales, and how much room there is
static const char *g_q = nullptr, *g_s = nullptr;
static size_t g_q_bytes = 0, g_s_bytes = 0;

static void check_storage(const uint8_t* q, int64_t ldq, const uint8_t* s, int64_t lds, int64_t rows, int64_t n, int fmt)
{
    require((uintptr_t)q % 16 == 0 && (uintptr_t)s % 16 == 0 && ldq % 16 == 0 && lds % 16 == 0, "alignment of a stored matrix");
    require(ldq >= (n + 127) / 128 * (fmt == ZR_MX_E2M1 ? 64 : 128) && lds >= (n + 511) / 512 * 16, "pitch of a stored matrix");
    if ((const char*)q == g_q) require((size_t)(rows - 1) * ldq + (size_t)mx_row_bytes(n, fmt) <= g_q_bytes, "elements past their buffer");
    if ((const char*)s == g_s) require((size_t)(rows - 1) * lds + (size_t)mx_scale_bytes(n) <= g_s_bytes, "scales past their buffer");
}

int launch_mx_quantize_rows(const void* src, int64_t ld, int rows, int cols, const int32_t* keep, int n, int, int fmt, uint8_t* q, int64_t ldq, uint8_t* s,
                            int64_t lds, hipStream_t)
{
    ++g_launches;
    require(src && ld >= cols && n >= 1 && n <= cols && (keep || n == cols), "rows into blocks");
    check_storage(q, ldq, s, lds, rows, n, fmt);
    return ZR_OK;
}
int launch_mx_quantize_cols(const void* src, int64_t ld, int rows, int cols, const int32_t* keep, int n, int, int fmt, uint8_t* q, int64_t ldq, uint8_t* s,
                            int64_t lds, hipStream_t)
{
    ++g_launches;
    require(src && ld >= cols && n >= 1 && n <= rows && (keep || n == rows), "columns into blocks");
    check_storage(q, ldq, s, lds, cols, n, fmt);
    return ZR_OK;
}
int launch_mx_dequantize(const MxArg& x, int rows, int n, void* out, int64_t ldo, int width, int dtype, hipStream_t)
{
    ++g_launches;
    check_storage(x.q, x.ldq, x.s, x.lds, rows, n, x.fmt);
    require(out && width >= n && width <= (n + 127) / 128 * 128 && ldo >= width, "values");
    if ((const char*)out == g_ws_begin)
        require(g_ws_begin + (size_t)rows * ldo * (dtype == ZR_BF16 ? 2 : 4) <= g_ws_end, "values past the workspace");
    return ZR_OK;
}
int launch_mx_product(const MxProduct& p, hipStream_t)
{
    ++g_launches;
    require(p.M >= 1 && p.J >= 1 && p.C >= 1 && p.Y && p.ldy >= p.N, "product extents");
    require(p.w_rows ? p.J < p.N && p.w_extent == p.N : p.J == p.N, "rows of the weight");
    require(!p.prev || p.w_rows, "previous values without a scatter");
    check_storage(p.W.q, p.W.ldq, p.W.s, p.W.lds, p.w_extent, p.C, p.W.fmt);
    if (p.raw) require(p.M <= MX_FEW && p.ldraw >= p.raw_extent && p.C <= p.raw_extent && (p.raw_cols || p.C == p.raw_extent), "raw input");
    else check_storage(p.X.q, p.X.ldq, p.X.s, p.X.lds, p.M, p.C, p.X.fmt);
    return ZR_OK;
}
}  // namespace zr

using namespace zr;

int main()
{
    std::mt19937 rng(7);
    auto pick = [&](int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); };
    std::vector<char> room((size_t)1 << 20);
    char* p = (char*)(((uintptr_t)room.data() + 255) / 256 * 256);
    const size_t ws_room = (size_t)80 << 20;
    char* ws = (char*)aligned_alloc(256, ws_room);       // never touched, only measured
    int refused = 0, done = 0;
    for (int it = 0; it < 200000; ++it) {
        const int M = pick(0, 40), K = pick(0, 700), N = pick(0, 300), mode = pick(0, 1), dtype = pick(0, 1), policy = pick(0, 2), layout = pick(0, 1);
        const int len = mode == ZR_DROP_N ? N : K, n_keep = pick(0, 9) ? (len ? pick(1, len) : 0) : len + 1;
        const bool list = pick(0, 3) != 0;
        const int held = mode == ZR_DROP_K && list ? n_keep : K;
        const int xf = pick(0, 3), wf = pick(0, 3);
        const int64_t ldq = (int64_t)zr_mx_row_bytes(held, xf) + 16 * pick(-1, 2), lds = (int64_t)zr_mx_scale_bytes(held) + 16 * pick(-1, 2) * (pick(0, 3) == 0);
        const int64_t ldwq = (int64_t)zr_mx_row_bytes(held, wf), ldws = (int64_t)zr_mx_scale_bytes(held);
        g_q = p + 4096; g_s = p + 8192;
        g_q_bytes = M > 0 && ldq > 0 ? (size_t)M * ldq : 0; g_s_bytes = M > 0 && lds > 0 ? (size_t)M * lds : 0;
        const int before = g_launches;
        int st;
        if (it % 3 == 0) {
            const int axis = pick(0, 1);
            const int rows = axis ? M : K, cols = axis ? K : M, nk = list ? n_keep : K;
            const int64_t a = (int64_t)zr_mx_row_bytes(nk, xf) + 16 * pick(-1, 1), b = (int64_t)zr_mx_scale_bytes(nk);
            g_q_bytes = M > 0 && a > 0 ? (size_t)M * a : 0; g_s_bytes = M > 0 ? (size_t)M * b : 0;
            st = zr_mx_quantize(p, cols + pick(-1, 3), rows, cols, axis, list ? (const int32_t*)p : nullptr, nk, dtype, xf, p + 4096, a, p + 8192, b, nullptr);
        } else if (it % 3 == 1) {
            const bool raw = pick(0, 1), keep_q = !raw || pick(0, 1);
            st = zr_mx_linear_fwd(raw ? p : nullptr, K + pick(0, 2), keep_q ? p + 4096 : nullptr, ldq, keep_q ? p + 8192 : nullptr, lds, xf, p + 12288, ldwq,
                                  p + 16384, ldws, wf, p + 20480, N + pick(-1, 3), M, K, N, list ? (const int32_t*)p : nullptr, n_keep, mode, dtype, policy,
                                  pick(0, 1) ? p : nullptr, nullptr);
        } else {
            const size_t need = zr_mx_bwd_workspace_bytes(M, K, N, n_keep, mode, dtype);
            const size_t bytes = need ? need / (size_t)pick(1, 3) : 0;
            require(bytes + 64 <= ws_room, "room for the largest workspace");
            char* w = ws + (pick(0, 20) ? 0 : 8);
            g_ws_begin = w; g_ws_end = w + bytes;
            const bool dx = pick(0, 3) != 0, dw = pick(0, 3) != 0;
            const int64_t lw = layout == ZR_W_KN ? N : K;
            st = zr_resized_linear_bwd_mx(p + 4096, ldq, p + 8192, lds, xf, p + 65536, lw, p + 131072, N, dx ? p + 262144 : nullptr, K, dw ? p + 393216 : nullptr, lw,
                                          M, K, N, (const int32_t*)p, n_keep, mode, layout, dtype, policy, pick(0, 1) ? p : nullptr, pick(0, 1) ? p : nullptr,
                                          pick(0, 9) ? w : nullptr, bytes, nullptr);
        }
        if (st != ZR_OK) { require(g_launches == before, "a refused call enqueued work"); ++refused; }
        else { require(g_launches > before, "an accepted call enqueued nothing"); ++done; }
    }
    require(refused > 10000 && done > 10000, "both kinds of calls");
    printf("OK %d done, %d refused\n", done, refused);
    free(ws);
    return 0;
}
