// C ABI of the block-scaled operators: argument checks and the mapping onto their kernels (zr_mx.h) and onto the
// resized layer's backward products.
#include "zr_mx.h"

using namespace zr;

namespace {

constexpr int32_t kMaxExtent = 65535 * 32;      // as for the other calls

bool valid_format(int f) { return f == ZR_MX_E4M3 || f == ZR_MX_E2M1 || f == ZR_MX_INT8; }
bool valid_dtype(int dt) { return dt == ZR_F32 || dt == ZR_BF16; }
size_t size_of(int dtype) { return dtype == ZR_BF16 ? 2 : 4; }
bool off_element(const void* p, int dtype) { return (uintptr_t)p % size_of(dtype) != 0; }

// storage of a matrix in blocks, n values a row
bool bad_storage(const void* q, int64_t ldq, const void* s, int64_t lds, int32_t n, int format)
{
    return (uintptr_t)q % 16 != 0 || (uintptr_t)s % 16 != 0 || ldq % 16 != 0 || lds % 16 != 0 ||
           ldq < mx_row_bytes(n, format) || lds < mx_scale_bytes(n);
}

int64_t round_up64(int64_t v) { return (v + 63) / 64 * 64; }

// columns that the checkpoint of the layer's input holds
int32_t held_columns(int32_t K, int32_t n_keep, int mode) { return mode == ZR_DROP_K ? n_keep : K; }
size_t values_bytes(int32_t M, int32_t held, int dtype) { return (size_t)M * (size_t)round_up64(held) * size_of(dtype); }

}  // namespace

extern "C" {

size_t zr_mx_row_bytes(int32_t n, int format) { return n < 1 || !valid_format(format) ? 0 : (size_t)mx_row_bytes(n, format); }
size_t zr_mx_scale_bytes(int32_t n) { return n < 1 ? 0 : (size_t)mx_scale_bytes(n); }

int zr_mx_quantize(const void* src, int64_t ld, int32_t rows, int32_t cols, int axis, const int32_t* keep_idx, int32_t n_keep,
                   int dtype, int format, void* q, int64_t ldq, void* scales, int64_t lds, void* stream)
{
    if (!src || !q || !scales) return ZR_ERR_NULL;
    if (!valid_dtype(dtype) || !valid_format(format)) return ZR_ERR_DTYPE;
    if (rows < 1 || cols < 1 || ld < cols || (axis != 0 && axis != 1) || off_element(src, dtype)) return ZR_ERR_SHAPE;
    if (rows > kMaxExtent || cols > kMaxExtent) return ZR_ERR_LIMIT;
    const int32_t len = axis == 1 ? cols : rows;
    if (!keep_idx) n_keep = len;
    if (n_keep < 1 || n_keep > len) return ZR_ERR_INDEX;
    if (bad_storage(q, ldq, scales, lds, n_keep, format)) return ZR_ERR_SHAPE;
    const int32_t* S = n_keep == len ? nullptr : keep_idx;       // (ascending, unique and all: the identity)
    const auto launch = axis == 1 ? launch_mx_quantize_rows : launch_mx_quantize_cols;
    return launch(src, ld, rows, cols, S, n_keep, dtype, format, (uint8_t*)q, ldq, (uint8_t*)scales, lds, (hipStream_t)stream);
}

int zr_mx_dequantize(const void* q, int64_t ldq, const void* scales, int64_t lds, int32_t rows, int32_t n, int format,
                     void* out, int64_t ldo, int dtype, void* stream)
{
    if (!q || !scales || !out) return ZR_ERR_NULL;
    if (!valid_dtype(dtype) || !valid_format(format)) return ZR_ERR_DTYPE;
    if (rows < 1 || n < 1 || ldo < n || off_element(out, dtype)) return ZR_ERR_SHAPE;
    if (rows > kMaxExtent || n > kMaxExtent) return ZR_ERR_LIMIT;
    if (bad_storage(q, ldq, scales, lds, n, format)) return ZR_ERR_SHAPE;
    return launch_mx_dequantize(MxArg{(const uint8_t*)q, ldq, (const uint8_t*)scales, lds, format}, rows, n, out, ldo, n, dtype, (hipStream_t)stream);
}

int zr_mx_linear_fwd(const void* X, int64_t ldx, void* Xq, int64_t ldxq, void* Xs, int64_t ldxs, int x_format,
                     const void* Wq, int64_t ldwq, const void* Ws, int64_t ldws, int w_format,
                     void* Y, int64_t ldy, int32_t M, int32_t K, int32_t N, const int32_t* keep_idx, int32_t n_keep,
                     int mode, int dtype, int policy, const void* prev_Y, void* stream)
{
    if (!Wq || !Ws || !Y || (!X && (!Xq || !Xs)) || !Xq != !Xs) return ZR_ERR_NULL;
    if (!valid_dtype(dtype) || (x_format != ZR_MX_E4M3 && x_format != ZR_MX_E2M1)) return ZR_ERR_DTYPE;
    if (w_format != x_format && w_format != ZR_MX_E2M1) return ZR_ERR_DTYPE;
    if (mode != ZR_DROP_N && mode != ZR_DROP_K) return ZR_ERR_MODE;
    if (policy != ZR_IMPUTE_ZERO && policy != ZR_IMPUTE_AVERAGE && policy != ZR_IMPUTE_SAME) return ZR_ERR_POLICY;
    if (M < 1 || K < 1 || N < 1 || ldy < N || (X && ldx < K)) return ZR_ERR_SHAPE;
    if (M > kMaxExtent || K > kMaxExtent || N > kMaxExtent) return ZR_ERR_LIMIT;
    const int32_t len = mode == ZR_DROP_N ? N : K;
    if (!keep_idx) n_keep = len;
    if (n_keep < 1 || n_keep > len) return ZR_ERR_INDEX;
    const bool full = n_keep == len;
    const int32_t C = held_columns(K, n_keep, mode);
    if (bad_storage(Wq, ldwq, Ws, ldws, C, w_format) || (Xq && bad_storage(Xq, ldxq, Xs, ldxs, C, x_format))) return ZR_ERR_SHAPE;
    if (off_element(X, dtype) || off_element(Y, dtype) || off_element(prev_Y, dtype)) return ZR_ERR_SHAPE;
    if (!Xq && M > MX_FEW) return ZR_ERR_NULL;
    const bool scatter = mode == ZR_DROP_N && !full;
    if (scatter && policy == ZR_IMPUTE_SAME && !prev_Y) return ZR_ERR_POLICY;

    hipStream_t s = (hipStream_t)stream;
    const int32_t* cols = mode == ZR_DROP_K && !full ? keep_idx : nullptr;
    if (X && Xq) {
        const int st = launch_mx_quantize_rows(X, ldx, M, K, cols, C, dtype, x_format, (uint8_t*)Xq, ldxq, (uint8_t*)Xs, ldxs, s);
        if (st != ZR_OK) return st;
    }
    MxProduct p;
    p.X = MxArg{(const uint8_t*)Xq, ldxq, (const uint8_t*)Xs, ldxs, x_format};
    p.W = MxArg{(const uint8_t*)Wq, ldwq, (const uint8_t*)Ws, ldws, w_format};
    p.w_rows = scatter ? keep_idx : nullptr;
    p.w_extent = N;
    p.M = M; p.J = mode == ZR_DROP_N ? n_keep : N; p.C = C;
    p.Y = Y; p.ldy = ldy; p.N = N; p.dtype = dtype;
    p.prev = scatter && policy == ZR_IMPUTE_SAME ? prev_Y : nullptr;
    p.raw = Xq ? nullptr : X;
    p.ldraw = ldx; p.raw_cols = cols; p.raw_extent = K;
    const int st = launch_mx_product(p, s);
    if (st != ZR_OK || !scatter || policy != ZR_IMPUTE_AVERAGE) return st;
    return launch_impute(Y, ldy, M, N, 1, keep_idx, n_keep, ZR_IMPUTE_AVERAGE, nullptr, dtype, s);
}

size_t zr_mx_bwd_workspace_bytes(int32_t M, int32_t K, int32_t N, int32_t n_keep, int mode, int dtype)
{
    if (M < 1 || K < 1 || N < 1 || n_keep < 1 || !valid_dtype(dtype)) return 0;
    return values_bytes(M, held_columns(K, n_keep, mode), dtype) + zr_workspace_bytes(M, K, N, n_keep, mode, dtype);
}

int zr_resized_linear_bwd_mx(const void* Xq, int64_t ldxq, const void* Xs, int64_t ldxs, int x_format,
                             const void* W, int64_t ldw, const void* dY, int64_t lddy,
                             void* dX, int64_t lddx, void* dW, int64_t lddw, int32_t M, int32_t K, int32_t N,
                             const int32_t* keep_idx, int32_t n_keep, int mode, int w_layout, int dtype, int policy,
                             const void* prev_dX, const void* prev_dW, void* workspace, size_t workspace_bytes, void* stream)
{
    const bool x_kept = mode == ZR_DROP_K;
    const int32_t held = held_columns(K, n_keep, mode);
    const int64_t ldv = round_up64(held);
    // (the values' place stands in for X in the checks; every pointer that they want is there or missed by them)
    int st = check_linear_bwd(dW && Xq && Xs ? workspace : nullptr, ldv, W, ldw, dY, lddy, dX, lddx, dW, lddw, M, K, N, keep_idx, n_keep,
                              mode, w_layout, dtype, policy, prev_dX, prev_dW, x_kept);
    if (st != ZR_OK) return st;
    size_t used = 0;
    if (dW) {
        if (!valid_format(x_format)) return ZR_ERR_DTYPE;
        if (bad_storage(Xq, ldxq, Xs, ldxs, held, x_format)) return ZR_ERR_SHAPE;
        used = values_bytes(M, held, dtype);
        if ((uintptr_t)workspace % 16 != 0 || workspace_bytes < used) return ZR_ERR_SHAPE;
        st = launch_mx_dequantize(MxArg{(const uint8_t*)Xq, ldxq, (const uint8_t*)Xs, ldxs, x_format}, M, held, workspace, ldv, (int)ldv, dtype, (hipStream_t)stream);
        if (st != ZR_OK) return st;
    }
    char* rest = workspace ? (char*)workspace + used : nullptr;
    const size_t left = workspace ? workspace_bytes - used : 0;
    return resized_linear_bwd(dW ? workspace : nullptr, ldv, W, ldw, dY, lddy, dX, lddx, dW, lddw, M, K, N, keep_idx, n_keep, mode, w_layout, dtype, policy,
                              prev_dX, prev_dW, rest, left, 0, x_kept, false, (hipStream_t)stream);
}

}  // extern "C"
