// C ABI of what stands around the products of a block: argument checks, and the mapping onto the kernels (zr_act.h) and onto the
// resized layer's products.
#include "zr_act.h"

using namespace zr;

namespace {

constexpr int32_t kMaxExtent = 65535 * 32;      // as for the other calls
constexpr size_t kSliceBytes = (size_t)64 << 20;

bool valid_dtype(int dt) { return dt == ZR_F32 || dt == ZR_BF16; }
size_t size_of(int dtype) { return dtype == ZR_BF16 ? 2 : 4; }
bool valid_act(int a) { return a >= ZR_ACT_NONE && a <= ZR_ACT_SILU; }
template <class... P> bool off_element(int dtype, P... p) { return ((((uintptr_t)p) % size_of(dtype) != 0) || ...); }

// 0 <= p < 1: the halves below which an element is dropped; the generator where there are any
int check_dropout(double p, const uint64_t* rng, uint32_t& drop)
{
    if (!(p >= 0.0) || !(p < 1.0)) return ZR_ERR_RATIO;
    drop = drop_below(p);
    if (drop == 0) return ZR_OK;
    if (!rng) return ZR_ERR_NULL;
    return (uintptr_t)rng % 8 != 0 ? ZR_ERR_SHAPE : ZR_OK;
}

int check_layer(int32_t M, int32_t K, int32_t N, const int32_t* keep_idx, int32_t& n_keep, int mode, int w_layout, int dtype, int act)
{
    if (!valid_dtype(dtype)) return ZR_ERR_DTYPE;
    if ((mode != ZR_DROP_N && mode != ZR_DROP_K) || (w_layout != ZR_W_KN && w_layout != ZR_W_NK) || !valid_act(act)) return ZR_ERR_MODE;
    if (M < 1 || K < 1 || N < 1) return ZR_ERR_SHAPE;
    if (M > kMaxExtent || K > kMaxExtent || N > kMaxExtent) return ZR_ERR_LIMIT;
    const int32_t n = mode == ZR_DROP_N ? N : K;
    if (!keep_idx) n_keep = n;
    return n_keep < 1 || n_keep > n ? ZR_ERR_INDEX : ZR_OK;
}

size_t round_up16(size_t v) { return (v + 15) & ~(size_t)15; }

// The workspace of the backward pass: dZ [M x pitch], the column sums of its slabs, and zr_resized_linear_bwd's scratch.
int64_t dz_pitch(int32_t N) { return ((int64_t)N + 7) / 8 * 8; }
size_t dz_bytes(int32_t M, int32_t N, int dtype) { return round_up16((size_t)M * (size_t)((N + 63) / 64 * 64) * size_of(dtype)); }
size_t sums_bytes(int32_t M, int32_t N) { return round_up16((size_t)act_slabs(M, N) * (size_t)N * 4); }

}  // namespace

extern "C" {

int zr_dropout(const void* x, int64_t ldx, void* out, int64_t ldo, int32_t rows, int32_t cols, double p, const uint64_t* rng,
               int dtype, void* stream)
{
    if (!x || !out) return ZR_ERR_NULL;
    if (!valid_dtype(dtype)) return ZR_ERR_DTYPE;
    if (rows < 1 || cols < 1 || ldx < cols || ldo < cols || off_element(dtype, x, out)) return ZR_ERR_SHAPE;
    if (rows > kMaxExtent || cols > kMaxExtent) return ZR_ERR_LIMIT;
    uint32_t drop;
    const int st = check_dropout(p, rng, drop);
    if (st != ZR_OK) return st;
    return launch_dropout(x, ldx, out, ldo, rows, cols, rng, drop, kept_factor(drop), dtype, (hipStream_t)stream);
}

size_t zr_act_fwd_workspace_bytes(int32_t M, int32_t K, int32_t N, int32_t n_keep, int mode, int dtype)
{
    if (M < 1 || K < 1 || N < 1 || n_keep < 1 || !valid_dtype(dtype)) return 0;
    // (bf16) the kept columns of X, which DROP_K multiplies, and the slices of a split contraction
    const size_t held = mode == ZR_DROP_K && n_keep < K && dtype == ZR_BF16 ? (size_t)M * (size_t)((n_keep + 63) / 64 * 64) * 2 : 0;
    return held + (dtype == ZR_BF16 ? kSliceBytes : 0) + 16;
}

int zr_resized_linear_act_fwd(const void* X, int64_t ldx, const void* W, int64_t ldw, void* Y, int64_t ldy,
                              int32_t M, int32_t K, int32_t N, const int32_t* keep_idx, int32_t n_keep, int mode, int w_layout, int dtype,
                              const void* bias, int act, const void* gate, int64_t ldg, double p, const uint64_t* rng,
                              const void* residual, int64_t ldr, void* Z, int64_t ldz,
                              void* workspace, size_t workspace_bytes, void* stream)
{
    if (!X || !W || !Y) return ZR_ERR_NULL;
    int st = check_layer(M, K, N, keep_idx, n_keep, mode, w_layout, dtype, act);
    if (st != ZR_OK) return st;
    if (ldx < K || ldw < (w_layout == ZR_W_KN ? N : K) || ldy < N) return ZR_ERR_SHAPE;
    if ((gate && ldg < N) || (residual && ldr < N) || (Z && ldz < N)) return ZR_ERR_SHAPE;
    if (off_element(dtype, X, W, Y, bias, gate, residual, Z)) return ZR_ERR_SHAPE;
    Finish f;
    st = check_dropout(p, rng, f.drop);
    if (st != ZR_OK) return st;
    f.bias = bias; f.gate = gate; f.ldg = ldg; f.residual = residual; f.ldr = ldr; f.Z = Z; f.ldz = ldz;
    f.rng = rng; f.factor = kept_factor(f.drop); f.act = act;
    return resized_linear_fwd(X, ldx, W, ldw, Y, ldy, M, K, N, keep_idx, n_keep, mode, w_layout, dtype, ZR_IMPUTE_ZERO, nullptr, &f,
                              workspace, workspace_bytes, (hipStream_t)stream);
}

size_t zr_act_bwd_workspace_bytes(int32_t M, int32_t K, int32_t N, int32_t n_keep, int mode, int dtype)
{
    if (M < 1 || K < 1 || N < 1 || n_keep < 1 || !valid_dtype(dtype)) return 0;
    return dz_bytes(M, N, dtype) + sums_bytes(M, N) + zr_workspace_bytes(M, K, N, n_keep, mode, dtype);
}

int zr_resized_linear_act_bwd(const void* X, int64_t ldx, const void* W, int64_t ldw, const void* dY, int64_t lddy,
                              const void* Z, int64_t ldz, const void* gate, int64_t ldg,
                              void* dX, int64_t lddx, void* dW, int64_t lddw, void* dbias, void* dgate, int64_t lddg,
                              int32_t M, int32_t K, int32_t N, const int32_t* keep_idx, int32_t n_keep, int mode, int w_layout, int dtype,
                              int act, double p, const uint64_t* rng, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!dY || (!dX && !dW && !dbias && !dgate)) return ZR_ERR_NULL;
    if ((dX && !W) || (dW && !X)) return ZR_ERR_NULL;
    int st = check_layer(M, K, N, keep_idx, n_keep, mode, w_layout, dtype, act);
    if (st != ZR_OK) return st;
    const bool needs_z = act != ZR_ACT_NONE || dgate;
    if (needs_z && !Z) return ZR_ERR_NULL;
    if (lddy < N || (needs_z && ldz < N) || (gate && ldg < N) || (dgate && lddg < N)) return ZR_ERR_SHAPE;
    const bool kn = w_layout == ZR_W_KN;
    if (dX && (ldw < (kn ? N : K) || lddx < K)) return ZR_ERR_SHAPE;
    if (dW && (ldx < K || lddw < (kn ? N : K))) return ZR_ERR_SHAPE;
    if (off_element(dtype, X, W, dY, Z, gate, dX, dW, dbias, dgate)) return ZR_ERR_SHAPE;
    ActBack a;
    st = check_dropout(p, rng, a.drop);
    if (st != ZR_OK) return st;

    const bool products = dX || dW;
    // dZ is not dY itself, or dY may be where dgate goes
    const bool changes = act != ZR_ACT_NONE || gate || a.drop || dgate;
    const bool holds = products && changes;
    // bf16 products of kept columns read them side by side: dZ is written that way
    const bool kept = holds && dtype == ZR_BF16 && mode == ZR_DROP_N && n_keep < N && N > ACT_KEPT_ABOVE;
    const int64_t pitch = kept ? (n_keep + 63) / 64 * 64 : dz_pitch(N);
    const size_t dz = holds ? round_up16((size_t)M * (size_t)pitch * size_of(dtype)) : 0, sums = dbias ? sums_bytes(M, N) : 0;
    if (dz + sums) {
        if (!workspace) return ZR_ERR_NULL;
        if ((uintptr_t)workspace % 16 != 0 || workspace_bytes < dz + sums) return ZR_ERR_SHAPE;
    }
    hipStream_t s = (hipStream_t)stream;
    if (holds || dbias || dgate) {
        a.dY = dY; a.lddy = lddy; a.Z = needs_z ? Z : nullptr; a.ldz = ldz; a.gate = gate; a.ldg = ldg; a.dgate = dgate; a.lddg = lddg;
        a.dz = holds ? workspace : nullptr; a.lddz = pitch;
        a.keep = kept ? keep_idx : nullptr; a.n_keep = n_keep; a.width = (int)pitch;
        a.partial = dbias ? (float*)((char*)workspace + dz) : nullptr;
        a.rng = rng; a.factor = kept_factor(a.drop); a.act = act; a.M = M; a.N = N;
        st = launch_act_back(a, dtype, s);
        if (st != ZR_OK) return st;
        if (dbias) {
            st = launch_sum_slabs(a.partial, act_slabs(M, N), N, dbias, dtype, s);
            if (st != ZR_OK) return st;
        }
    }
    if (!products) return ZR_OK;
    char* rest = workspace ? (char*)workspace + dz + sums : nullptr;
    // (without a list every index is kept, and the list is not read: any address stands in for it)
    return resized_linear_bwd(X, ldx, W, ldw, holds ? workspace : dY, holds ? pitch : lddy, dX, lddx, dW, lddw, M, K, N,
                              keep_idx ? keep_idx : (const int32_t*)dY, n_keep, mode, w_layout, dtype, ZR_IMPUTE_ZERO, nullptr, nullptr,
                              rest, workspace ? workspace_bytes - dz - sums : 0, 0, false, kept, s);
}

static int check_join(int32_t rows, int32_t cols, int norms, int norm, double eps, int dtype)
{
    if (!valid_dtype(dtype)) return ZR_ERR_DTYPE;
    if ((norms & ~(ZR_JOIN_POST | ZR_JOIN_PRE)) != 0 || (norm != ZR_NORM_RMS && norm != ZR_NORM_LAYER)) return ZR_ERR_MODE;
    if (rows < 1 || cols < 1) return ZR_ERR_SHAPE;
    if (rows > kMaxExtent || cols > join_max_cols()) return ZR_ERR_LIMIT;
    return eps >= 0.0 ? ZR_OK : ZR_ERR_RATIO;
}

int zr_block_join_fwd(const void* y, int64_t ldy, const void* x, int64_t ldx, void* x_out, int64_t ldxo, void* h, int64_t ldh,
                      int32_t rows, int32_t cols, int norms, int norm, double eps, double p, const uint64_t* rng, double scale,
                      const void* bias, const void* gate, const void* post_w, const void* post_b, const void* pre_w, const void* pre_b,
                      int dtype, void* stream)
{
    const bool pre = (norms & ZR_JOIN_PRE) != 0;
    if (!y || !x || !x_out || (pre && !h)) return ZR_ERR_NULL;
    int st = check_join(rows, cols, norms, norm, eps, dtype);
    if (st != ZR_OK) return st;
    if (ldy < cols || ldx < cols || ldxo < cols || (pre && ldh < cols)) return ZR_ERR_SHAPE;
    if (off_element(dtype, y, x, x_out, h, bias, gate, post_w, post_b, pre_w, pre_b)) return ZR_ERR_SHAPE;
    Join j = {};
    st = check_dropout(p, rng, j.drop);
    if (st != ZR_OK) return st;
    j.y = y; j.ldy = ldy; j.x = x; j.ldx = ldx; j.x_out = x_out; j.ldxo = ldxo; j.h = h; j.ldh = ldh;
    j.bias = bias; j.gate = gate; j.post_w = post_w; j.post_b = post_b; j.pre_w = pre_w; j.pre_b = pre_b;
    j.scale = (float)scale; j.eps = (float)eps; j.post = (norms & ZR_JOIN_POST) != 0; j.pre = pre; j.layer = norm == ZR_NORM_LAYER;
    j.rng = rng; j.factor = kept_factor(j.drop); j.rows = rows; j.cols = cols;
    return launch_join(j, dtype, (hipStream_t)stream);
}

size_t zr_block_join_workspace_bytes(int32_t rows, int32_t cols)
{
    if (rows < 1 || cols < 1 || cols > join_max_cols()) return 0;
    return (size_t)JOIN_SUMS * (size_t)join_most_slabs(rows, cols) * (size_t)cols * 4;
}

int zr_block_join_bwd(const void* dx_out, int64_t lddxo, const void* dh, int64_t lddh, const void* x_out, int64_t ldxo,
                      const void* y, int64_t ldy, void* dx, int64_t lddx, void* dy, int64_t lddy,
                      int32_t rows, int32_t cols, int norms, int norm, double eps, double p, const uint64_t* rng, double scale,
                      const void* bias, const void* gate, const void* post_w, const void* post_b, const void* pre_w,
                      void* dbias, void* dgate, void* dpost_w, void* dpost_b, void* dpre_w, void* dpre_b,
                      void* workspace, size_t workspace_bytes, int dtype, void* stream)
{
    const bool post = (norms & ZR_JOIN_POST) != 0, pre = (norms & ZR_JOIN_PRE) != 0;
    const bool vectors = dbias || dgate || dpost_w || dpost_b || dpre_w || dpre_b;
    if (!dx && !dy && !vectors) return ZR_ERR_NULL;
    if ((pre && (!dh || !x_out)) || (!pre && !dx_out) || ((post || dgate) && !y)) return ZR_ERR_NULL;
    int st = check_join(rows, cols, norms, norm, eps, dtype);
    if (st != ZR_OK) return st;
    if ((!post && (dpost_w || dpost_b)) || (!pre && (dpre_w || dpre_b))) return ZR_ERR_MODE;
    const bool needs_y = post || dgate;
    if ((dx_out && lddxo < cols) || (pre && (lddh < cols || ldxo < cols)) || (needs_y && ldy < cols)) return ZR_ERR_SHAPE;
    if ((dx && lddx < cols) || (dy && lddy < cols)) return ZR_ERR_SHAPE;
    if (off_element(dtype, dx_out, dh, x_out, y, dx, dy, bias, gate, post_w, post_b, pre_w, dbias, dgate, dpost_w, dpost_b, dpre_w, dpre_b))
        return ZR_ERR_SHAPE;
    Join j = {};
    st = check_dropout(p, rng, j.drop);
    if (st != ZR_OK) return st;
    if (vectors) {
        if (!workspace) return ZR_ERR_NULL;
        if ((uintptr_t)workspace % 16 != 0 || workspace_bytes < zr_block_join_workspace_bytes(rows, cols)) return ZR_ERR_SHAPE;
    }
    j.y = needs_y ? y : nullptr; j.ldy = ldy; j.x = x_out; j.ldx = ldxo;
    j.bias = needs_y ? bias : nullptr; j.gate = gate; j.post_w = post_w; j.post_b = post_b; j.pre_w = pre_w;
    j.scale = (float)scale; j.eps = (float)eps; j.post = post; j.pre = pre; j.layer = norm == ZR_NORM_LAYER;
    j.rng = rng; j.factor = kept_factor(j.drop); j.rows = rows; j.cols = cols;
    j.dx_out = dx_out; j.lddxo = lddxo; j.dh = dh; j.lddh = lddh; j.dx = dx; j.lddx = lddx; j.dy = dy; j.lddy = lddy;
    j.partial = vectors ? (float*)workspace : nullptr;
    j.biases = dbias || dpost_b || dpre_b || (dgate && post && post_b);
    j.slabs = join_slabs(j);
    hipStream_t s = (hipStream_t)stream;
    st = launch_join_back(j, dtype, s);
    if (st != ZR_OK || !vectors) return st;
    void* const gradients[6] = {dbias, dgate, dpost_w, dpost_b, dpre_w, dpre_b};
    std::copy(gradients, gradients + 6, j.vectors);
    return launch_join_sums(j, dtype, s);
}

}  // extern "C"
