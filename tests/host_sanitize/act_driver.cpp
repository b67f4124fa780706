// Drives the C entry points of what stands around a block's products (zr_act_api.hip, with zr_api.hip for the products) on the CPU
// under AddressSanitizer and UndefinedBehaviorSanitizer.  The launchers are stand-ins that check what the kernels rely
// on, among it that nothing they are handed of the workspace reaches past it.
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "zr_act.h"

namespace zr {
extern int g_launches;
extern const char* g_ws_begin;
extern const char* g_ws_end;

static void require(bool ok, const char* what)
{
    if (!ok) { fprintf(stderr, "act stub invariant violated: %s\n", what); abort(); }
}
static bool within(const void* p, size_t bytes) { return (const char*)p >= g_ws_begin && (const char*)p + bytes <= g_ws_end; }
static void check_drop(const uint64_t* rng, uint32_t drop, float factor)
{
    require(drop <= 65535 && (drop == 0 || (rng && (uintptr_t)rng % 8 == 0)), "the generator");
    require(factor >= 1.f && factor <= 65536.f, "the factor");
}

int act_slabs(int M, int) { return (M + 12) / 13; }
int launch_act_back(const ActBack& a, int dtype, hipStream_t)
{
    ++g_launches;
    const size_t es = dtype == ZR_BF16 ? 2 : 4;
    require(a.dY && a.M >= 1 && a.N >= 1 && a.lddy >= a.N, "dY");
    require(a.Z ? a.ldz >= a.N : a.act == ZR_ACT_NONE && !a.dgate, "Z");
    require((!a.gate || a.ldg >= a.N) && (!a.dgate || a.lddg >= a.N), "gates");
    require(a.dz || a.partial || a.dgate, "a pass for nothing");
    if (a.dz) require(within(a.dz, (size_t)a.M * a.lddz * es) && (uintptr_t)a.dz % 16 == 0, "dZ past the workspace");
    if (a.dz && a.keep) require(dtype == ZR_BF16 && a.N > ACT_KEPT_ABOVE && a.n_keep >= 1 && a.n_keep < a.N && a.width >= a.n_keep && a.width % 64 == 0 && a.lddz == a.width, "kept columns");
    if (a.dz && !a.keep) require(a.lddz >= a.N && a.lddz % 8 == 0, "pitch of dZ");
    if (a.partial) require(within(a.partial, (size_t)act_slabs(a.M, a.N) * a.N * 4) && (uintptr_t)a.partial % 16 == 0, "sums past the workspace");
    if (a.partial && a.dz) require((const char*)a.dz + (size_t)a.M * a.lddz * es <= (const char*)a.partial, "dZ runs into the sums");
    check_drop(a.rng, a.drop, a.factor);
    return ZR_OK;
}
int launch_sum_slabs(const float* partial, int slabs, int n, void* out, int, hipStream_t)
{
    ++g_launches;
    require(slabs >= 1 && n >= 1, "sums");
    require(within(partial, (size_t)slabs * n * 4), "sums past the workspace");
    require(out != nullptr, "sums for nobody");
    return ZR_OK;
}
int launch_join_sums(const Join& j, int, hipStream_t)
{
    ++g_launches;
    require(j.slabs >= 1 && within(j.partial, (size_t)(j.biases ? (int)JOIN_SUMS : 2) * j.slabs * j.cols * 4), "sums past the workspace");
    bool any = false;
    for (void* v : j.vectors) any |= v != nullptr;
    require(any, "sums for nobody");
    require(j.biases || (!j.vectors[0] && !j.vectors[3] && !j.vectors[5] && !(j.vectors[1] && j.post && j.post_b)), "sums that were not taken");
    require(j.pre || (!j.vectors[4] && !j.vectors[5]), "a norm's gradients without one");
    return ZR_OK;
}
int launch_dropout(const void* x, int64_t ldx, void* out, int64_t ldo, int rows, int cols, const uint64_t* rng, uint32_t drop, float factor, int, hipStream_t)
{
    ++g_launches;
    require(x && out && rows >= 1 && cols >= 1 && ldx >= cols && ldo >= cols, "dropout");
    check_drop(rng, drop, factor);
    return ZR_OK;
}
int join_max_cols() { return 600; }
int join_most_slabs(int rows, int) { return rows < 9 ? rows : 9; }
int join_slabs(const Join& j) { return join_most_slabs(j.rows, j.cols) - (j.biases && j.rows > 1); }
static void check_join(const Join& j)
{
    require(j.rows >= 1 && j.cols >= 1 && j.cols <= join_max_cols() && j.eps >= 0.f, "extents of a join");
    require((!j.post || true) && (j.layer == 0 || j.layer == 1), "norms of a join");
    check_drop(j.rng, j.drop, j.factor);
}
int launch_join(const Join& j, int, hipStream_t)
{
    ++g_launches;
    check_join(j);
    require(j.y && j.x && j.x_out && j.ldy >= j.cols && j.ldx >= j.cols && j.ldxo >= j.cols, "tensors of a join");
    require(!j.pre || (j.h && j.ldh >= j.cols), "h");
    return ZR_OK;
}
int launch_join_back(const Join& j, int, hipStream_t)
{
    ++g_launches;
    check_join(j);
    require(j.pre ? j.dh && j.x && j.lddh >= j.cols && j.ldx >= j.cols : j.dx_out != nullptr, "gradients that come in");
    require(!j.post || j.y, "the post norm's input");
    require((!j.y || j.ldy >= j.cols) && (!j.dx_out || j.lddxo >= j.cols) && (!j.dx || j.lddx >= j.cols) && (!j.dy || j.lddy >= j.cols), "pitches");
    require(j.dx || j.dy || j.partial, "a pass for nothing");
    if (j.partial) require(within(j.partial, (size_t)(j.biases ? (int)JOIN_SUMS : 2) * j.slabs * j.cols * 4), "sums past the workspace");
    return ZR_OK;
}
}  // namespace zr

using namespace zr;

int main()
{
    std::mt19937 rng(11);
    auto pick = [&](int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); };
    std::vector<char> room((size_t)1 << 20);
    char* p = (char*)(((uintptr_t)room.data() + 255) / 256 * 256);
    const size_t ws_room = (size_t)160 << 20;
    char* ws = (char*)aligned_alloc(256, ws_room);       // never touched, only measured
    int refused = 0, done = 0;
    auto maybe = [&](char* q, int of = 3) -> char* { return pick(0, of) ? q : nullptr; };
    for (int it = 0; it < 200000; ++it) {
        const int M = pick(0, 30) ? pick(1, 40) : 0, K = pick(1, 400), N = pick(0, 30) ? pick(1, 700) : 0;
        const int mode = pick(0, 40) ? pick(0, 1) : 2, dtype = pick(0, 40) ? pick(0, 1) : 2, layout = pick(0, 1), act = pick(0, 40) ? pick(0, 4) : 5;
        const int len = mode == ZR_DROP_N ? N : K, n_keep = pick(0, 9) ? (len ? pick(1, len) : 0) : len + 1;
        const bool list = pick(0, 3) != 0;
        const double prob = pick(0, 1) ? 0.0 : pick(0, 20) ? pick(0, 99) / 100.0 : 1.0;
        const uint64_t* gen = (const uint64_t*)(pick(0, 5) ? p + (pick(0, 20) ? 0 : 4) : nullptr);
        const int64_t lw = layout == ZR_W_KN ? N : K, ln = N + (pick(0, 20) ? pick(0, 2) : -1);
        const int kept = list ? n_keep : len;
        const int before = g_launches;
        int st;
        char* w = ws + (pick(0, 20) ? 0 : 8);
        auto give = [&](size_t need) {
            const size_t bytes = pick(0, 3) ? need : need / (size_t)pick(1, 5);
            require(bytes + 64 <= ws_room, "room for the largest workspace");
            g_ws_begin = w; g_ws_end = w + bytes;
            return bytes;
        };
        if (it % 4 == 0) {
            const size_t bytes = give(zr_act_fwd_workspace_bytes(M, K, N, kept, mode, dtype));
            st = zr_resized_linear_act_fwd(p, K + pick(0, 2), p, lw, p, ln, M, K, N, list ? (const int32_t*)p : nullptr, n_keep, mode, layout, dtype,
                                           maybe(p), act, maybe(p), N, prob, gen, maybe(p), N + pick(0, 1), maybe(p), N, maybe(w), bytes, nullptr);
        } else if (it % 4 == 1) {
            const size_t bytes = give(zr_act_bwd_workspace_bytes(M, K, N, kept, mode, dtype));
            char *dx = maybe(p + 262144), *dw = maybe(p + 393216);
            st = zr_resized_linear_act_bwd(maybe(p, 9), K, maybe(p, 9), lw, p, ln, maybe(p, 9), N, maybe(p), N, dx, K, dw, lw, maybe(p), maybe(p), N, M, K, N,
                                           list ? (const int32_t*)p : nullptr, n_keep, mode, layout, dtype, act, prob, gen, maybe(w, 9), bytes, nullptr);
        } else if (it % 4 == 2) {
            const bool back = pick(0, 2) != 0;
            const int norms = pick(0, 30) ? pick(0, 3) : 4, norm = pick(0, 1);
            const double eps = pick(0, 30) ? 1e-5 : -1.0;
            if (!back) {
                st = zr_block_join_fwd(p, ln, p, N, p, N, maybe(p, 9), N, M, N, norms, norm, eps, prob, gen, 0.5, maybe(p), maybe(p), maybe(p), maybe(p), maybe(p),
                                       maybe(p), dtype, nullptr);
            } else {
                const size_t bytes = give(zr_block_join_workspace_bytes(M, N));
                const bool po = norms & 1, pr = norms & 2;
                st = zr_block_join_bwd(maybe(p), ln, maybe(p, 9), N, maybe(p, 9), N, maybe(p, 9), N, maybe(p), N, maybe(p), N, M, N, norms, norm, eps, prob, gen, 0.5,
                                       maybe(p), maybe(p), maybe(p), maybe(p), maybe(p), maybe(p), maybe(p), po || !pick(0, 30) ? maybe(p) : nullptr,
                                       po ? maybe(p) : nullptr, pr || !pick(0, 30) ? maybe(p) : nullptr, pr ? maybe(p) : nullptr, maybe(w, 9), bytes, dtype, nullptr);
            }
        } else {
            st = zr_dropout(maybe(p, 20), ln, maybe(p, 20), N, M, N, prob, gen, dtype, nullptr);
        }
        if (st != ZR_OK) { require(g_launches == before, "a refused call enqueued work"); ++refused; }
        else { require(g_launches > before, "an accepted call enqueued nothing"); ++done; }
    }
    require(refused > 10000 && done > 10000, "both kinds of calls");
    printf("OK %d done, %d refused\n", done, refused);
    free(ws);
    return 0;
}
