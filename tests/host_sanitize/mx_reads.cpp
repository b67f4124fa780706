// The reads of the kernel that puts blocks back into values (mx_read_at and mx_read of zr_mx.h, the very functions that the
// kernel calls), for every lane of rows of every length, on the CPU under AddressSanitizer: a row's storage is a buffer of its
// own, so a byte before or behind it is a failure, and what a lane keeps is compared with the elements that were put there.
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "zr_mx.h"

using namespace zr;

static long g_lanes = 0, g_idle = 0;

static void require(bool ok, const char* what, int n, int width, int at)
{
    if (!ok) { printf("FAILED %s: n %d, width %d, at %d\n", what, n, width, at); exit(1); }
}

template <int FMT, int PER, bool VEC> void row(int n, int width)
{
    const int bytes = (int)mx_row_bytes(n, FMT), held = (n + 127) / 128 * 128;
    uint8_t* q = (uint8_t*)malloc(bytes);
    auto element = [](int i) { return (uint32_t)(i * 7 + i / 16 * 5 + 3) & (FMT == ZR_MX_E2M1 ? 15u : 255u); };
    for (int i = 0; i < bytes; ++i) q[i] = (uint8_t)(FMT == ZR_MX_E2M1 ? element(2 * i) | element(2 * i + 1) << 4 : element(i));
    std::vector<int> stored(width);
    // off: elements between an aligned address and the row's first one
    for (int off = 0; off < (VEC ? 1 : PER); ++off) {
        stored.assign(width, 0);
        for (int chunk = 0; chunk < mx_value_segs(width, PER, VEC) * 64; ++chunk) {
            const int at = chunk * PER - off;
            const MxRead a = mx_read_at<FMT, PER, VEC>(at, n, width);
            constexpr int took = FMT == ZR_MX_E2M1 ? PER / 2 : PER;
            require(a.b >= 0 && a.b + took <= bytes && a.more >= 0 && a.more < bytes, "a read past the row", n, width, at);
            require(a.e >= 0 && a.e < held && (a.e + PER - 1 < width ? a.e + PER - 1 : width - 1) / 32 < (int)mx_scale_bytes(n), "a scale past the row", n, width, at);
            const uint2 w = mx_read<FMT, PER, VEC>(q, a);
            const uint64_t bits = w.x | (uint64_t)w.y << 32;
            ++g_lanes;
            if (at >= width) ++g_idle;
            // what the kernel keeps: elements e + i of [at, at + PER) within the row
            for (int i = 0; i < PER; ++i) {
                const int k = a.e + i;
                if (k < at || k >= at + PER || k >= width) continue;
                require((bits >> (FMT == ZR_MX_E2M1 ? 4 * i : 8 * i) & (FMT == ZR_MX_E2M1 ? 15u : 255u)) == element(k), "an element", n, width, at);
                ++stored[k];
            }
        }
        for (int k = 0; k < width; ++k) require(stored[k] == 1, "an element that no lane stores, or two", n, width, k);
    }
    free(q);
}

template <int FMT> void length(int n, int width)
{
    row<FMT, 8, true>(n, width);
    row<FMT, 4, true>(n, width);
    row<FMT, 8, false>(n, width);
    row<FMT, 4, false>(n, width);
}

int main()
{
    std::vector<int> lengths;
    for (int n = 1; n <= 1300; ++n) lengths.push_back(n);
    for (int n : {2047, 2048, 2064, 2176, 2751, 2752, 2816, 5503, 5504, 6912, 11008, 16384}) lengths.push_back(n);
    for (int n : lengths)
        for (int width : {n, (n + 63) / 64 * 64}) {         // on its own; before a backward product
            length<ZR_MX_E4M3>(n, width);
            length<ZR_MX_E2M1>(n, width);
            length<ZR_MX_INT8>(n, width);
        }
    printf("OK %ld lanes, %ld idle\n", g_lanes, g_idle);
    return 0;
}
