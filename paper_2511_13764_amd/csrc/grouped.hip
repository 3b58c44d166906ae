// Plan and launches of the grouped products (grouped.hpp).
#include "variants.hpp"
#include "grouped.hpp"

namespace brg {

namespace {

// HIP keeps the grid of a launch as 32-bit counts of threads: larger ones are launched in halves, as elsewhere.
constexpr int64_t kMostTiles = 0xffffffffLL / 512;

inline int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

}  // namespace

hipError_t launch_grouped(GroupedCall &c)
{
    Problem &p = c.p;
    const int64_t rows = most_row_tiles(p.M, c.g.groups + 2 * c.g.cover, 32);
    if (rows > kMostTiles)
        return hipErrorInvalidValue;                // (the caller refuses these)
    if (rows * ((p.N + 31) / 32) > kMostTiles) {
        const int64_t n = p.N <= 256 ? round_up(p.N / 2, 32) : round_up(p.N / 2, 256);
        const int64_t esz = in_16bit(p) ? 2 : 4;
        GroupedCall rest = c;
        p.N = n;
        rest.p.N -= n;
        rest.p.B = (const char *)p.B + n * (p.transB ? p.ldb : 1) * esz;
        rest.p.C = (char *)p.C + n * (p.c_f32 ? 4 : 2);
        rest.p.bias = p.bias ? p.bias + n : nullptr;
        rest.low.up = c.low.up ? c.low.up + n * (p.transB ? c.low.ld_up : 1) * esz : nullptr;
        const hipError_t e = launch_grouped(c);
        return e == hipSuccess ? launch_grouped(rest) : e;
    }
    return grouped_general(c);
}

hipError_t launch_grouped_wgrad(GroupedCall &c)
{
    Problem &p = c.p;
    const int64_t tiles = ((p.M + 63) / 64) * ((p.N + 63) / 64);
    GroupedCall rest = c;
    const int64_t csz = p.c_f32 ? 4 : 2;
    if (tiles > kMostTiles) {
        const int64_t m = round_up(p.M / 2, 256);
        p.M = m;
        rest.p.M -= m;
        rest.p.A = (const char *)p.A + m * (in_16bit(p) ? 2 : 4);
        rest.p.C = (char *)p.C + m * p.ldc * csz;
    } else if (tiles * c.g.groups > kMostTiles) {
        const int half = c.g.groups / 2;
        c.g.groups = half;
        rest.g.groups -= half;
        rest.g.offsets += half;
        rest.p.C = (char *)p.C + half * c.g.stride_c * csz;
    } else {
        return grouped_general_wgrad(c);
    }
    const hipError_t e = launch_grouped_wgrad(c);
    return e == hipSuccess ? launch_grouped_wgrad(rest) : e;
}

}  // namespace brg
