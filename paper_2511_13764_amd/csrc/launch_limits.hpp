// What one launch holds (host only, no HIP in it).  HIP keeps the grid of a launch as a 32-bit count of threads and cuts a larger one
// off: a call that needs more is launched in parts.
#pragma once
#include <stdint.h>

namespace brg {

constexpr int64_t kMostTiles = 0xffffffffLL / 512;         // workgroups of 512 threads

// Adapters' first product, H = X x down, in tiles of 16 rows (`row_tiles` at most) by 16 and more of the rank, and a launch that holds them
// and `beside` other workgroups of 512 threads.
inline bool first_product_fits(int64_t row_tiles, int64_t rank, int64_t beside)
{
    const int64_t across = (rank + 15) / 16;        // (of at most 2^31 values, like row_tiles and beside: no product of two of them wraps)
    return row_tiles * across + beside <= kMostTiles;
}

// Workgroups of a weight gradient: eight shares of every group's tiles (find_reduction).
inline int64_t reduction_grid(int64_t tiles, int64_t groups) { return (tiles + 7) / 8 * 8 * groups; }

// A weight gradient's results, `groups` of M x N, in the smallest tiles there are (64 x 64): all of it where one launch holds that, else
// its first part.  The longer side is cut, at a multiple of every tile and alignment rule, and is then far longer than that
// (one group that no launch holds has more than 2896 tiles along it), so that a part is always less than the whole; or the groups are.
struct ReductionPart {
    int64_t m, n, groups;
};
inline ReductionPart reduction_part(int64_t M, int64_t N, int64_t groups)
{
    const int64_t tiles = ((M + 63) / 64) * ((N + 63) / 64);
    if (reduction_grid(tiles, 1) > kMostTiles) {
        const int64_t half = ((M >= N ? M : N) / 2 + 255) / 256 * 256;
        return M >= N ? ReductionPart{half, N, groups} : ReductionPart{M, half, groups};
    }
    return ReductionPart{M, N, reduction_grid(tiles, groups) > kMostTiles ? groups / 2 : groups};
}

}  // namespace brg
