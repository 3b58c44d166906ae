// Products with a 4-bit image, few rows: operands go from memory to registers, the waves of a workgroup share the reduction.
//
// Decode reads every weight once for a few rows, so what counts is requests in flight: a wave takes 256 columns of 16 TN weights at a time, two
// 16-byte reads a lane for each 16, and waves w, w + W, ... take blocks of the reduction in turn; their sums meet in LDS, in a fixed order.
#include "mx4_direct.hpp"

namespace brg {

namespace {

template <int LEFT, int TM, int TN, int W, bool GROUPED>
__global__ void __launch_bounds__(64 * W, TM == 1 ? 4 : 2)
mx4_direct_kernel(Mx4Args p, GroupArgs g)
{
    __shared__ __attribute__((aligned(16))) float sums[W * 16 * TM * (16 * TN + 4)];
    int tm, tn;
    if constexpr (GROUPED) {
        GroupTile t;
        if (!find_tile<16 * TM>(g, p.tiles_n, p.walk, t))
            return;
        select_piece(p, g, t);
        tm = t.tm;
        tn = t.tn;
    } else {
        tile_coords(blockIdx.x, p.tiles_m, p.tiles_n, p.walk, tm, tn);
    }
    direct_body<LEFT, TM, TN, W>(p, tm, tn, (int)blockIdx.y, (LDS_AS float *)sums);
}

template <int LEFT, int TM, int TN, int W>
hipError_t launch(const Mx4Call &c)
{
    return mx4_launch<16 * TM, 16 * TN>(c.grouped ? mx4_direct_kernel<LEFT, TM, TN, W, true> : mx4_direct_kernel<LEFT, TM, TN, W, false>, c, 64 * W, 0);
}

template <int LEFT>
hipError_t pick(const Mx4Call &c)
{
    const int64_t rows = c.grouped ? (c.a.M + c.g.groups - 1) / c.g.groups : c.a.M;
    // 16 columns a workgroup, or 32: one workgroup a CU or less up to N = 4096 (K = 4096, 16 bf16 rows 7.2 us with 16 columns and 8.5 with 32, binary16
    // 7.4 and 9.3, images 5.2 and 5.8), from 10000 on more rounds (N = 16384: 20.9 and 14.7, 21.2 and 15.9, 11.3 and 9.7).  In between 16 rows are
    // better off with 32 (8192: 11.7 and 8.8; off 16 bytes, K = 4001, 17.3 and 12.2), one row is not (binary16 6.9 and 7.2).
    if (rows <= 16)
        return c.a.N <= 8192 ? launch<LEFT, 1, 1, 8>(c) : launch<LEFT, 1, 2, 8>(c);
    if (rows <= 32)
        return launch<LEFT, 2, 2, 8>(c);
    return launch<LEFT, 4, 4, 2>(c);
}

}  // namespace

hipError_t mx4_direct(const Mx4Call &c)
{
    return c.left == LEFT_MX4 ? pick<LEFT_MX4>(c) : c.left == LEFT_BF16 ? pick<LEFT_BF16>(c) : pick<LEFT_F16>(c);
}

}  // namespace brg
