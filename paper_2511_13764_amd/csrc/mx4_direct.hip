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
