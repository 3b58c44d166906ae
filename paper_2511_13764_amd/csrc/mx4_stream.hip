// Kernels of the tiles of 16 to 128 rows (mx4_stream.hpp).
#include "mx4_stream.hpp"

namespace brg {

namespace {

template <int LEFT, int BM, int BN, bool GROUPED>
__global__ void __launch_bounds__(512, BM == 128 || (BM == 64 && LEFT != LEFT_MX4) ? 2 : 4)
mx4_stream_kernel(Mx4Args p, GroupArgs g)
{
    int tm, tn;
    if constexpr (GROUPED) {
        GroupTile t;
        if (!find_tile<BM>(g, p.tiles_n, p.walk, t))
            return;
        select_piece(p, g, t);
        tm = t.tm;
        tn = t.tn;
    } else {
        tile_coords(blockIdx.x, p.tiles_m, p.tiles_n, p.walk, tm, tn);
    }
    mx4_stream_tile<LEFT, BM, BN>(p, tm, tn, (int)blockIdx.y);
}

template <int LEFT, int BM, int BN>
hipError_t launch(const Mx4Call &c)
{
    return mx4_launch<BM, BN>(c.grouped ? mx4_stream_kernel<LEFT, BM, BN, true> : mx4_stream_kernel<LEFT, BM, BN, false>, c, 512, Mx4Ring<LEFT, BM, BN>::LDS);
}

template <int LEFT>
hipError_t pick(const Mx4Call &c, int bm, int bn)
{
    if constexpr (LEFT != LEFT_MX4) {
        if (bm < 64)
            return bm == 16 ? launch<LEFT, 16, 64>(c) : launch<LEFT, 32, 64>(c);
    }
    return bm == 128 ? launch<LEFT, 128, 128>(c) : bn == 128 ? launch<LEFT, 64, 128>(c) : launch<LEFT, 64, 64>(c);
}

}  // namespace

hipError_t mx4_stream(const Mx4Call &c, int bm, int bn)
{
    return c.left == LEFT_MX4 ? pick<LEFT_MX4>(c, bm, bn) : c.left == LEFT_BF16 ? pick<LEFT_BF16>(c, bm, bn) : pick<LEFT_F16>(c, bm, bn);
}

}  // namespace brg
