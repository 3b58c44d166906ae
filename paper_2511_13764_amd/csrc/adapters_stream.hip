// Instances of the streaming kernel with loading and multiplying waves for a projection with adapters, in tiles of 128 x 256,
// 128 x 128, 128 x 64 and 64 x 64.
#include "grouped_tuned.hpp"

namespace brg {

namespace {

template <int BM, int BN, int KIND>
void (*pick(const Problem &p))(Bf16Args, GroupArgs, LowRank)
{
    if (p.K % BK == 0)
        return p.transB ? adapters_stream_kernel<BM, BN, LAY_K, KIND, false> : adapters_stream_kernel<BM, BN, LAY_MN, KIND, false>;
    return p.transB ? adapters_stream_kernel<BM, BN, LAY_K, KIND, true> : adapters_stream_kernel<BM, BN, LAY_MN, KIND, true>;
}

template <int BM, int BN>
hipError_t launch(const GroupedCall &c)
{
    return launch_adapters<BM, BN>(c.p.in_f16 ? pick<BM, BN, KIND_F16>(c.p) : pick<BM, BN, KIND_BF16>(c.p), c, S128<BN, BM>::kLds);
}

}  // namespace

hipError_t adapters_stream(const GroupedCall &c, int tile)
{
    return tile == GEN_WIDE ? launch<128, 256>(c) : tile == GEN_128 ? launch<128, 128>(c) : tile == GEN_MID ? launch<128, 64>(c) : launch<64, 64>(c);
}

}  // namespace brg
