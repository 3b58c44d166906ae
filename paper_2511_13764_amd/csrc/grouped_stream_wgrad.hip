// Instances of the streaming kernel with loading and multiplying waves whose reduction is a group's rows.
#include "grouped_tuned.hpp"

namespace brg {

namespace {

template <int BM, int BN>
hipError_t launch(const GroupedCall &c)
{
    return launch_tuned<BM, BN>(c.p.in_f16 ? grouped_stream_wgrad_kernel<BM, BN, KIND_F16> : grouped_stream_wgrad_kernel<BM, BN, KIND_BF16>, c, true,
                                S128<BN, BM>::kLds);
}

}  // namespace

hipError_t grouped_stream_wgrad(const GroupedCall &c, int tile)
{
    return tile == GEN_128 ? launch<128, 128>(c) : tile == GEN_MID ? launch<128, 64>(c) : launch<64, 64>(c);
}

}  // namespace brg
