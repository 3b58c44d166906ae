// Instances of the 256 x 256 x 64 ping-pong kernel for a projection with adapters.
#include "grouped_tuned.hpp"

namespace brg {

namespace {

template <int KIND>
void (*pick(const Problem &p))(Bf16Args, GroupArgs, LowRank)
{
    if (p.K % BK == 0)
        return p.transB ? adapters_pingpong_kernel<LAY_K, KIND, false> : adapters_pingpong_kernel<LAY_MN, KIND, false>;
    return p.transB ? adapters_pingpong_kernel<LAY_K, KIND, true> : adapters_pingpong_kernel<LAY_MN, KIND, true>;
}

}  // namespace

hipError_t adapters_pingpong(const GroupedCall &c)
{
    return launch_adapters<PP_BM, PP_BN>(c.p.in_f16 ? pick<KIND_F16>(c.p) : pick<KIND_BF16>(c.p), c, (size_t)PP_SLOTS * PP_SLOT);
}

}  // namespace brg
