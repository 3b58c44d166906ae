// Instances of the 256 x 256 x 64 ping-pong kernel on rows grouped by their weights.
#include "grouped_tuned.hpp"

namespace brg {

namespace {

template <int KIND>
void (*pick(const Problem &p))(Bf16Args, GroupArgs)
{
    if (p.K % BK == 0)
        return p.transB ? grouped_pingpong_kernel<LAY_K, KIND, false> : grouped_pingpong_kernel<LAY_MN, KIND, false>;
    return p.transB ? grouped_pingpong_kernel<LAY_K, KIND, true> : grouped_pingpong_kernel<LAY_MN, KIND, true>;
}

}  // namespace

hipError_t grouped_pingpong(const GroupedCall &c)
{
    return launch_tuned<PP_BM, PP_BN>(c.p.in_f16 ? pick<KIND_F16>(c.p) : pick<KIND_BF16>(c.p), c, false, (size_t)PP_SLOTS * PP_SLOT);
}

}  // namespace brg
