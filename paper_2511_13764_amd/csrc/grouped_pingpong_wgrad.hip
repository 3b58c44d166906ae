// Instances of the 256 x 256 x 64 ping-pong kernel whose reduction is a group's rows.
#include "grouped_tuned.hpp"

namespace brg {

hipError_t grouped_pingpong_wgrad(const GroupedCall &c)
{
    return launch_tuned<PP_BM, PP_BN>(c.p.in_f16 ? grouped_pingpong_wgrad_kernel<KIND_F16> : grouped_pingpong_wgrad_kernel<KIND_BF16>, c, true,
                                      (size_t)PP_SLOTS * PP_SLOT);
}

}  // namespace brg
