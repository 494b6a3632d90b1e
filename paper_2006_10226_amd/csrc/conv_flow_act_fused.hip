// Instantiations of the short-loop kernel (conv_flow_kernel.h) for matrix
// products whose epilogue applies an activation by table, then a residual
// qnn.add.
#include "conv_flow_kernel.h"

namespace qnn {

hipError_t launch_conv_flow_act_fused(const ConvArgs &a, int tile, hipStream_t st)
{
    if (!a.act || !a.res || !a.staged)
        return hipErrorInvalidValue;
    return launch_flow_act_from<0, true>(a, tile, st);
}

}  // namespace qnn
