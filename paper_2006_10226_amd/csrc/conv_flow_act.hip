// Instantiations of the short-loop kernel (conv_flow_kernel.h) for matrix
// products whose epilogue applies an activation by table.
#include "conv_flow_kernel.h"

namespace qnn {

hipError_t launch_conv_flow_act(const ConvArgs &a, int tile, hipStream_t st)
{
    if (!a.act || a.res)
        return hipErrorInvalidValue;
    return launch_flow_act_from<0, false>(a, tile, st);
}

}  // namespace qnn
