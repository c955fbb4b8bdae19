// linear_tiles.h: the gradient of the layer's weights.
#include "linear_tiles.h"

namespace dass {

dass_status launch_dw(const char *fn, const Plan &plan, const Operands<uint16_t> &a, const Epilogue<uint16_t> &ep, const Split &split,
                           hipStream_t stream)
{
    return launch_plan<uint16_t, kWeightGrad>(fn, plan, a, ep, split, stream);
}

dass_status launch_dw(const char *fn, const Plan &plan, const Operands<float> &a, const Epilogue<float> &ep, const Split &split,
                           hipStream_t stream)
{
    return launch_plan<float, kWeightGrad>(fn, plan, a, ep, split, stream);
}

}  // namespace dass
