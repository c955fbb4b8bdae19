// linear_tiles.h: the product itself.
#include "linear_tiles.h"

namespace dass {

dass_status launch_forward(const char *fn, const Plan &plan, const Operands<uint16_t> &a, const Epilogue<uint16_t> &ep, const Split &split,
                           hipStream_t stream)
{
    return launch_plan<uint16_t, kForward>(fn, plan, a, ep, split, stream);
}

dass_status launch_forward(const char *fn, const Plan &plan, const Operands<float> &a, const Epilogue<float> &ep, const Split &split,
                           hipStream_t stream)
{
    return launch_plan<float, kForward>(fn, plan, a, ep, split, stream);
}

}  // namespace dass
