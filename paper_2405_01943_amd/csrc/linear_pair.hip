// linear_tiles.h: both products and the bias sums of a gradient in one launch (bf16).  None needs another's result, so that the
// tiles of the one fill the rounds that the other leaves (pair_of in linear.hip has the sizes and what they measured).
#include "linear_tiles.h"

namespace dass {

// Workgroups of dX, of dW (`each` an expert) and, at the end, of the bias sums.  The product with more k comes first, so that short
// tiles fill the last round.
struct PairParts {
    TileOrder x_order, w_order;
    uint32_t x, w, each, bias_strips;
    bool w_first;
};

template <int RB, int CB, bool SHORT>
__global__ __launch_bounds__(256) void product_pair_kernel(const Operands<uint16_t> ax, const Epilogue<uint16_t> ex,
                                                           const Operands<uint16_t> aw, const Epilogue<uint16_t> ew,
                                                           const BiasSums bias, const PairParts parts)
{
    const Split whole = {nullptr, 0, 1};
    const uint32_t i = blockIdx.x, x = parts.w_first ? i - parts.w : i, w = parts.w_first ? i : i - parts.x;
    if (x < parts.x) {   // (below 0 is beyond)
        product_tile<uint16_t, kInputGrad, RB, CB, SHORT>(ax, ex, parts.x_order, whole, x, 0, 0);
        return;
    }
    if (w < parts.w) {
        const uint32_t expert = w / parts.each;
        product_tile<uint16_t, kWeightGrad, RB, CB, SHORT>(aw, ew, parts.w_order, whole, w - expert * parts.each, expert, 0);
        return;
    }
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const uint32_t sum = i - parts.x - parts.w, expert = sum / parts.bias_strips;
    sum_bias<uint16_t>(bias, sum - expert * parts.bias_strips, expert, reinterpret_cast<float(*)[64]>(lds));
}

template <int RB, int CB, bool SHORT = false>
static dass_status launch(const char *fn, const Operands<uint16_t> &ax, const Epilogue<uint16_t> &ex, const Operands<uint16_t> &aw,
                          const Epilogue<uint16_t> &ew, const BiasSums &bias, hipStream_t stream)
{
    PairParts parts = {};
    parts.x_order = order_tiles<uint16_t, kInputGrad, 32 * RB, 32 * CB>(ax, ex);
    parts.w_order = order_tiles<uint16_t, kWeightGrad, 32 * RB, 32 * CB>(aw, ew);
    const int64_t strips = (bias.cols + 63) / 64, sums = bias.dbias ? strips * bias.seg.n : 0;
    const int64_t w = (int64_t)parts.w_order.blocks * aw.seg.n;
    if (parts.x_order.blocks == 0 || parts.w_order.blocks == 0 || parts.x_order.blocks + w + sums > 0xffffffffLL / 256)
        return fail(DASS_ERR_SHAPE, "%s: too many tiles for one launch; split the rows", fn);
    const dass_status s = reserve_lds<product_pair_kernel<RB, CB, SHORT>, lds_bytes<SHORT>()>(fn);
    if (s != DASS_OK)
        return s;
    parts.x = parts.x_order.blocks;
    parts.each = parts.w_order.blocks;
    parts.w = (uint32_t)w;
    parts.bias_strips = (uint32_t)strips;
    parts.w_first = ax.depth < aw.seg.rows / aw.seg.n;
    hipLaunchKernelGGL((product_pair_kernel<RB, CB, SHORT>), dim3((unsigned)(parts.x + w + sums)), dim3(256), lds_bytes<SHORT>(), stream,
                       ax, ex, aw, ew, bias, parts);
    return check_launch("gradient kernel");
}

dass_status launch_pair(const char *fn, int tile, const Operands<uint16_t> &ax, const Epilogue<uint16_t> &ex, const Operands<uint16_t> &aw,
                        const Epilogue<uint16_t> &ew, const BiasSums &bias, hipStream_t stream)
{
    if (tile == 0)
        return launch<8, 8>(fn, ax, ex, aw, ew, bias, stream);
    if (tile == 1)
        return launch<4, 8>(fn, ax, ex, aw, ew, bias, stream);
    return tile == 2 ? launch<4, 4>(fn, ax, ex, aw, ew, bias, stream) : launch<4, 4, true>(fn, ax, ex, aw, ew, bias, stream);
}

}  // namespace dass
