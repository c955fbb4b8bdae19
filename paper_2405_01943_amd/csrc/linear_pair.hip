// linear_tiles.h: both products and the bias sums of a small gradient in one launch (bf16).  None needs another's result, and
// neither product has tiles enough to fill the chip (pair_of in linear.hip has the sizes and what they measured).
#include "linear_tiles.h"

namespace dass {

// Workgroups 0 .. x - 1 dX's, the next w dW's, `each` an expert, the rest the bias sums'.
struct PairParts {
    TileOrder x_order, w_order;
    uint32_t x, w, each, bias_strips;
};

template <bool SHORT>
__global__ __launch_bounds__(256) void product_pair_kernel(const Operands<uint16_t> ax, const Epilogue<uint16_t> ex,
                                                           const Operands<uint16_t> aw, const Epilogue<uint16_t> ew,
                                                           const BiasSums bias, const PairParts parts)
{
    const Split whole = {nullptr, 0, 1};
    uint32_t i = blockIdx.x;
    if (i < parts.x) {
        product_tile<uint16_t, kInputGrad, 4, 4, SHORT>(ax, ex, parts.x_order, whole, i, 0, 0);
        return;
    }
    i -= parts.x;
    if (i < parts.w) {
        const uint32_t expert = i / parts.each;
        product_tile<uint16_t, kWeightGrad, 4, 4, SHORT>(aw, ew, parts.w_order, whole, i - expert * parts.each, expert, 0);
        return;
    }
    i -= parts.w;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const uint32_t expert = i / parts.bias_strips;
    sum_bias<uint16_t>(bias, i - expert * parts.bias_strips, expert, reinterpret_cast<float(*)[64]>(lds));
}

template <bool SHORT>
static dass_status launch(const char *fn, const Operands<uint16_t> &ax, const Epilogue<uint16_t> &ex, const Operands<uint16_t> &aw,
                          const Epilogue<uint16_t> &ew, const BiasSums &bias, hipStream_t stream)
{
    PairParts parts = {};
    parts.x_order = order_tiles<uint16_t, kInputGrad, 128, 128>(ax, ex);
    parts.w_order = order_tiles<uint16_t, kWeightGrad, 128, 128>(aw, ew);
    const int64_t strips = (bias.cols + 63) / 64, sums = bias.dbias ? strips * bias.seg.n : 0;
    const int64_t w = (int64_t)parts.w_order.blocks * aw.seg.n;
    if (parts.x_order.blocks == 0 || parts.w_order.blocks == 0 || parts.x_order.blocks + w + sums > 0xffffffffLL / 256)
        return fail(DASS_ERR_SHAPE, "%s: too many tiles for one launch; split the rows", fn);
    const dass_status s = reserve_lds<product_pair_kernel<SHORT>, lds_bytes<SHORT>()>(fn);
    if (s != DASS_OK)
        return s;
    parts.x = parts.x_order.blocks;
    parts.each = parts.w_order.blocks;
    parts.w = (uint32_t)w;
    parts.bias_strips = (uint32_t)strips;
    hipLaunchKernelGGL(product_pair_kernel<SHORT>, dim3((unsigned)(parts.x + w + sums)), dim3(256), lds_bytes<SHORT>(), stream,
                       ax, ex, aw, ew, bias, parts);
    return check_launch("gradient kernel");
}

dass_status launch_pair(const char *fn, bool short_tiles, const Operands<uint16_t> &ax, const Epilogue<uint16_t> &ex,
                        const Operands<uint16_t> &aw, const Epilogue<uint16_t> &ew, const BiasSums &bias, hipStream_t stream)
{
    return short_tiles ? launch<true>(fn, ax, ex, aw, ew, bias, stream) : launch<false>(fn, ax, ex, aw, ew, bias, stream);
}

}  // namespace dass
