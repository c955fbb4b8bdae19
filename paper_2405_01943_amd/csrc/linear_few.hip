// Products with few output tiles: the forward product of few rows (bf16, f32) and small f32 products of every kind.  A gradient's
// two products and its bias sums are parts of one launch, as none needs another's result: a gradient of 301 rows of 256 x 688 with
// its bias 12.1 us in graphs, 19.6 with three launches (7.7, 5.3 and 2.6 us of them), of 1024 rows of 512 x 512 22.5 and 28.5.
//
// A workgroup owns 16 TB rows x 16 CB columns of the output and its WAVES wavefronts split k between them, so that a
// grid of few tiles still has loads on their way in every compute unit; the partial sums meet in LDS once.  Fragments
// come straight from global memory (each is used by one wavefront alone, so LDS would only add a trip): lane l of a
// fragment holds 16 bytes of row l % 16, k = 4 (8 for bf16) (l / 16) .. of 16 (32), two fragments of a row side by side are
// a 128-byte line, and the wavefronts take these lines in turn.  For one token the weights are all there is to read: the
// kernel's time is theirs.  Stored k by k (f32 only), the four k of a lane are four 4-byte loads.
#include "linear.h"

namespace dass {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;

template <typename T_>
struct Few;
template <>
struct Few<uint16_t> {
    static constexpr int K = 32, LANE = 8;   // k of a fragment, of a lane of it
    static __device__ __forceinline__ f32x4 multiply(const u32x4 &q, const u32x4 &p, const f32x4 &acc)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, q), __builtin_bit_cast(bf16x8, p), acc, 0, 0, 0);
    }
};
template <>
struct Few<float> {
    static constexpr int K = 16, LANE = 4;
    static __device__ __forceinline__ f32x4 multiply(const u32x4 &q, const u32x4 &p, f32x4 acc)
    {
        const f32x4 a = __builtin_bit_cast(f32x4, q), b = __builtin_bit_cast(f32x4, p);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], acc, 0, 0, 0);
        return acc;
    }
};

// One workgroup's tile; `expert` is given for dW and found for the others.
template <typename T_, Product PRODUCT, int TB, int CB, int WAVES, int PAIRS>
__device__ __forceinline__ void few_tile(const Operands<T_> &a, const Epilogue<T_> &ep, uint32_t tile_r, uint32_t tile_c, int expert,
                                         f32x4 *lds)
{
    typedef Few<T_> F;
    constexpr bool P_ROWS = PRODUCT != kWeightGrad, Q_ROWS = PRODUCT == kForward;   // stored row by row
    static_assert(PRODUCT == kForward || sizeof(T_) == 4, "k by k in f32 only");
    const int lane = threadIdx.x & 63, fr = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int64_t r0, r_end, k0 = 0, k_end = a.depth;
    if constexpr (PRODUCT == kWeightGrad) {
        const Span k = segment(a.seg, expert);
        k0 = k.lo;
        k_end = k.hi;
        r0 = (int64_t)tile_r * 16 * TB;
        r_end = a.out_rows;
    } else {
        Span r;
        if (!rows_of_tile(a.seg, tile_r, 16 * TB, expert, r))
            return;
        r0 = r.lo;
        r_end = r.hi;
    }
    const int64_t c0 = (int64_t)tile_c * 16 * CB;
    const T_ *Q = PRODUCT == kWeightGrad ? a.Q : a.Q + (int64_t)expert * a.q_stride;

    // Rows and columns past the end read the last one's: what they give is not stored.  k past the end becomes 0.
    const T_ *p_row[TB], *q_row[CB];
#pragma unroll
    for (int j = 0; j < TB; ++j) {
        const int64_t r = r0 + 16 * j + fr, rr = r < r_end ? r : r_end - 1;
        p_row[j] = a.P + (P_ROWS ? rr * a.ldp : rr);
    }
#pragma unroll
    for (int i = 0; i < CB; ++i) {
        const int64_t c = c0 + 16 * i + fr, cc = c < ep.cols ? c : ep.cols - 1;
        q_row[i] = Q + (Q_ROWS ? cc * a.ldq : cc);
    }
    auto load = [&](const T_ *row, int64_t ld, auto by_rows, int64_t k) __attribute__((always_inline)) {
        if constexpr (decltype(by_rows)::value) {
            const bool in = k < k_end;
            const u32x4 v = *reinterpret_cast<const u32x4 *>(row + (in ? k : k0));
            return in ? v : u32x4{0, 0, 0, 0};
        } else {
            u32x4 v;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool in = k + i < k_end;
                const uint32_t w = __builtin_bit_cast(uint32_t, (float)row[(in ? k + i : k0) * ld]);
                v[i] = in ? w : 0;
            }
            return v;
        }
    };

    f32x4 acc[CB][TB];
#pragma unroll
    for (int i = 0; i < CB; ++i)
#pragma unroll
        for (int j = 0; j < TB; ++j)
            acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    constexpr int PAIR = 2 * F::K;
    for (int64_t k = k0 + wave * PAIR; k < k_end; k += (int64_t)WAVES * PAIR * PAIRS) {
        u32x4 p[2 * PAIRS][TB], q[2 * PAIRS][CB];
#pragma unroll
        for (int x = 0; x < 2 * PAIRS; ++x) {
            const int64_t kk = k + (int64_t)(x / 2) * WAVES * PAIR + x % 2 * F::K + g * F::LANE;
#pragma unroll
            for (int i = 0; i < CB; ++i)
                q[x][i] = load(q_row[i], a.ldq, std::integral_constant<bool, Q_ROWS>{}, kk);
#pragma unroll
            for (int j = 0; j < TB; ++j)
                p[x][j] = load(p_row[j], a.ldp, std::integral_constant<bool, P_ROWS>{}, kk);
        }
#pragma unroll
        for (int x = 0; x < 2 * PAIRS; ++x)
#pragma unroll
            for (int i = 0; i < CB; ++i)
#pragma unroll
                for (int j = 0; j < TB; ++j)
                    acc[i][j] = F::multiply(q[x][i], p[x][j], acc[i][j]);
    }

    // The partial sums meet: a thread adds up four neighbouring columns of one row, in the order of the wavefronts.
    auto sums = reinterpret_cast<f32x4(*)[CB * TB][64]>(lds);   // [WAVES]
#pragma unroll
    for (int i = 0; i < CB; ++i)
#pragma unroll
        for (int j = 0; j < TB; ++j)
            sums[wave][i * TB + j][lane] = acc[i][j];
    __syncthreads();
    Epilogue<T_> e2 = ep;
    if constexpr (PRODUCT == kWeightGrad)
        e2.out += (int64_t)expert * a.out_stride;
    for (int b = wave; b < CB * TB; b += WAVES) {
        f32x4 s = sums[0][b][lane];
#pragma unroll
        for (int w = 1; w < WAVES; ++w)
            s += sums[w][b][lane];
        const int64_t r = r0 + 16 * (b % TB) + fr, c = c0 + 16 * (b / TB) + 4 * g;
        if (r < r_end && c < ep.cols)
            finish4(e2, expert, r, c, s);
    }
}

// Wavefronts of a workgroup in f32, with the loads that each has on its way where the blocks are small.  8 against 4 with twice the
// loads: 16 rows of 1024 x 1024 5.7 and 6.9 us, 301 of 256 x 688 (blocks of 32) 4.7 and 5.2.  16 read no more at a time and have
// more sums to add: the gradient of 16 rows of 1024 x 1024 10.5 us, with 16 13.2 (100 of 64 x 4096 23.9 and 18.6).
constexpr int kFewWaves = 8;
static constexpr int few_pairs(int blocks) { return 2 / blocks; }

template <typename T_, int BLOCKS, int WAVES, int PAIRS>
__global__ __launch_bounds__(64 * WAVES) void few_forward_kernel(const Operands<T_> a, const Epilogue<T_> ep, uint32_t tiles_c)
{
    __shared__ f32x4 lds[WAVES * BLOCKS * BLOCKS * 64];
    const uint32_t tile_r = blockIdx.x / tiles_c;
    few_tile<T_, kForward, BLOCKS, BLOCKS, WAVES, PAIRS>(a, ep, tile_r, blockIdx.x - tile_r * tiles_c, 0, lds);
}

// Workgroups 0 .. x - 1 dX's, the next w dW's, expert by expert, the rest the bias sums'.
struct FewParts {
    uint32_t x, x_cols, w, w_rows, w_cols, bias_strips;
};

template <int BX, int BW>
__global__ __launch_bounds__(64 * kFewWaves) void few_grad_kernel(const Operands<float> ax, const Epilogue<float> ex,
                                                                  const Operands<float> aw, const Epilogue<float> ew, const BiasSums bias,
                                                                  const FewParts parts)
{
    constexpr int MOST = BX > BW ? BX : BW;
    __shared__ f32x4 lds[kFewWaves * MOST * MOST * 64];
    uint32_t i = blockIdx.x;
    if (i < parts.x) {
        const uint32_t tile_r = i / parts.x_cols;
        few_tile<float, kInputGrad, BX, BX, kFewWaves, few_pairs(BX)>(ax, ex, tile_r, i - tile_r * parts.x_cols, 0, lds);
        return;
    }
    i -= parts.x;
    if (i < parts.w) {
        const uint32_t line = i / parts.w_cols, expert = line / parts.w_rows;
        few_tile<float, kWeightGrad, BW, BW, kFewWaves, few_pairs(BW)>(aw, ew, line - expert * parts.w_rows, i - line * parts.w_cols,
                                                                       expert, lds);
        return;
    }
    i -= parts.w;
    const uint32_t expert = i / parts.bias_strips;
    sum_bias<float>(bias, i - expert * parts.bias_strips, expert, reinterpret_cast<float(*)[64]>(lds));
}

template <typename T_, int BLOCKS, int WAVES, int PAIRS>
static dass_status launch_rows(const char *fn, const Operands<T_> &a, const Epilogue<T_> &ep, hipStream_t stream)
{
    const int64_t tiles_r = tile_numbers(a.seg, 16 * BLOCKS), tiles_c = (ep.cols + 16 * BLOCKS - 1) / (16 * BLOCKS);
    if (tiles_r > 0xffffffffLL / (64 * WAVES) / tiles_c)
        return fail(DASS_ERR_SHAPE, "%s: too many tiles for one launch; split the rows", fn);
    hipLaunchKernelGGL((few_forward_kernel<T_, BLOCKS, WAVES, PAIRS>), dim3((unsigned)(tiles_r * tiles_c)), dim3(64 * WAVES), 0, stream, a,
                       ep, (uint32_t)tiles_c);
    return check_launch("few-tile product kernel");
}

// Wavefronts of a workgroup and loads that each has on its way, in graphs: one row of 4096 x 11008 4 wavefronts x 8 fragments 20.0
// us, 8 x 4 19.1, 16 x 4 17.7; of 4096 x 4096 9.4, 8.8, 8.3; but of 1024 x 4096 4.0 (x 4 3.9), 4.0, 5.1, four rows of 512 x 512
// 3.4 (x 4 2.8), 3.4, 3.6.  At the limit, 4 and 16 wavefronts on weights that no cache holds: one row to 14336 columns from 1536 11.8 and
// 13.8, 2048 15.6 and 14.0, 2560 17.9 and 18.8, 3584 22.3 and 23.4, 4096 25.0 and 23.6, 5120 31.0 and 33.1, 8192 52.2 and 45.4; 16 rows
// over 8 experts to 4096 columns from 2048 27.8 and 30.4, 3584 42.6 and 45.4, 4096 48.4 and 44.9, 8192 101 and 89.  (16 wavefronts take
// 2048 of k at a time, so that they lead at its multiples, and lose up to a tenth between them.)
dass_status launch_few(const char *fn, const Plan &, const Operands<uint16_t> &a, const Epilogue<uint16_t> &ep, hipStream_t stream)
{
    if (a.depth >= 4096)
        return launch_rows<uint16_t, 1, 16, 2>(fn, a, ep, stream);
    return launch_rows<uint16_t, 1, 4, 2>(fn, a, ep, stream);
}

dass_status launch_few(const char *fn, const Plan &plan, const Operands<float> &a, const Epilogue<float> &ep, hipStream_t stream)
{
    if (plan.blocks == 1)
        return launch_rows<float, 1, kFewWaves, few_pairs(1)>(fn, a, ep, stream);
    return launch_rows<float, 2, kFewWaves, few_pairs(2)>(fn, a, ep, stream);
}

template <int BX, int BW>
static dass_status launch_grads(const char *fn, const FewGrads &f, hipStream_t stream)
{
    const auto pieces = [](int64_t n, int64_t of) { return (n + of - 1) / of; };
    const int64_t x_cols = pieces(f.ex.cols, 16 * BX), x = f.blocks_x ? tile_numbers(f.x.seg, 16 * BX) * x_cols : 0;
    const int64_t w_rows = pieces(f.w.out_rows, 16 * BW), w_cols = pieces(f.ew.cols, 16 * BW);
    const int64_t w = f.blocks_w ? w_rows * w_cols * f.w.seg.n : 0;
    const int64_t strips = pieces(f.bias.cols, 64), bias = f.bias.dbias ? strips * f.bias.seg.n : 0;
    if (x + w + bias > 0xffffffffLL / (64 * kFewWaves))
        return fail(DASS_ERR_SHAPE, "%s: too many tiles for one launch; split the rows", fn);
    const FewParts parts = {(uint32_t)x, (uint32_t)x_cols, (uint32_t)w, (uint32_t)w_rows, (uint32_t)w_cols, (uint32_t)strips};
    hipLaunchKernelGGL((few_grad_kernel<BX, BW>), dim3((unsigned)(x + w + bias)), dim3(64 * kFewWaves), 0, stream, f.x, f.ex, f.w, f.ew,
                       f.bias, parts);
    return check_launch("few-tile gradient kernel");
}

dass_status launch_few_grads(const char *fn, const FewGrads &f, hipStream_t stream)
{
    const int bx = f.blocks_x ? f.blocks_x : f.blocks_w, bw = f.blocks_w ? f.blocks_w : f.blocks_x;
    if (bx == 1)
        return bw == 1 ? launch_grads<1, 1>(fn, f, stream) : launch_grads<1, 2>(fn, f, stream);
    return bw == 1 ? launch_grads<2, 1>(fn, f, stream) : launch_grads<2, 2>(fn, f, stream);
}

}  // namespace dass
