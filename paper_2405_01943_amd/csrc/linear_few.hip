// Products with few output tiles: the forward product of few rows (bf16, f32) and small f32 products of every kind.
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

template <typename T_, Product PRODUCT, int TB, int CB, int WAVES, int PAIRS>
__global__ __launch_bounds__(64 * WAVES) void product_few_kernel(const Operands<T_> a, const Epilogue<T_> ep, uint32_t tiles_c)
{
    typedef Few<T_> F;
    constexpr bool P_ROWS = PRODUCT != kWeightGrad, Q_ROWS = PRODUCT == kForward;   // stored row by row
    static_assert(PRODUCT == kForward || sizeof(T_) == 4, "k by k in f32 only");
    const int lane = threadIdx.x & 63, fr = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t tile_r = blockIdx.x / tiles_c, tile_c = blockIdx.x - tile_r * tiles_c;
    int expert;
    int64_t r0, r_end, k0 = 0, k_end = a.depth;
    if constexpr (PRODUCT == kWeightGrad) {
        expert = blockIdx.y;
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
    __shared__ f32x4 sums[WAVES][CB * TB][64];
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

template <typename T_, Product PRODUCT, int TB, int CB, int WAVES, int PAIRS>
static dass_status launch(const char *fn, const Operands<T_> &a, const Epilogue<T_> &ep, hipStream_t stream)
{
    const int64_t tiles_r = PRODUCT == kWeightGrad ? (a.out_rows + 16 * TB - 1) / (16 * TB) : tile_numbers(a.seg, 16 * TB);
    const int64_t tiles_c = (ep.cols + 16 * CB - 1) / (16 * CB);
    const unsigned experts = PRODUCT == kWeightGrad ? a.seg.n : 1;
    if (tiles_r > 0xffffffffLL / (64 * WAVES) / tiles_c / experts)
        return fail(DASS_ERR_SHAPE, "%s: too many tiles for one launch; split the rows", fn);
    hipLaunchKernelGGL((product_few_kernel<T_, PRODUCT, TB, CB, WAVES, PAIRS>), dim3((unsigned)(tiles_r * tiles_c), experts),
                       dim3(64 * WAVES), 0, stream, a, ep, (uint32_t)tiles_c);
    return check_launch("few-tile product kernel");
}

// Wavefronts of a workgroup and loads that each has on its way, in graphs: one row of 4096 x 11008 4 wavefronts x 8 fragments 20.0 us, 8
// x 4 19.1, 16 x 4 17.7; of 4096 x 4096 9.4, 8.8, 8.3; but of 1024 x 4096 4.0 (x 4 3.9), 4.0, 5.1, four rows of 512 x 512 3.4 (x 4
// 2.8), 3.4, 3.6.
dass_status launch_few(const char *fn, Product, const Plan &, const Operands<uint16_t> &a, const Epilogue<uint16_t> &ep, hipStream_t stream)
{
    if (a.depth >= 4096)
        return launch<uint16_t, kForward, 1, 1, 16, 2>(fn, a, ep, stream);
    return launch<uint16_t, kForward, 1, 1, 4, 2>(fn, a, ep, stream);
}

// The same in f32, 8 wavefronts against 4 with twice the loads: 16 rows of 1024 x 1024 5.7 and 6.9 us, 301 of 256 x 688 (blocks of 32) 4.7
// and 5.2, its dX 7.7 and 9.1, dW 5.3 and 6.6.
template <int BLOCKS>
static dass_status launch_blocks(const char *fn, Product product, const Operands<float> &a, const Epilogue<float> &ep, hipStream_t stream)
{
    if (product == kForward)
        return launch<float, kForward, BLOCKS, BLOCKS, 8, 2 / BLOCKS>(fn, a, ep, stream);
    if (product == kInputGrad)
        return launch<float, kInputGrad, BLOCKS, BLOCKS, 8, 2 / BLOCKS>(fn, a, ep, stream);
    return launch<float, kWeightGrad, BLOCKS, BLOCKS, 8, 2 / BLOCKS>(fn, a, ep, stream);
}

dass_status launch_few(const char *fn, Product product, const Plan &plan, const Operands<float> &a, const Epilogue<float> &ep,
                       hipStream_t stream)
{
    return plan.blocks == 1 ? launch_blocks<1>(fn, product, a, ep, stream) : launch_blocks<2>(fn, product, a, ep, stream);
}

}  // namespace dass
