// dass_linear and dass_linear_backward in f32 on the f32 matrix instruction (256 flop a clock and compute unit).
//
// A workgroup owns TILE x TILE outputs, its four wavefronts a quarter each; slabs of 32 k of both operands go through
// registers into LDS, one slab ahead.  An operand that is contiguous in k lies there by rows and one 16-byte read
// gives a lane four k (4 g .. 4 g + 3 of 16, g = lane / 16); one that is stored k by k lies there k by k and the same four k are
// four reads.  The i-th of the four goes into the i-th v_mfma_f32_16x16x4_f32 of the 16, which so covers k = i, 4 + i,
// 8 + i, 12 + i of both operands.  Rows are padded by four floats: reads and writes meet no bank twice.  Output
// columns are the instruction's M index: a lane holds four neighbouring ones of one row and finishes them in registers.
#include "linear.h"

namespace dass {

constexpr int kDepth = 32;   // k of a slab

template <typename T_, Product PRODUCT, int TILE>
__global__ __launch_bounds__(256) void product_f32_kernel(const Operands<T_> a, const Epilogue<T_> ep, uint32_t tiles_c)
{
    constexpr bool P_ROWS = PRODUCT != kWeightGrad, Q_ROWS = PRODUCT == kForward;   // stored row by row
    constexpr int BY_ROW = kDepth + 4, BY_K = TILE + 4;   // LDS strides
    constexpr int P_SIZE = P_ROWS ? TILE * BY_ROW : kDepth * BY_K, Q_SIZE = Q_ROWS ? TILE * BY_ROW : kDepth * BY_K;
    constexpr int LOADS = TILE * kDepth / 4 / 256, B = TILE / 32;
    __shared__ __attribute__((aligned(16))) float lds[2][P_SIZE + Q_SIZE];

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t tile_r = blockIdx.x / tiles_c, tile_c = blockIdx.x - tile_r * tiles_c;
    int expert;
    int64_t r0, r_end, k0, k_end;
    if constexpr (PRODUCT == kWeightGrad) {
        expert = blockIdx.y;
        const Span k = segment(a.seg, expert);
        k0 = k.lo;
        k_end = k.hi;
        r0 = (int64_t)tile_r * TILE;
        r_end = a.out_rows;
    } else {
        Span r;
        if (!rows_of_tile(a.seg, tile_r, TILE, expert, r))
            return;
        r0 = r.lo;
        r_end = r.hi;
        k0 = 0;
        k_end = a.depth;
    }
    const int64_t c0 = (int64_t)tile_c * TILE;
    const T_ *Q = PRODUCT == kWeightGrad ? a.Q : a.Q + (int64_t)expert * a.q_stride;

    // Rows and columns past the end read the last one's: what they give is not stored.  k past the end becomes 0.
    f32x4 st[2][LOADS];
    auto load = [&](const T_ *base, int64_t ld, bool by_row, int64_t m0, int64_t m_end, int64_t k, int p) {
        const int i = tid + p * 256;
        if (by_row) {
            const int64_t m = m0 + i / (kDepth / 4), kk = k + i % (kDepth / 4) * 4;
            const f32x4 v = load4(base + (m < m_end ? m : m_end - 1) * ld + (kk < k_end ? kk : k0));
            return kk < k_end ? v : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
        const int64_t kk = k + i / (TILE / 4), m = m0 + i % (TILE / 4) * 4;
        const f32x4 v = load4(base + (kk < k_end ? kk : k0) * ld + (m < m_end ? m : m_end - 4));
        return kk < k_end ? v : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    };
    auto fetch = [&](int64_t k) {
#pragma unroll
        for (int p = 0; p < LOADS; ++p) {
            st[0][p] = load(a.P, a.ldp, P_ROWS, r0, r_end, k, p);
            st[1][p] = load(Q, a.ldq, Q_ROWS, c0, ep.cols, k, p);
        }
    };
    auto place = [&](float *dst, bool by_row, const f32x4 &v, int p) {
        const int i = tid + p * 256;
        if (by_row)
            *reinterpret_cast<f32x4 *>(dst + i / (kDepth / 4) * BY_ROW + i % (kDepth / 4) * 4) = v;
        else
            *reinterpret_cast<f32x4 *>(dst + i / (TILE / 4) * BY_K + i % (TILE / 4) * 4) = v;
    };
    auto stage = [&](int buf) {
#pragma unroll
        for (int p = 0; p < LOADS; ++p) {
            place(lds[buf], P_ROWS, st[0][p], p);
            place(lds[buf] + P_SIZE, Q_ROWS, st[1][p], p);
        }
    };

    f32x4 acc[B][B];   // [column block][row block]
#pragma unroll
    for (int i = 0; i < B; ++i)
#pragma unroll
        for (int j = 0; j < B; ++j)
            acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const int fr = lane & 15, g = lane >> 4, wr = wave >> 1, wc = wave & 1;
    auto fragment = [&](const float *src, bool by_row, int m, int kk) {
        if (by_row)
            return *reinterpret_cast<const f32x4 *>(src + m * BY_ROW + kk + 4 * g);
        f32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            v[i] = src[(kk + 4 * g + i) * BY_K + m];
        return v;
    };

    if (k0 < k_end) {
        fetch(k0);
        stage(0);
    }
    __syncthreads();
    int buf = 0;
    for (int64_t k = k0; k < k_end; k += kDepth, buf ^= 1) {
        const bool more = k + kDepth < k_end;
        if (more)
            fetch(k + kDepth);
#pragma unroll
        for (int kk = 0; kk < kDepth; kk += 16) {
            f32x4 pf[B], qf[B];
#pragma unroll
            for (int i = 0; i < B; ++i) {
                pf[i] = fragment(lds[buf], P_ROWS, wr * (TILE / 2) + i * 16 + fr, kk);
                qf[i] = fragment(lds[buf] + P_SIZE, Q_ROWS, wc * (TILE / 2) + i * 16 + fr, kk);
            }
#pragma unroll
            for (int x = 0; x < 4; ++x)
#pragma unroll
                for (int i = 0; i < B; ++i)
#pragma unroll
                    for (int j = 0; j < B; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(qf[i][x], pf[j][x], acc[i][j], 0, 0, 0);
        }
        if (more)
            stage(buf ^ 1);
        __syncthreads();
    }

    Epilogue<T_> e2 = ep;
    if constexpr (PRODUCT == kWeightGrad)
        e2.out += (int64_t)expert * a.out_stride;
#pragma unroll
    for (int j = 0; j < B; ++j) {
        const int64_t r = r0 + wr * (TILE / 2) + j * 16 + fr;
#pragma unroll
        for (int i = 0; i < B; ++i) {
            const int64_t c = c0 + wc * (TILE / 2) + i * 16 + 4 * g;
            if (r < r_end && c < ep.cols)
                finish4(e2, expert, r, c, acc[i][j]);
        }
    }
}

template <typename T_, Product PRODUCT, int TILE>
static dass_status launch_tile(const char *fn, const Operands<T_> &a, const Epilogue<T_> &ep, hipStream_t stream)
{
    const int64_t tiles_r = PRODUCT == kWeightGrad ? (a.out_rows + TILE - 1) / TILE : tile_numbers(a.seg, TILE);
    const int64_t tiles_c = (ep.cols + TILE - 1) / TILE;
    if (tiles_r > 0xffffffffLL / 256 / tiles_c)
        return fail(DASS_ERR_SHAPE, "%s: too many tiles for one launch; split the rows", fn);
    hipLaunchKernelGGL((product_f32_kernel<T_, PRODUCT, TILE>), dim3((unsigned)(tiles_r * tiles_c), PRODUCT == kWeightGrad ? a.seg.n : 1),
                       dim3(256), 0, stream, a, ep, (uint32_t)tiles_c);
    return check_launch("f32 product kernel");
}

template <typename T_>
static dass_status launch_any(const char *fn, Product product, const Operands<T_> &a, const Epilogue<T_> &ep, hipStream_t stream)
{
    if (product == kForward)
        return launch_tile<T_, kForward, 64>(fn, a, ep, stream);
    if (product == kInputGrad)
        return launch_tile<T_, kInputGrad, 64>(fn, a, ep, stream);
    return launch_tile<T_, kWeightGrad, 64>(fn, a, ep, stream);
}

dass_status launch_product_f32(const char *fn, Product product, const Operands<float> &a, const Epilogue<float> &ep,
                               hipStream_t stream)
{
    return launch_any(fn, product, a, ep, stream);
}

}  // namespace dass
