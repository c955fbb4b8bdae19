// What the kernels of dass_linear and dass_linear_backward share: rows that are grouped by expert, the epilogue, and the
// launches behind the entry points.
#pragma once

#include "activations.h"
#include "chunk.h"
#include "dass_internal.h"

#include <type_traits>

namespace dass {

typedef __attribute__((ext_vector_type(4))) float f32x4;

// Rows [offsets[e], offsets[e + 1]) belong to expert e; offsets = nullptr: all rows to one.  The bounds are held to
// [0, rows] whatever the array holds, so that no row outside the matrices is ever addressed.
struct Segments {
    const int32_t *offsets;
    int64_t rows;
    int n;
};

struct Span {
    int64_t lo, hi;
};

__device__ __forceinline__ Span segment(const Segments &s, int e)
{
    if (!s.offsets)
        return {0, s.rows};
    const int64_t a = s.offsets[e], b = s.offsets[e + 1];
    const int64_t lo = a < 0 ? 0 : a < s.rows ? a : s.rows, hi = b < lo ? lo : b < s.rows ? b : s.rows;
    return {lo, hi};
}

// Tiles of `bm` rows that do not cross experts, numbered without a scan: expert e's first tile is number
// floor(lo_e / bm) + e.  These numbers rise by more than an expert has tiles (ceil(n / bm) <= floor((lo + n) / bm) -
// floor(lo / bm) + 1), so floor(rows / bm) + n numbers hold every tile, some of them none.  A wavefront finds the
// expert of a number by counting the first tiles that are not beyond it, 64 experts at a time.
__device__ __forceinline__ bool rows_of_tile(const Segments &s, int64_t number, int bm, int &expert, Span &span)
{
    expert = 0;
    if (!s.offsets) {
        span = {number * bm, s.rows};
        return span.lo < s.rows;
    }
    const int lane = threadIdx.x & 63;
    int n = 0;
    for (int e0 = 0; e0 < s.n; e0 += 64) {
        const int e = e0 + lane;
        int64_t lo = e < s.n ? s.offsets[e] : 0;
        lo = lo < 0 ? 0 : lo < s.rows ? lo : s.rows;
        n += __popcll(__ballot(e < s.n && lo / bm + e <= number));
    }
    if (n == 0)
        return false;   // offsets that do not begin with 0
    expert = __builtin_amdgcn_readfirstlane(n - 1);
    span = segment(s, expert);
    const int64_t nth = number - (span.lo / bm + expert);
    span.lo += nth * bm;
    return nth >= 0 && span.lo < span.hi;   // (offsets that fall have no tiles)
}

inline int64_t tile_numbers(const Segments &s, int64_t bm)
{
    return s.offsets ? s.rows / bm + s.n : (s.rows + bm - 1) / bm;
}

// The same tiles in a row, without the numbers that hold none: their count and the rows of the tile-th, by a scan over the
// experts.  For kernels that place tiles by their position in the list: tiles that are none, most of them with the smallest experts, left
// some XCDs with an eighth less to do than others.
struct TileList {
    int total, scan;   // scan: tiles of the first 64 experts up to and with this lane's

    static __device__ __forceinline__ int scan_64(const Segments &s, int e0, int bm, int &tiles)
    {
        const int lane = threadIdx.x & 63, e = e0 + lane;
        tiles = 0;
        if (e < s.n) {
            const Span r = segment(s, e);
            tiles = (int)((r.hi - r.lo + bm - 1) / bm);
        }
        int sum = tiles;
#pragma unroll
        for (int step = 1; step < 64; step *= 2) {
            const int up = __shfl_up(sum, step, 64);
            sum += lane >= step ? up : 0;
        }
        return sum;
    }
    __device__ __forceinline__ TileList(const Segments &s, int bm)
    {
        int tiles;
        scan = scan_64(s, 0, bm, tiles);
        int64_t sum = __builtin_amdgcn_readlane(scan, 63);
        for (int e0 = 64; e0 < s.n; e0 += 64)
            sum += __builtin_amdgcn_readlane(scan_64(s, e0, bm, tiles), 63);
        const int64_t most = s.rows / bm + s.n;   // (more where offsets fall)
        total = (int)(sum < most ? sum : most);
    }
    // `tile` below total
    __device__ __forceinline__ Span rows(const Segments &s, int bm, int tile, int &expert) const
    {
        int before = 0, e0 = 0, sum = scan, tiles;
        for (;;) {
            const int last = before + __builtin_amdgcn_readlane(sum, 63);
            if (tile < last || e0 + 64 >= s.n)
                break;
            before = last;
            e0 += 64;
            sum = scan_64(s, e0, bm, tiles);
        }
        const int below = __popcll(__ballot(before + sum <= tile));
        expert = e0 + below;
        if (below > 0)
            before += __builtin_amdgcn_readlane(sum, below - 1);
        Span r = segment(s, expert);
        r.lo += (int64_t)(tile - before) * bm;
        return r;
    }
};

// out = act(sum + bias) * mul + residual, pre = sum + bias.  Absent parts are nullptr.  All strides in elements.
template <typename T_>
struct Epilogue {
    T_ *out;
    int64_t ldo;
    const T_ *bias;        // [n_experts][cols]
    const T_ *mul;
    int64_t ldm;
    const T_ *residual;
    int64_t ldr;
    T_ *pre;
    int64_t ldp;
    int64_t cols;
    int act;
};

// Four neighbouring elements as f32 and back: 8 bytes of bf16, 16 of f32.
__device__ __forceinline__ f32x4 load4(const uint16_t *p)
{
    const uint2 c = *reinterpret_cast<const uint2 *>(p);
    return f32x4{__builtin_bit_cast(float, c.x << 16), __builtin_bit_cast(float, c.x & 0xffff0000u),
                 __builtin_bit_cast(float, c.y << 16), __builtin_bit_cast(float, c.y & 0xffff0000u)};
}
__device__ __forceinline__ f32x4 load4(const float *p) { return *reinterpret_cast<const f32x4 *>(p); }
__device__ __forceinline__ void store4(uint16_t *p, const f32x4 &v)
{
    typedef __attribute__((ext_vector_type(2))) float f2;
    typedef __attribute__((ext_vector_type(2))) __bf16 b2;
    uint2 c;
    c.x = __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{v[0], v[1]}, b2));
    c.y = __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{v[2], v[3]}, b2));
    *reinterpret_cast<uint2 *>(p) = c;
}
__device__ __forceinline__ void store4(float *p, const f32x4 &v) { *reinterpret_cast<f32x4 *>(p) = v; }

// Four neighbouring columns of one row; `col` is a multiple of 4 and inside.
template <typename T_>
__device__ __forceinline__ void finish4(const Epilogue<T_> &ep, int expert, int64_t row, int64_t col, f32x4 v)
{
    constexpr bool FAST = sizeof(T_) == 2;
    if (ep.bias)
        v += load4(ep.bias + (int64_t)expert * ep.cols + col);
    if (ep.pre)
        store4(ep.pre + row * ep.ldp + col, v);
    float w[4] = {v[0], v[1], v[2], v[3]};
    act_values<FAST>(w, ep.act);
    v = f32x4{w[0], w[1], w[2], w[3]};
    if (ep.mul)
        v *= load4(ep.mul + row * ep.ldm + col);
    if (ep.residual)
        v += load4(ep.residual + row * ep.ldr + col);
    store4(ep.out + row * ep.ldo + col, v);
}

// C[r, c] = sum over k of P[r, k] Q[c, k], r the rows of the output and c its contiguous columns.  An operand is stored
// either row by row (k contiguous) or k by k (r or c contiguous); three of the four combinations occur:
//   forward  P = X  [rows, d_in],  Q = W [d_out, d_in]            both by rows, r in the rows of an expert
//   dX       P = g  [rows, d_out], Q = W [d_out, d_in]            Q k by k, r in the rows of an expert
//   dW       P = g, Q = X                                         both k by k, k in the rows of an expert
enum Product { kForward, kInputGrad, kWeightGrad };

template <typename T_>
struct Operands {
    const T_ *P, *Q;
    int64_t ldp, ldq;
    int64_t q_stride;      // forward, dX: elements from one expert's Q to the next
    int64_t out_stride;    // dW: elements from one expert's C to the next
    int64_t out_rows;      // dW: rows of C
    int64_t depth;         // forward, dX: k
    int64_t lo;            // > 0: P is g in two parts, the second `lo` elements behind the first, and k runs over both
    Segments seg;
};

// Shares of k that the launch's third dimension takes apart: each writes its sums, f32 [rows of the output][cols], to
// partial + share * stride.  n = 1: no split.
struct Split {
    float *partial;
    int64_t stride;
    int n;
};

// Which kernel a product takes (plan_product in linear.hip).
struct Plan {
    enum Kind { kTiles, kFew } kind;
    int tile;     // kTiles: 0: 256 x 256, 1: 128 x 256, 2: 128 x 128 (f32: always 2), 3: 128 x 128, two a compute unit
    int splits;   // kTiles: shares of k
    int blocks;   // kFew: 16-row (and in f32 16-column) blocks of a workgroup
    double us;    // the estimate, where it is one of several launches to choose from
};

// One launch each, two with split k; errors as the entry points report them.
#define DASS_DECLARE_TILES(name)                                                                                              \
    dass_status name(const char *fn, const Plan &plan, const Operands<uint16_t> &a, const Epilogue<uint16_t> &ep,             \
                     const Split &split, hipStream_t stream);                                                                 \
    dass_status name(const char *fn, const Plan &plan, const Operands<float> &a, const Epilogue<float> &ep, const Split &split, \
                     hipStream_t stream);
DASS_DECLARE_TILES(launch_forward)
DASS_DECLARE_TILES(launch_dx)
DASS_DECLARE_TILES(launch_dw)
#undef DASS_DECLARE_TILES
// The forward product with few tiles.
dass_status launch_few(const char *fn, const Plan &plan, const Operands<uint16_t> &a, const Epilogue<uint16_t> &ep, hipStream_t stream);
dass_status launch_few(const char *fn, const Plan &plan, const Operands<float> &a, const Epilogue<float> &ep, hipStream_t stream);

// The bias sums of a gradient: db[e] = the sum of the partial sums of e's tiles of rows.
struct BiasSums {
    const float *partial;   // [tile number][cols]
    int64_t cols;
    Segments seg;
    int tile_rows;
    void *dbias;            // [n_experts][cols]
};

// 64 columns of one expert, in a fixed order: the workgroup's first four wavefronts take every fourth tile.
template <typename T_>
__device__ __forceinline__ void sum_bias(const BiasSums &b, uint32_t strip, int expert, float (*sums)[64])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Span r = segment(b.seg, expert);
    const int64_t first = b.seg.offsets ? r.lo / b.tile_rows + expert : 0, tiles = (r.hi - r.lo + b.tile_rows - 1) / b.tile_rows;
    const int64_t c = (int64_t)strip * 64 + lane;
    float s = 0.0f;
    if (c < b.cols && wave < 4) {
#pragma unroll 8
        for (int64_t i = wave; i < tiles; i += 4)
            s += b.partial[(first + i) * b.cols + c];
    }
    if (wave < 4)
        sums[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && c < b.cols) {
        s = (sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]);
        T_ *const to = static_cast<T_ *>(b.dbias) + (int64_t)expert * b.cols + c;
        if constexpr (sizeof(T_) == 2)
            *to = __builtin_bit_cast(uint16_t, (__bf16)s);
        else
            *to = s;
    }
}

// A gradient's parts with few tiles (f32), in one launch: dX and dW where their blocks (Plan) are not 0, the bias sums where dbias
// is given.
struct FewGrads {
    Operands<float> x, w;
    Epilogue<float> ex, ew;
    int blocks_x, blocks_w;
    BiasSums bias;
};
dass_status launch_few_grads(const char *fn, const FewGrads &grads, hipStream_t stream);

// The same for both products with the same tiles (Plan), none of them split (bf16); the bias sums where dbias is given.
dass_status launch_pair(const char *fn, int tile, const Operands<uint16_t> &ax, const Epilogue<uint16_t> &ex, const Operands<uint16_t> &aw,
                        const Epilogue<uint16_t> &ew, const BiasSums &bias, hipStream_t stream);

}  // namespace dass
