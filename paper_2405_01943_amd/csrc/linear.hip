// dass_linear: out = act(X W^T + b) * mul + residual, with one W for all rows or that of each row's expert, and its
// gradients.  This file has the checks, the element-wise part of the gradient and the bias sums; the products are in
// linear_tiles.h and linear_few.hip.
//
// Gradients, with g = dout * mul * act'(pre):  dX = g W,  dW = g^T X over an expert's rows,  db = sum of its g,
// dmul = dout * act(pre).  g is read by both products, so it is written once, in dtype dt: rounded to bf16
// there because the matrix cores take nothing wider (each term of a sum is off by half a step of its own, which adds about as
// much to a sum as its own rounding does: 0.00235 of the whole where f32 would leave 0.00166).  Where g, dX or dW is small
// chance makes it more (two rows of 144: 0.0026; dW of 8 x 8: 0.0034), and there g is kept as two bf16 numbers, its leading bits and what
// they leave, and the products run over both.  Everywhere that would cost as much as the products do: 6001 rows over 8 experts of 4096 x
// 11008 in one part 1174 us, in two 2140.  Without activation and mul, g is dout itself and nothing is written.
#include "linear.h"

#include <algorithm>
#include <initializer_list>

namespace dass {

constexpr int kMaxLinearExperts = 1024;
constexpr int64_t kMaxRows = 1 << 30, kMaxWidth = 1 << 20, kMaxStride = 1LL << 36;
constexpr int64_t kMaxReadRow = 1 << 23;   // bytes between rows that a tile addresses: 256 of them with 32-bit offsets

// ------------------------------------------------------ element-wise gradient and sums --
// g as two bf16 numbers: its leading bits, returned, and what they leave, to `rest` (to be rounded: 2^-16 of g at most).  Both have g's
// sign and neither is 0 where g is not, 2^-24 of g at least (2^-126 for the smallest), so that the products with an infinite
// element of X or W are two infinities of one sign, as g's own is one: with g rounded to nearest and the signed rest, 0 or the
// other sign met the infinity and gave NaN.
__device__ __forceinline__ float two_parts(float g, float &rest)
{
    const float lead = g == g ? __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, g) & 0xffff0000u) : g;
    const float size = fabsf(lead);
    const float left = size < INFINITY ? fmaxf(fabsf(g - lead), 0x1p-24f * size) : 0.0f;
    rest = g == 0.0f ? 0.0f : copysignf(fmaxf(left, 0x1p-126f), g);
    return lead;
}

// A wavefront owns 64 chunks of 16 bytes of columns and every fourth row of a tile of rows of one expert.  One pass:
// reads dout, pre and mul, writes g and dmul, and adds g up for the bias in f32 before it is rounded, over the tile.
template <typename T_>
__global__ __launch_bounds__(256) void slope_kernel(const T_ *__restrict__ dout, int64_t ldg, const T_ *__restrict__ pre,
                                                    int64_t ldp, const T_ *__restrict__ mul, int64_t ldm, int act, int64_t cols,
                                                    Segments seg, int tile_rows, T_ *__restrict__ g_out, int64_t ldk, int64_t lo,
                                                    T_ *__restrict__ w_out, int64_t w_lo, T_ *__restrict__ dmul, int64_t lddm,
                                                    float *__restrict__ partial, uint32_t strips)
{
    constexpr int N = Chunk<T_>::N;
    constexpr bool FAST = sizeof(T_) == 2;
    __shared__ float sums[4][64][N + 1];
    const uint32_t number = blockIdx.x / strips, strip = blockIdx.x - number * strips;
    int expert;
    Span r;
    if (!rows_of_tile(seg, number, tile_rows, expert, r))
        return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c = ((int64_t)strip * 64 + lane) * N;
    const int64_t end = r.lo + tile_rows < r.hi ? r.lo + tile_rows : r.hi;
    float sum[N];
#pragma unroll
    for (int x = 0; x < N; ++x)
        sum[x] = 0.0f;
    if (c < cols) {
        for (int64_t row = r.lo + wave; row < end; row += 4) {
            float g[N], p[N], m[N];
            Chunk<T_>::widen(*reinterpret_cast<const u32x4 *>(dout + row * ldg + c), g);
            if (pre)
                Chunk<T_>::widen(*reinterpret_cast<const u32x4 *>(pre + row * ldp + c), p);
            if (mul)
                Chunk<T_>::widen(*reinterpret_cast<const u32x4 *>(mul + row * ldm + c), m);
            if (dmul) {
                float y[N];
#pragma unroll
                for (int x = 0; x < N; ++x)
                    y[x] = p[x];
                act_values<FAST>(y, act);
#pragma unroll
                for (int x = 0; x < N; ++x)
                    y[x] *= g[x];
                *reinterpret_cast<u32x4 *>(dmul + row * lddm + c) = Chunk<T_>::narrow(y);
            }
            if (mul) {
#pragma unroll
                for (int x = 0; x < N; ++x)
                    g[x] *= m[x];
            }
            if (act != DASS_ACT_NONE) {
                float y[N];
                act_slopes<FAST>(p, y, act);
#pragma unroll
                for (int x = 0; x < N; ++x)
                    g[x] *= y[x];
            }
#pragma unroll
            for (int x = 0; x < N; ++x)
                sum[x] += g[x];
            if (g_out && lo == 0)
                *reinterpret_cast<u32x4 *>(g_out + row * ldk + c) = Chunk<T_>::narrow(g);
            if (lo > 0 || w_lo > 0) {
                float rest[N];
#pragma unroll
                for (int x = 0; x < N; ++x)
                    g[x] = two_parts(g[x], rest[x]);
                T_ *const to = lo > 0 ? g_out + row * ldk + c : w_out + row * cols + c;
                *reinterpret_cast<u32x4 *>(to) = Chunk<T_>::narrow(g);
                *reinterpret_cast<u32x4 *>(to + (lo > 0 ? lo : w_lo)) = Chunk<T_>::narrow(rest);
            }
        }
    } else if (c < lo) {   // to whole slabs
        for (int64_t row = r.lo + wave; row < end; row += 4)
            *reinterpret_cast<u32x4 *>(g_out + row * ldk + c) = *reinterpret_cast<u32x4 *>(g_out + row * ldk + lo + c) = u32x4{0, 0, 0, 0};
    }
    if (!partial)
        return;
#pragma unroll
    for (int x = 0; x < N; ++x)
        sums[wave][lane][x] = sum[x];
    __syncthreads();
    for (int i = threadIdx.x; i < 64 * N; i += 256) {
        const int64_t col = (int64_t)strip * 64 * N + i;
        if (col < cols) {
            float s = 0.0f;
#pragma unroll
            for (int w = 0; w < 4; ++w)
                s += sums[w][i / N][i % N];
            partial[number * cols + col] = s;
        }
    }
}

template <typename T_>
__global__ __launch_bounds__(256) void bias_kernel(const BiasSums b)
{
    __shared__ float sums[4][64];
    sum_bias<T_>(b, blockIdx.x, blockIdx.y, sums);
}

// ------------------------------------------------------------------ host side --
// Rows of a tile of the two kernels above: as many as leave 512 workgroups, 8 to 64 (a wavefront takes every fourth row, one after the
// other: 301 rows of 688 f32 in tiles of 64 12.6 us, of 8 4.2), and more where that makes over 512 tiles, whose sums one
// workgroup adds.
static int sum_tile_rows(int64_t rows, int64_t cols, int dt)
{
    const int64_t strips = (cols + 64 * vec_elems(dt) - 1) / (64 * vec_elems(dt));
    int64_t t = 8;
    while (t < 64 && rows / (2 * t) * strips >= 512)
        t *= 2;
    while (rows / t > 512)
        t *= 2;
    return (int)(t < (1 << 24) ? t : 1 << 24);
}

// How g is kept, in elements.  In two parts (two_parts) where the result or g itself has so few elements that the mean squares of
// the errors are not near their expectation: both in each row, whole slabs, for both products where g has up to 16384 elements or
// dX up to 8192, and for dW alone, in two matrices of its own, where it has up to 8192 (of all experts).  61104 gradients of random sizes, 1 to
// 65536 rows, widths of 8 to 4096, dense and by 2 to 33 experts: the error is 1.36 times that of a g in f32 in the mean where g is in one part,
// 1.473 times at most, and 1.001 times at most in two; without the rule for dW 2.07.  It costs 4096 rows of 64 x 64 18.8 -> 23.2 us,
// 65536 of 64 x 128 88 -> 138, 2^20 of 8 x 8 1160 -> 2040 and three times the g in the workspace.
struct KeptG {
    int64_t ld, lo;         // its rows; lo > 0: from a row's first part to the second
    int64_t w_lo;           // > 0: dW's own two matrices follow, this far apart
    size_t before, bytes;   // bytes of the first matrix and of all
};

static KeptG kept_g(int64_t rows, int64_t d_in, int64_t d_out, int64_t n_experts, dass_dtype dt, bool dX, bool dW)
{
    const size_t matrix = round_up((size_t)rows * (size_t)d_out * elem_bytes(dt), 256);
    KeptG k = {d_out, 0, 0, matrix, matrix};
    if (dt == DASS_BF16 && (rows * d_out <= 16384 || rows * d_in <= 8192)) {
        k.lo = round_up((size_t)d_out, 64);
        k.ld = 2 * k.lo;
        k.before = k.bytes = round_up((size_t)rows * (size_t)k.ld * 2, 256);
    } else if (dt == DASS_BF16 && dW && n_experts * d_out * d_in <= 8192) {
        k.w_lo = matrix / 2;
        k.before = dX ? matrix : 0;
        k.bytes = k.before + 2 * matrix;
    }
    return k;
}

static size_t partial_bytes(int64_t rows, int64_t d_out, int64_t n_experts, int dt)
{
    return round_up((size_t)(rows / sum_tile_rows(rows, d_out, dt) + 1 + n_experts) * (size_t)d_out * 4, 256);
}

// The longest row stride of an operand of the products, in elements: 256 of them stay below 2^31 bytes.
static int64_t longest_read(int dt) { return kMaxReadRow / (dt == DASS_BF16 ? 2 : 4) - vec_elems(dt); }

struct Arguments {
    const char *fn;
    int vec;
    dass_status status = DASS_OK;

    // a matrix of `rows` rows of `width` elements; absent optional ones are fine
    void matrix(const char *name, const void *p, int64_t rows, int64_t ld, int64_t width, bool required, int64_t longest = kMaxStride)
    {
        if (status != DASS_OK || (!p && !required))
            return;
        if (!p)
            status = fail(DASS_ERR_NULL, "%s: %s must not be NULL", fn, name);
        else if (ld < width || ld > longest)
            status = fail(DASS_ERR_SHAPE, "%s: row stride %lld of %s is shorter than its rows of %lld or beyond %lld", fn, (long long)ld,
                          name, (long long)width, (long long)longest);
        else if (rows > kMaxSpan / ld)
            status = fail(DASS_ERR_SHAPE, "%s: %lld rows of %s with stride %lld span more than 2^46 elements", fn, (long long)rows, name,
                          (long long)ld);
        else if (!aligned16(p) || ld % vec != 0)
            status = fail(DASS_ERR_ALIGN, "%s: %s must be 16-byte aligned, its row stride a multiple of %d elements", fn, name, vec);
    }
    // an output that begins where something else of the call does
    void apart(const char *name, const void *out, std::initializer_list<const void *> others)
    {
        for (const void *p : others)
            if (status == DASS_OK && out && p == out)
                status = fail(DASS_ERR_ARG, "%s: %s must not overlap another operand", fn, name);
    }
    void vector(const char *name, const void *p)
    {
        if (status == DASS_OK && p && !aligned16(p))
            status = fail(DASS_ERR_ALIGN, "%s: %s must be 16-byte aligned", fn, name);
    }
    void sizes(int64_t T, int64_t d_in, int64_t d_out, int64_t n_experts, const int32_t *offsets, int dt, int act)
    {
        if (!valid_dtype(dt))
            status = fail(DASS_ERR_DTYPE, "%s: unknown dtype %d", fn, dt);
        else if (act < DASS_ACT_SILU || act > DASS_ACT_NONE)
            status = fail(DASS_ERR_DTYPE, "%s: unknown activation %d", fn, act);
        else if (T <= 0 || d_in <= 0 || d_out <= 0)
            status = fail(DASS_ERR_SHAPE, "%s: T=%lld d_in=%lld d_out=%lld must be positive", fn, (long long)T, (long long)d_in,
                          (long long)d_out);
        else if (T > kMaxRows || d_in > kMaxWidth || d_out > kMaxWidth)
            status = fail(DASS_ERR_SHAPE, "%s: T=%lld must be at most 2^30, d_in=%lld and d_out=%lld at most 2^20", fn, (long long)T,
                          (long long)d_in, (long long)d_out);
        else if (d_in % vec_elems(dt) != 0 || d_out % vec_elems(dt) != 0)
            status = fail(DASS_ERR_SHAPE, "%s: d_in=%lld and d_out=%lld must be multiples of %d", fn, (long long)d_in,
                          (long long)d_out, vec_elems(dt));
        else if (n_experts <= 0 || n_experts > kMaxLinearExperts || (!offsets && n_experts != 1))
            status = fail(DASS_ERR_SHAPE, "%s: n_experts=%lld must be 1 without offsets, 1 to %d with them", fn,
                          (long long)n_experts, kMaxLinearExperts);
        else if (reinterpret_cast<uintptr_t>(offsets) & 3u)
            status = fail(DASS_ERR_ALIGN, "%s: offsets must be 4-byte aligned", fn);
    }
    void stride(const char *name, int64_t stride, int64_t ld, int64_t d_in, int64_t d_out, int64_t n_experts)
    {
        if (status == DASS_OK && n_experts > 1 && (stride < (d_out - 1) * ld + d_in || stride > 1LL << 50))
            status = fail(DASS_ERR_SHAPE, "%s: expert stride %lld of %s is shorter than a matrix or beyond 2^50", fn, (long long)stride,
                          name);
        if (status == DASS_OK && n_experts > 1 && stride % vec != 0)
            status = fail(DASS_ERR_ALIGN, "%s: expert stride of %s must be a multiple of %d elements", fn, name, vec);
    }
};

static int64_t pieces(int64_t n, int64_t of) { return (n + of - 1) / of; }

// The tiles of a product in the direction of its rows; experts of uneven size have half a tile more each.
static int64_t row_tiles(Product product, int64_t groups, int64_t rows, int64_t of)
{
    if (product == kWeightGrad || groups == 1)
        return groups * pieces(rows, of);
    const int64_t used = std::min(groups, rows);
    return std::max(used, rows / of + used / 2);
}

struct Tile {
    int rows, cols, slots;   // slots: workgroups that the card holds
    double start, slab;      // us of a workgroup and of each slab of k
    // alone on its compute unit a workgroup of the short tile is not held up by a second
    double time(int64_t slabs, int64_t tiles) const
    {
        return slots == 512 && tiles <= 256 ? 4.47 + slabs * 0.689 : start + slabs * slab;
    }
};
static const Tile kTiles[] = {{256, 256, 256, 8.8, 1.34}, {128, 256, 256, 5.4, 0.87}, {128, 128, 256, 4.06, 0.517},
                              {128, 128, 512, 3.47, 0.985}},
                  kTileF32 = {128, 128, 256, 3.4, 2.49};

// The kernel, the tile and the split of k that are expected to be fastest for the products of `groups` experts: cols columns,
// `depth` of k each, and `rows` rows each (dW) or all together.  The estimates, in us, are fitted to times of 149 bf16 and 45
// f32 products of 1 to 16384 rows and every tile with 1 to 16 shares; over the bf16 ones the choice is 1 % slower than the best
// in the mean, 27 % at the worst (dX of 8 rows for each of 64 experts of 2048 x 1408).
//
//   tiles   rounds of `slots` workgroups x (start + slabs x slab), or what memory takes for the weights and the output, and with a
//           split 8 bytes for each share's sum (written and read) and the second launch.  A tile's slab takes as long as its
//           bytes from L2, whichever shape; large tiles read least in all, small ones and shares fill the chip.  1024 rows of
//           4096 x 4096, 256 x 256 / 128 x 256 / 128 x 128: 93 / 56 / 39 us, 52 / 46 / 55 with 4, 2 and 2 shares; 16384
//           rows of 4096 x 11008: 1197 us with 256 x 256; dX of 6000 rows of 4096 x 11008 473 / 503 / -; 64 rows of 11008 x
//           4096 (128 x 128) 88 us, 27 with 8 shares; dW of 16384 rows of 512 x 512 145, 28 with 8; one share where the
//           tiles fill the chip: 2048 rows of 4096 x 4096 59 us, 86 with 2.
//   short   (bf16) two 128 x 128 workgroups a compute unit with shorter rings: one's stores run beside the other's products, so
//           it leads where k is short, 8192 rows of 64 x 4096 26 us (the best other tile 36), 512 x 4096 49 (52), 1024 x
//           4096 74 (72); and alone on a compute unit its slabs are slower than the others': no shares.
//   few     (f32) a fixed part that grows with k, or the workgroups and their multiplications.  512 rows of 256 x 688: blocks
//           of 16 / of 32 / tiles 13.2 / 6.7 / 16.6 us, 16 of 1024 x 1024 5.7 / 8.9 / 11.5, 1024 of 512 x 512 17 / 10 / 19,
//           4096 of 1024 x 1024 225 / 119 / 71.
//           (bf16, forward only) the weights' bytes, or one workgroup's.  Up to 8 rows: one row of 2048 x 32000 30.0 us (tiles
//           36.5), 8 of it 34.5 (37.7); but one row of 16384 x 1024 20.6 (tiles with 16 shares 15.6).  16 rows over 8 experts
//           of 4096 x 14336 171 (186), 64 over 8 204 (182).
static Plan plan_product(Product product, int dt, int64_t groups, int64_t rows, int64_t cols, int64_t depth, int parts = 1)
{
    const bool bf16 = dt == DASS_BF16;
    const int64_t share = product == kWeightGrad ? rows : pieces(rows, groups);   // of an expert, were they even
    const int64_t used = std::min(groups, rows);
    static const int kShares[] = {1, 2, 3, 4, 6, 8, 12, 16};
    const double join = bf16 ? 3.64 : 2.4, byte = bf16 ? 1 / 6.13e6 : 1 / 4.5e6;   // us, us a byte
    const int64_t slabs = parts * pieces(depth, bf16 ? 64 : 32), outputs = (product == kWeightGrad ? groups : 1) * rows * cols;
    const double weights = product == kWeightGrad ? 0 : (bf16 ? 6 : 0) + (bf16 ? 2.0 / 5.2e6 : 4.0 / 4.6e6) * used * cols * depth;
    const double written = bf16 ? 2.0 / 3.38e6 * outputs : 0;
    Plan best = {Plan::kTiles, bf16 ? 0 : 2, 1, 0, 0};
    double best_time = 1e300;
    for (int k = bf16 ? 0 : 2; k < (bf16 ? 4 : 3); ++k) {
        const Tile &t = bf16 ? kTiles[k] : kTileF32;
        const int64_t tiles = row_tiles(product, groups, rows, t.rows) * pieces(cols, t.cols);
        for (const int z : kShares) {
            if (z > 1 && (k == 3 || slabs < 2 * z || (double)z * outputs * 4 > 256e6))
                break;
            const double busy = pieces(tiles * z, t.slots) * t.time(pieces(slabs, z), tiles), memory = weights + (z == 1 ? written : 0);
            const double time = std::max(busy, memory) + (bf16 ? 0.093 * std::min(busy, memory) : 0) +
                                (z > 1 ? join + z * 8.0 * outputs * byte : 0);
            if (time < best_time) {
                best_time = time;
                best = {Plan::kTiles, k, z, 0, time};
            }
        }
    }
    const auto one_launch = [&](int of, int threads) {   // of workgroups of `of` x `of` outputs
        const int64_t most = product == kWeightGrad ? groups * pieces(rows, of) : rows / of + groups;
        return (double)most * pieces(cols, of) * threads < 0x3fffffff;   // (a gradient's parts share one)
    };
    if (bf16 && product == kForward && share <= 8 && one_launch(16, 1024)) {
        const double bytes = 2.0 * used * cols * depth * (1 + 0.025 * (share - 1));
        if ((share == 1 && groups > 1) || std::max(2 + 0.0011 * depth, 2 + bytes / 5.1e6) < best_time)
            return {Plan::kFew, 0, 1, 1, 0};
    }
    for (int blocks = 1; !bf16 && blocks <= 2; ++blocks) {
        const double workgroups = (double)row_tiles(product, groups, rows, 16 * blocks) * pieces(cols, 16 * blocks);
        if (!one_launch(16 * blocks, 512))
            continue;
        const double products = workgroups * 256 * blocks * blocks * depth;
        const double fixed = blocks == 1 ? 2.8 + 0.0028 * depth : 2.6 + 0.0065 * depth;
        const double busy = blocks == 1 ? 2 + 0.0085 * workgroups + 23e-9 * products : 3 + 0.001 * workgroups + 27e-9 * products;
        if (fixed < best_time && busy < best_time) {
            best_time = std::max(fixed, busy);
            best = {Plan::kFew, 0, 1, blocks, best_time};
        }
    }
    return best;
}

// parts: of g, that k runs over
static Plan plan_of(Product product, int dt, int64_t T, int64_t d_in, int64_t d_out, int64_t n_experts, int parts = 1)
{
    if (product == kForward)
        return plan_product(product, dt, n_experts, T, d_out, d_in);
    if (product == kInputGrad)
        return plan_product(product, dt, n_experts, T, d_in, d_out, parts);
    return plan_product(product, dt, n_experts, d_out, d_in, (T + n_experts - 1) / n_experts, parts);
}

// When n1 workgroups of t1 and after them n2 of t2 <= t1 are done on `slots` places, each taking the next one when it is free.
static double makespan(int64_t n1, double t1, int64_t n2, double t2, int64_t slots)
{
    const int64_t rounds = n1 / slots, late = n1 % slots;   // late: places that have one more of the first
    const double from[2] = {rounds * t1, (rounds + 1) * t1};
    const auto done = [&](double t) {   // of the second, at time t
        const auto each = [&](double begin) { return t < begin ? 0 : (int64_t)((t - begin) / t2 + 1e-6); };
        return late * each(from[1]) + (slots - late) * each(from[0]);
    };
    double first = 1e300;
    for (int i = 0; i < (late ? 2 : 1); ++i) {
        int64_t m = std::max((int64_t)0, n2 / slots - (i ? (int64_t)(t1 / t2) + 1 : 0));
        while (done(from[i] + m * t2) < n2)
            ++m;
        first = std::min(first, from[i] + m * t2);
    }
    return std::max(first, late ? from[1] : from[0]);
}

// The tile of both products of a bf16 gradient (and its bias sums) in one launch, or -1 for a launch each: the tiles of the one
// fill the rounds that the other leaves, the longer ones first.  In graphs, with the element-wise pass and bias sums: 301 rows of
// 256 x 688 22.0 us, in one launch 13.1; 1030 of 576 x 520 29.4, 18.2; 2000 rows over 8 experts of 512 x 1024 35.3, 22.9; 4100 of 2056 x
// 2056 159, 113 with 256 x 256; 8192 over 8 experts of 4096 x 14336 2000, 1863; but 512 of 1024 x 4096 34.0, 43.1, and 16384
// of 512 x 512 57.5, 170.8, where k has to be split.  Over 97 sizes the choice is 1 % slower than the best in the mean, and 1.26
// times as fast as two launches always.
static int pair_of(const Plan &x, const Plan &w, int64_t T, int64_t d_in, int64_t d_out, int64_t n_experts, int parts_x,
                   int parts_w)
{
    const int64_t slabs_x = parts_x * pieces(d_out, 64), slabs_w = parts_w * pieces(pieces(T, n_experts), 64);
    const double memory = 6 + 2.0 / 5.2e6 * std::min(n_experts, T) * d_in * d_out + 2.0 / 3.38e6 * ((double)T + n_experts * d_out) * d_in;
    int best = -1;
    double best_time = x.us + w.us + 2;   // 2: the second launch
    for (int k = 0; k <= 3; ++k) {
        const Tile &t = kTiles[k];
        const int64_t tiles_x = row_tiles(kInputGrad, n_experts, T, t.rows) * pieces(d_in, t.cols);
        const int64_t tiles_w = n_experts * pieces(d_out, t.rows) * pieces(d_in, t.cols), tiles = tiles_x + tiles_w;
        const double one_x = t.time(slabs_x, tiles), one_w = t.time(slabs_w, tiles);
        if (tiles > 1 << 20 || (tiles_x * one_x + tiles_w * one_w) / t.slots >= best_time)
            continue;
        const double busy = slabs_x >= slabs_w ? makespan(tiles_x, one_x, tiles_w, one_w, t.slots)
                                               : makespan(tiles_w, one_w, tiles_x, one_x, t.slots);
        const double time = std::max(busy, memory);
        if (time < best_time) {
            best_time = time;
            best = k;
        }
    }
    return best;
}

static int64_t output_size(Product product, int64_t T, int64_t d_in, int64_t d_out, int64_t n_experts)
{
    return product == kForward ? T * d_out : product == kInputGrad ? T * d_in : n_experts * d_out * d_in;
}

static size_t split_bytes(const Plan &plan, Product product, int64_t T, int64_t d_in, int64_t d_out, int64_t n_experts)
{
    return plan.splits > 1 ? round_up((size_t)plan.splits * output_size(product, T, d_in, d_out, n_experts) * 4, 256) : 0;
}

// What a gradient's call takes and needs: g if it is kept, then the most of the bias sums and of the split products' shares.
struct GradPlan {
    KeptG g;    // all 0: it is not kept
    Plan x, w;
    int pair;   // the tile of both products in one launch; -1: none
    size_t bytes;
};

static GradPlan plan_grad(int64_t T, int64_t d_in, int64_t d_out, dass_dtype dt, int64_t n_experts, bool keeps_g, bool dX, bool dW,
                          bool dbias)
{
    GradPlan p = {};
    if (keeps_g)
        p.g = kept_g(T, d_in, d_out, n_experts, dt, dX, dW);
    const int parts_x = p.g.lo > 0 ? 2 : 1, parts_w = p.g.lo > 0 || p.g.w_lo > 0 ? 2 : 1;
    p.pair = -1;
    if (dX)
        p.x = plan_of(kInputGrad, dt, T, d_in, d_out, n_experts, parts_x);
    if (dW)
        p.w = plan_of(kWeightGrad, dt, T, d_in, d_out, n_experts, parts_w);
    if (dX && dW && dt == DASS_BF16)
        p.pair = pair_of(p.x, p.w, T, d_in, d_out, n_experts, parts_x, parts_w);
    p.bytes = dbias ? partial_bytes(T, d_out, n_experts, dt) : 0;
    if (dX && p.pair < 0)
        p.bytes = std::max(p.bytes, split_bytes(p.x, kInputGrad, T, d_in, d_out, n_experts));
    if (dW && p.pair < 0)
        p.bytes = std::max(p.bytes, split_bytes(p.w, kWeightGrad, T, d_in, d_out, n_experts));
    p.bytes += p.g.bytes;
    return p;
}

template <typename T_>
static dass_status launch_product(const char *fn, Product product, const Plan &plan, int64_t d_in, int64_t d_out, const Operands<T_> &a,
                                  const Epilogue<T_> &ep, void *workspace, hipStream_t stream)
{
    const Split split = {static_cast<float *>(workspace), output_size(product, a.seg.rows, d_in, d_out, a.seg.n), plan.splits};
    if (product == kForward)
        return plan.kind == Plan::kFew ? launch_few(fn, plan, a, ep, stream) : launch_forward(fn, plan, a, ep, split, stream);
    return product == kInputGrad ? launch_dx(fn, plan, a, ep, split, stream) : launch_dw(fn, plan, a, ep, split, stream);
}

template <typename T_>
static dass_status run_linear(const char *fn, const dass_linear_task &t, const Plan &plan, void *workspace, hipStream_t stream)
{
    Operands<T_> a = {};
    a.P = static_cast<const T_ *>(t.X);
    a.ldp = t.ldx;
    a.Q = static_cast<const T_ *>(t.W);
    a.ldq = t.ldw;
    a.q_stride = t.expert_stride;
    a.depth = t.d_in;
    a.seg = {t.offsets, t.T, (int)t.n_experts};
    const Epilogue<T_> ep = {static_cast<T_ *>(t.out), t.ldo, static_cast<const T_ *>(t.bias), static_cast<const T_ *>(t.mul),
                             t.ldm, static_cast<const T_ *>(t.residual), t.ldr, static_cast<T_ *>(t.pre_out), t.ldp, t.d_out,
                             (int)t.act};
    return launch_product(fn, kForward, plan, t.d_in, t.d_out, a, ep, workspace, stream);
}

// Whether g is a matrix of its own.
static bool keeps_g(const dass_linear_grad_task &t) { return (t.act != DASS_ACT_NONE || t.mul) && (t.dX || t.dW); }

template <typename T_>
static dass_status run_linear_grad(const char *fn, const dass_linear_grad_task &t, const GradPlan &plan, char *workspace,
                                   hipStream_t stream)
{
    constexpr int N = Chunk<T_>::N;
    const Segments seg = {t.offsets, t.T, (int)t.n_experts};
    const bool own_g = keeps_g(t);
    // the workspace: g if it is kept, then the partial sums of the bias, whose place the split products take after them
    char *const shares = workspace + plan.g.bytes;
    T_ *const kept = plan.g.before > 0 ? reinterpret_cast<T_ *>(workspace) : nullptr;
    T_ *const kept_w = plan.g.w_lo > 0 ? reinterpret_cast<T_ *>(workspace + plan.g.before) : nullptr;
    const BiasSums bias = {reinterpret_cast<float *>(shares), t.d_out, seg, sum_tile_rows(t.T, t.d_out, t.dt), t.dbias};
    if (own_g || t.dbias || t.dmul) {
        const int64_t numbers = tile_numbers(seg, bias.tile_rows), strips = (t.d_out + 64 * N - 1) / (64 * N);
        if (numbers > 0xffffffffLL / 256 / strips)
            return fail(DASS_ERR_SHAPE, "%s: too many tiles for one launch; split the rows", fn);
        hipLaunchKernelGGL(slope_kernel<T_>, dim3((unsigned)(numbers * strips)), dim3(256), 0, stream,
                           static_cast<const T_ *>(t.dout), t.ldg, static_cast<const T_ *>(t.pre), t.ldp,
                           static_cast<const T_ *>(t.mul), t.ldm, (int)t.act, t.d_out, seg, bias.tile_rows, kept, plan.g.ld, plan.g.lo,
                           kept_w, plan.g.w_lo, static_cast<T_ *>(t.dmul), t.lddm,
                           t.dbias ? reinterpret_cast<float *>(shares) : nullptr, (uint32_t)strips);
        const dass_status s = check_launch("slope kernel");
        if (s != DASS_OK)
            return s;
    }

    Operands<T_> ax = {}, aw = {};
    Epilogue<T_> ex = {}, ew = {};
    ax.P = own_g ? kept : static_cast<const T_ *>(t.dout);
    ax.ldp = own_g ? plan.g.ld : t.ldg;
    ax.lo = plan.g.lo;
    aw.P = kept_w ? kept_w : ax.P;
    aw.ldp = kept_w ? t.d_out : ax.ldp;
    aw.lo = kept_w ? plan.g.w_lo : plan.g.lo;
    ax.seg = aw.seg = seg;
    ex.cols = ew.cols = t.d_in;
    ex.act = ew.act = DASS_ACT_NONE;
    ax.Q = static_cast<const T_ *>(t.W);
    ax.ldq = t.ldw;
    ax.q_stride = t.expert_stride;
    ax.depth = t.d_out;
    ex.out = static_cast<T_ *>(t.dX);
    ex.ldo = t.lddx;
    aw.Q = static_cast<const T_ *>(t.X);
    aw.ldq = t.ldx;
    aw.out_stride = t.dw_stride;
    aw.out_rows = t.d_out;
    ew.out = static_cast<T_ *>(t.dW);
    ew.ldo = t.lddw;
    const bool few_x = t.dX && plan.x.kind == Plan::kFew, few_w = t.dW && plan.w.kind == Plan::kFew;
    const bool tiles_x = t.dX && !few_x, tiles_w = t.dW && !few_w;
    // with the few tiles of the products, if no split product takes the partial sums' place
    const bool bias_with_few = (few_x || few_w) && !tiles_x && !tiles_w && (t.d_out + 63) / 64 * t.n_experts <= 1 << 20;
    if constexpr (sizeof(T_) == 2) {
        if (plan.pair >= 0)
            return launch_pair(fn, plan.pair, ax, ex, aw, ew, bias, stream);
    }
    if (t.dbias && !bias_with_few) {
        hipLaunchKernelGGL(bias_kernel<T_>, dim3((unsigned)((t.d_out + 63) / 64), (unsigned)t.n_experts), dim3(256), 0, stream, bias);
        const dass_status s = check_launch("bias kernel");
        if (s != DASS_OK)
            return s;
    }
    if constexpr (sizeof(T_) == 4) {
        if (few_x || few_w) {
            FewGrads few = {ax, aw, ex, ew, few_x ? plan.x.blocks : 0, few_w ? plan.w.blocks : 0, bias};
            if (!bias_with_few)
                few.bias.dbias = nullptr;
            const dass_status s = launch_few_grads(fn, few, stream);
            if (s != DASS_OK)
                return s;
        }
    }
    if (tiles_x) {
        const dass_status s = launch_product(fn, kInputGrad, plan.x, t.d_in, t.d_out, ax, ex, shares, stream);
        if (s != DASS_OK)
            return s;
    }
    return tiles_w ? launch_product(fn, kWeightGrad, plan.w, t.d_in, t.d_out, aw, ew, shares, stream) : DASS_OK;
}

}  // namespace dass

extern "C" size_t dass_linear_workspace_bytes(int64_t T, int64_t d_in, int64_t d_out, dass_dtype dt, int64_t n_experts)
{
    using namespace dass;
    if (T <= 0 || d_in <= 0 || d_out <= 0 || n_experts <= 0 || n_experts > kMaxLinearExperts || !valid_dtype(dt) || T > kMaxRows ||
        d_in > kMaxWidth || d_out > kMaxWidth)
        return 0;
    return split_bytes(plan_of(kForward, dt, T, d_in, d_out, n_experts), kForward, T, d_in, d_out, n_experts);
}

extern "C" dass_status dass_linear(const dass_linear_task *task, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    using namespace dass;
    const char *fn = "dass_linear";
    if (!task)
        return fail(DASS_ERR_NULL, "%s: task must not be NULL", fn);
    const dass_linear_task &t = *task;
    Arguments c{fn, valid_dtype(t.dt) ? vec_elems(t.dt) : 1};
    c.sizes(t.T, t.d_in, t.d_out, t.n_experts, t.offsets, (int)t.dt, (int)t.act);
    const int64_t read = longest_read(t.dt);
    c.matrix("X", t.X, t.T, t.ldx, t.d_in, true, read);
    c.matrix("W", t.W, t.d_out, t.ldw, t.d_in, true, read);
    c.matrix("mul", t.mul, t.T, t.ldm, t.d_out, false);
    c.matrix("residual", t.residual, t.T, t.ldr, t.d_out, false);
    c.matrix("pre_out", t.pre_out, t.T, t.ldp, t.d_out, false);
    c.matrix("out", t.out, t.T, t.ldo, t.d_out, true);
    c.vector("bias", t.bias);
    c.stride("W", t.expert_stride, t.ldw, t.d_in, t.d_out, t.n_experts);
    c.apart("out", t.out, {t.X, t.W, t.bias, t.pre_out});
    c.apart("pre_out", t.pre_out, {t.X, t.W, t.bias, t.mul, t.residual});
    if ((t.out == t.mul && t.ldo != t.ldm) || (t.out == t.residual && t.ldo != t.ldr))
        c.apart("out", t.out, {t.out});
    if (c.status != DASS_OK)
        return c.status;
    const Plan plan = plan_of(kForward, t.dt, t.T, t.d_in, t.d_out, t.n_experts);
    const size_t need = split_bytes(plan, kForward, t.T, t.d_in, t.d_out, t.n_experts);
    if (need > 0 && (!workspace || workspace_bytes < need))
        return fail(DASS_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", fn, workspace ? workspace_bytes : 0, need);
    if (need > 0 && !aligned16(workspace))
        return fail(DASS_ERR_ALIGN, "%s: workspace must be 16-byte aligned", fn);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    return t.dt == DASS_BF16 ? run_linear<uint16_t>(fn, t, plan, workspace, stream) : run_linear<float>(fn, t, plan, workspace, stream);
}

extern "C" size_t dass_linear_backward_workspace_bytes(int64_t T, int64_t d_in, int64_t d_out, dass_dtype dt, int64_t n_experts)
{
    using namespace dass;
    if (T <= 0 || d_in <= 0 || d_out <= 0 || n_experts <= 0 || n_experts > kMaxLinearExperts || !valid_dtype(dt) || T > kMaxRows ||
        d_in > kMaxWidth || d_out > kMaxWidth)
        return 0;
    // the most that a call of all or some of the gradients needs: one alone may be split where both together are not, and a g
    // that is not kept may be split otherwise
    size_t most = 0;
    for (const bool keeps : {false, true})
        for (const int which : {1, 2, 3})
            most = std::max(most, plan_grad(T, d_in, d_out, dt, n_experts, keeps, which & 1, which & 2, true).bytes);
    return most;
}

extern "C" dass_status dass_linear_backward(const dass_linear_grad_task *task, void *workspace, size_t workspace_bytes,
                                            void *hip_stream)
{
    using namespace dass;
    const char *fn = "dass_linear_backward";
    if (!task)
        return fail(DASS_ERR_NULL, "%s: task must not be NULL", fn);
    const dass_linear_grad_task &t = *task;
    Arguments c{fn, valid_dtype(t.dt) ? vec_elems(t.dt) : 1};
    c.sizes(t.T, t.d_in, t.d_out, t.n_experts, t.offsets, (int)t.dt, (int)t.act);
    if (c.status != DASS_OK)
        return c.status;
    if (!t.dX && !t.dW && !t.dbias && !t.dmul)
        return fail(DASS_ERR_NULL, "%s: no gradient is asked for", fn);
    if (t.dmul && !t.mul)
        return fail(DASS_ERR_NULL, "%s: dmul without mul", fn);
    const int64_t read = longest_read(t.dt);
    c.matrix("dout", t.dout, t.T, t.ldg, t.d_out, true, read);
    c.matrix("X", t.X, t.T, t.ldx, t.d_in, t.dW != nullptr, read);
    c.matrix("W", t.W, t.d_out, t.ldw, t.d_in, t.dX != nullptr, read);
    c.matrix("pre", t.pre, t.T, t.ldp, t.d_out, t.act != DASS_ACT_NONE || t.dmul);
    c.matrix("mul", t.mul, t.T, t.ldm, t.d_out, false);
    c.matrix("dX", t.dX, t.T, t.lddx, t.d_in, false);
    c.matrix("dW", t.dW, t.d_out, t.lddw, t.d_in, false);
    c.matrix("dmul", t.dmul, t.T, t.lddm, t.d_out, false);
    c.vector("dbias", t.dbias);
    const void *const inputs[] = {t.dout, t.X, t.W, t.pre, t.mul};
    void *const outputs[] = {t.dX, t.dW, t.dbias, t.dmul};
    const char *const names[] = {"dX", "dW", "dbias", "dmul"};
    for (int i = 0; i < 4; ++i) {
        for (const void *p : inputs)
            c.apart(names[i], outputs[i], {p});
        for (int j = 0; j < i; ++j)
            c.apart(names[i], outputs[i], {outputs[j]});
    }
    if (t.dX)
        c.stride("W", t.expert_stride, t.ldw, t.d_in, t.d_out, t.n_experts);
    if (t.dW)
        c.stride("dW", t.dw_stride, t.lddw, t.d_in, t.d_out, t.n_experts);
    if (c.status != DASS_OK)
        return c.status;
    const GradPlan plan = plan_grad(t.T, t.d_in, t.d_out, t.dt, t.n_experts, keeps_g(t), t.dX, t.dW, t.dbias);
    const size_t need = plan.bytes;
    if (need > 0 && (!workspace || workspace_bytes < need))
        return fail(DASS_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", fn, workspace ? workspace_bytes : 0, need);
    if (need > 0 && !aligned16(workspace))
        return fail(DASS_ERR_ALIGN, "%s: workspace must be 16-byte aligned", fn);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    char *ws = static_cast<char *>(workspace);
    return t.dt == DASS_BF16 ? run_linear_grad<uint16_t>(fn, t, plan, ws, stream) : run_linear_grad<float>(fn, t, plan, ws, stream);
}
