// Tokens sorted by expert and back (the rows of a mixture of GLU experts), and the gradients.
//
// A pair is one (token, slot) of the router's choice ids[T, k].  All of these move integers or rows:
//   sort      reads 4 (or 8) bytes a pair and writes 8; small ones are bound by the launch
//   gather    reads every token's row once and writes it to its k places
//   combine   reads a token's k rows and writes one: f32 sums in slot order, rounded once
//   gradient  reads a token's row and its k expert outputs once, writes k rows and k dot products
// Nothing is atomic in global memory and every sum has a fixed order: results are the same bits on every run.
#include "chunk.h"
#include "dass_internal.h"

namespace dass {

constexpr int kMaxExperts = 1024, kMaxSlots = 64;
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;

// ------------------------------------------------------------------------ sort --
// Expert of a pair; kMaxExperts for one that goes nowhere (any id outside 0 .. E - 1).
template <typename ID>
__device__ __forceinline__ int expert_of(const ID *__restrict__ ids, int64_t pair, int64_t end, int E)
{
    if (pair >= end)
        return kMaxExperts;
    const ID id = ids[pair];
    return id >= 0 && id < (ID)E ? (int)id : kMaxExperts;
}

// Lanes of this wavefront whose expert is this lane's, found bit by bit: a ballot for each bit of an expert's number.
__device__ __forceinline__ uint64_t same_expert(int e, int bits)
{
    uint64_t same = __ballot(e < kMaxExperts);
    if (e >= kMaxExperts)
        return 0;
    for (int b = 0; b < bits; ++b) {
        const uint64_t ones = __ballot((e >> b) & 1);
        same &= (e >> b) & 1 ? ones : ~ones;
    }
    return same;
}

__device__ __forceinline__ void wave_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Pairs of each expert in a block's range, for many pairs: counts[block][E].
template <typename ID>
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(const ID *__restrict__ ids, int64_t pairs, int64_t per_block,
                                                                  int E, int32_t *__restrict__ counts)
{
    __shared__ int32_t hist[kMaxExperts + 1];
    for (int e = threadIdx.x; e <= kMaxExperts; e += kSortThreads)
        hist[e] = 0;
    __syncthreads();
    const int64_t lo = (int64_t)blockIdx.x * per_block, end = lo + per_block < pairs ? lo + per_block : pairs;
    for (int64_t i = lo + threadIdx.x; i < end; i += kSortThreads)
        atomicAdd(&hist[expert_of(ids, i, end, E)], 1);
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += kSortThreads)
        counts[(int64_t)blockIdx.x * E + e] = hist[e];
}

// A stable counting sort.  A wavefront owns a contiguous range of its block's pairs: it counts them, learns where its
// pairs of each expert begin (experts before, blocks before, wavefronts before), and goes over them once more, 64 at a time: a
// pair's row is that place plus the lanes below it with the same expert.  With one block nothing is
// handed over through memory; with several, every block adds up the counts of all blocks by itself (at most 256 x E
// numbers out of L2), which saves a launch.
template <typename ID>
__global__ __launch_bounds__(kSortThreads) void sort_place_kernel(const ID *__restrict__ ids, int64_t pairs, int64_t per_block,
                                                                  int E, int bits, const int32_t *__restrict__ block_counts,
                                                                  int32_t *__restrict__ offsets, int32_t *__restrict__ order,
                                                                  int32_t *__restrict__ place)
{
    extern __shared__ int32_t mem[];
    int32_t *counts = mem;                                   // [wavefront][E + 1], the last for pairs that go nowhere
    __shared__ int32_t all[kMaxExperts], before[kMaxExperts], wave_sum[kSortWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, stride = E + 1;
    for (int i = tid; i < kSortWaves * stride; i += kSortThreads)
        counts[i] = 0;
    for (int e = tid; e < kMaxExperts; e += kSortThreads)
        all[e] = before[e] = 0;
    __syncthreads();

    const int64_t lo = (int64_t)blockIdx.x * per_block, end = lo + per_block < pairs ? lo + per_block : pairs;
    const int64_t per_wave = per_block / kSortWaves, w_lo = lo + wave * per_wave;   // a multiple of 64
    const int64_t w_end = w_lo + per_wave < end ? w_lo + per_wave : end;
    // the experts of the first HELD pairs of each lane stay in registers for the second pass
    constexpr int HELD = 8;
    int held[HELD];
#pragma unroll
    for (int h = 0; h < HELD; ++h)
        held[h] = expert_of(ids, w_lo + h * 64 + lane, w_end, E);
#pragma unroll
    for (int h = 0; h < HELD; ++h)
        if (w_lo + h * 64 + lane < w_end)
            atomicAdd(&counts[wave * stride + (held[h] < E ? held[h] : E)], 1);
    for (int64_t i = w_lo + HELD * 64 + lane; i < w_end; i += 64) {
        const int e = expert_of(ids, i, w_end, E);
        atomicAdd(&counts[wave * stride + (e < E ? e : E)], 1);
    }
    if (block_counts) {
        for (int64_t i = tid; i < (int64_t)gridDim.x * E; i += kSortThreads) {
            const int b = (int)(i / E), e = (int)(i - (int64_t)b * E), c = block_counts[i];
            if (c != 0) {
                atomicAdd(&all[e], c);
                if (b < (int)blockIdx.x)
                    atomicAdd(&before[e], c);
            }
        }
    }
    __syncthreads();

    // places of the experts: an exclusive scan of their totals, a thread an expert
    int total = 0;
    if (tid < E) {
        if (block_counts) {
            total = all[tid];
        } else {
            for (int w = 0; w < kSortWaves; ++w)
                total += counts[w * stride + tid];
        }
    }
    int scan = total;
#pragma unroll
    for (int step = 1; step < 64; step *= 2) {
        const int up = __shfl_up(scan, step, 64);
        scan += lane >= step ? up : 0;
    }
    if (lane == 63)
        wave_sum[wave] = scan;
    __syncthreads();
    int sum = 0, kept = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
        sum += w < wave ? wave_sum[w] : 0;
        kept += wave_sum[w];
    }
    const int first = sum + scan - total;
    if (tid < E) {
        int run = first + before[tid];
        for (int w = 0; w < kSortWaves; ++w) {
            const int c = counts[w * stride + tid];
            counts[w * stride + tid] = run;
            run += c;
        }
        if (blockIdx.x == 0) {
            offsets[tid] = first;
            if (tid == E - 1)
                offsets[E] = kept;
        }
    }
    __syncthreads();

    int32_t *mine = counts + wave * stride;
    auto place_64 = [&](int64_t i, int e) __attribute__((always_inline)) {
        const uint64_t same = same_expert(e, bits);
        int row = -1;
        if (e < kMaxExperts)
            row = mine[e] + __popcll(same & ((1ull << lane) - 1));
        wave_fence();
        if (e < kMaxExperts && (same >> lane) == 1)   // the highest lane of its expert
            mine[e] = row + 1;
        wave_fence();
        if (i < w_end) {
            place[i] = row;
            if (row >= 0)
                order[row] = (int32_t)i;
        }
    };
#pragma unroll
    for (int h = 0; h < HELD; ++h)
        if (w_lo + h * 64 < w_end)
            place_64(w_lo + h * 64 + lane, held[h]);
    for (int64_t i = w_lo + HELD * 64 + lane; i - lane < w_end; i += 64)
        place_64(i, expert_of(ids, i, w_end, E));
    for (int64_t p = kept + (int64_t)blockIdx.x * kSortThreads + tid; p < pairs; p += (int64_t)gridDim.x * kSortThreads)
        order[p] = -1;
}

// ---------------------------------------------------------------- rows to and fro --
// A thread owns one 16-byte chunk of one token's row: read once, written to the row of every slot.
__global__ __launch_bounds__(256) void gather_kernel(const char *__restrict__ X, int64_t row_bytes_x, uint32_t chunks,
                                                     int64_t total, const int32_t *__restrict__ place, int k, int64_t rows,
                                                     char *__restrict__ out, int64_t row_bytes_o)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= total)
        return;
    const int64_t t = i / chunks, c = i - t * chunks;
    const u32x4 v = *reinterpret_cast<const u32x4 *>(X + t * row_bytes_x + c * 16);
    for (int j = 0; j < k; ++j) {
        const int64_t p = place[t * k + j];
        if (p >= 0 && p < rows)
            *reinterpret_cast<u32x4 *>(out + p * row_bytes_o + c * 16) = v;
    }
}

// A thread owns one chunk of one token's sum.
template <typename T_>
__global__ __launch_bounds__(256) void combine_kernel(const T_ *__restrict__ Y, int64_t ldy, const int32_t *__restrict__ place,
                                                      uint32_t chunks, int64_t total, int k, int64_t rows,
                                                      const float *__restrict__ weights, const T_ *residual, int64_t ldr,
                                                      T_ *out, int64_t ldo)
{
    constexpr int N = Chunk<T_>::N;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= total)
        return;
    const int64_t t = i / chunks, c = (i - t * chunks) * N;
    float sum[N];
    if (residual) {
        Chunk<T_>::widen(*reinterpret_cast<const u32x4 *>(residual + t * ldr + c), sum);
    } else {
#pragma unroll
        for (int x = 0; x < N; ++x)
            sum[x] = 0.0f;
    }
    for (int j = 0; j < k; ++j) {
        const int64_t p = place[t * k + j];
        if (p >= 0 && p < rows) {
            const float w = weights ? weights[t * k + j] : 1.0f;
            float v[N];
            Chunk<T_>::widen(*reinterpret_cast<const u32x4 *>(Y + p * ldy + c), v);
#pragma unroll
            for (int x = 0; x < N; ++x)
                sum[x] = fmaf(w, v[x], sum[x]);
        }
    }
    *reinterpret_cast<u32x4 *>(out + t * ldo + c) = Chunk<T_>::narrow(sum);
}

// Gradient of the weighted sum: a wavefront owns a token.
template <typename T_>
__global__ __launch_bounds__(256) void combine_grad_kernel(const T_ *__restrict__ dout, int64_t ldg, const T_ *__restrict__ Y,
                                                           int64_t ldy, const int32_t *__restrict__ place, int64_t T, int k,
                                                           int64_t rows, const float *__restrict__ weights, uint32_t chunks,
                                                           T_ *__restrict__ dY, int64_t lddy, float *__restrict__ dweights)
{
    constexpr int N = Chunk<T_>::N;
    const int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (t >= T)
        return;
    for (int j = 0; j < k; ++j) {
        const int64_t p = place[t * k + j];
        float dot = 0.0f;
        if (p >= 0 && p < rows) {
            const float w = weights[t * k + j];
            for (uint32_t c = lane; c < chunks; c += 64) {
                float g[N], y[N];
                Chunk<T_>::widen(*reinterpret_cast<const u32x4 *>(dout + t * ldg + c * N), g);
                Chunk<T_>::widen(*reinterpret_cast<const u32x4 *>(Y + p * ldy + c * N), y);
#pragma unroll
                for (int x = 0; x < N; ++x) {
                    dot = fmaf(g[x], y[x], dot);
                    g[x] *= w;
                }
                *reinterpret_cast<u32x4 *>(dY + p * lddy + c * N) = Chunk<T_>::narrow(g);
            }
        }
#pragma unroll
        for (int step = 32; step > 0; step /= 2)
            dot += __shfl_xor(dot, step, 64);
        if (lane == 0)
            dweights[t * k + j] = dot;
    }
}

// ------------------------------------------------------------------ host side --
// One block sorts alone up to this many pairs; beyond, its time goes with the pairs.  8 and 256 experts in one launch and in two: 2048
// pairs 4.6 / 5.3 and 6.9 / 7.7 us, 4096 5.8 / 6.8 and 7.9 / 8.8, 6144 7.0 / 8.4 and 8.0 / 9.3, 8192 8.4 / 10.0 and 8.3 / 9.4, 16384 14.8 / 17.9
// and 8.5 / 9.6.
constexpr int64_t kSortAlone = 8192;

static int64_t sort_per_block(int64_t pairs)
{
    const int64_t even = (pairs + 255) / 256, least = 4096;   // at most 256 blocks
    return ((even > least ? even : least) + kSortThreads - 1) / kSortThreads * kSortThreads;
}

template <typename ID>
static dass_status launch_sort(const void *ids, int64_t pairs, int E, int32_t *offsets, int32_t *order, int32_t *place,
                               int32_t *counts, hipStream_t stream)
{
    const bool alone = pairs <= kSortAlone;
    const int64_t per_block = alone ? (pairs + kSortThreads - 1) / kSortThreads * kSortThreads : sort_per_block(pairs);
    const unsigned blocks = alone ? 1 : (unsigned)((pairs + per_block - 1) / per_block);
    const ID *p = static_cast<const ID *>(ids);
    if (!alone) {
        hipLaunchKernelGGL(sort_count_kernel<ID>, dim3(blocks), dim3(kSortThreads), 0, stream, p, pairs, per_block, E, counts);
        const dass_status s = check_launch("sort count kernel");
        if (s != DASS_OK)
            return s;
    }
    int bits = 0;
    while ((1 << bits) < E)
        ++bits;
    const size_t lds = (size_t)kSortWaves * (E + 1) * 4;
    if (lds > 48 * 1024) {   // beyond what a launch gets without asking (asking takes 0.9 us of every call)
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(sort_place_kernel<ID>),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize, kSortWaves * (kMaxExperts + 1) * 4);
        if (e != hipSuccess)
            return fail(DASS_ERR_HIP, "sort place kernel: %s", hipGetErrorString(e));
    }
    hipLaunchKernelGGL(sort_place_kernel<ID>, dim3(blocks), dim3(kSortThreads), lds, stream, p, pairs, per_block, E, bits,
                       alone ? nullptr : counts, offsets, order, place);
    return check_launch("sort place kernel");
}

static bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// Sizes that every call here has: T tokens of k slots whose pairs an int32 numbers.
static dass_status check_pairs(const char *fn, int64_t T, int64_t k)
{
    if (T <= 0 || k <= 0)
        return fail(DASS_ERR_SHAPE, "%s: T=%lld k=%lld must be positive", fn, (long long)T, (long long)k);
    if (k > kMaxSlots)
        return fail(DASS_ERR_SHAPE, "%s: k=%lld slots, at most %d", fn, (long long)k, kMaxSlots);
    if (T > 0x7fffffffLL / k)
        return fail(DASS_ERR_SHAPE, "%s: T * k = %lld * %lld pairs do not fit an int32", fn, (long long)T, (long long)k);
    return DASS_OK;
}

// A matrix of rows of d elements: pointer and stride.
static dass_status check_rows(const char *fn, const char *name, const void *p, int64_t rows, int64_t ld, int64_t d, int vec)
{
    if (!p)
        return fail(DASS_ERR_NULL, "%s: %s must not be NULL", fn, name);
    if (ld < d || ld > 1LL << 36)
        return fail(DASS_ERR_SHAPE, "%s: rows of %s: stride %lld < d=%lld or beyond 2^36", fn, name, (long long)ld, (long long)d);
    if (rows > kMaxSpan / ld)
        return fail(DASS_ERR_SHAPE, "%s: %lld rows of %s with stride %lld span more than 2^46 elements", fn, (long long)rows, name,
                    (long long)ld);
    if (!aligned16(p) || ld % vec != 0)
        return fail(DASS_ERR_ALIGN, "%s: %s must be 16-byte aligned, its row stride a multiple of %d elements", fn, name, vec);
    return DASS_OK;
}

static dass_status check_row_length(const char *fn, int64_t d, dass_dtype dt)
{
    if (!valid_dtype(dt))
        return fail(DASS_ERR_DTYPE, "%s: unknown dtype %d", fn, (int)dt);
    if (d <= 0 || d % vec_elems(dt) != 0 || d > 1 << 24)
        return fail(DASS_ERR_SHAPE, "%s: d=%lld must be a positive multiple of %d, at most 2^24", fn, (long long)d, vec_elems(dt));
    return DASS_OK;
}

// An output that begins where an input does.
static dass_status check_apart(const char *fn, const char *name, const void *out, const void *in)
{
    return out != in ? DASS_OK : fail(DASS_ERR_ARG, "%s: %s must not overlap an input", fn, name);
}

// Workgroups of 256 threads for a number of 16-byte chunks; 0: more than one launch holds.
static unsigned chunk_blocks(int64_t chunks)
{
    const int64_t blocks = (chunks + 255) / 256;
    return blocks <= 0xffffffffLL / 256 ? (unsigned)blocks : 0;   // a launch has fewer than 2^32 threads
}

}  // namespace dass

extern "C" size_t dass_expert_sort_workspace_bytes(int64_t T, int64_t k, int64_t n_experts)
{
    using namespace dass;
    if (T <= 0 || k <= 0 || n_experts <= 0 || n_experts > kMaxExperts || k > kMaxSlots || T > 0x7fffffffLL / k ||
        T * k <= kSortAlone)
        return 0;
    const int64_t per_block = sort_per_block(T * k);
    return (size_t)((T * k + per_block - 1) / per_block * n_experts * 4);
}

extern "C" dass_status dass_expert_sort(const void *experts, int expert_bytes, int64_t T, int64_t k, int64_t n_experts,
                                        int32_t *offsets, int32_t *order, int32_t *place, void *workspace,
                                        size_t workspace_bytes, void *hip_stream)
{
    using namespace dass;
    const char *fn = "dass_expert_sort";
    if (!experts || !offsets || !order || !place)
        return fail(DASS_ERR_NULL, "%s: experts, offsets, order and place must not be NULL", fn);
    if (expert_bytes != 4 && expert_bytes != 8)
        return fail(DASS_ERR_ARG, "%s: ids of %d bytes, must be 4 or 8", fn, expert_bytes);
    dass_status s = check_pairs(fn, T, k);
    if (s != DASS_OK)
        return s;
    if (n_experts <= 0 || n_experts > kMaxExperts)
        return fail(DASS_ERR_SHAPE, "%s: %lld experts, must be 1 to %d", fn, (long long)n_experts, kMaxExperts);
    if ((reinterpret_cast<uintptr_t>(experts) & (unsigned)(expert_bytes - 1)) || !aligned4(offsets) || !aligned4(order) ||
        !aligned4(place))
        return fail(DASS_ERR_ALIGN, "%s: the integer arrays must be aligned to their elements", fn);
    const size_t need = dass_expert_sort_workspace_bytes(T, k, n_experts);
    if (need > 0 && (!workspace || workspace_bytes < need))
        return fail(DASS_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", fn, workspace ? workspace_bytes : 0, need);
    if (need > 0 && !aligned16(workspace))
        return fail(DASS_ERR_ALIGN, "%s: workspace must be 16-byte aligned", fn);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    int32_t *counts = need > 0 ? static_cast<int32_t *>(workspace) : nullptr;
    return expert_bytes == 4 ? launch_sort<int32_t>(experts, T * k, (int)n_experts, offsets, order, place, counts, stream)
                             : launch_sort<int64_t>(experts, T * k, (int)n_experts, offsets, order, place, counts, stream);
}

extern "C" dass_status dass_expert_gather(const void *X, int64_t T, int64_t ldx, int64_t d, dass_dtype dt,
                                          const int32_t *place, int64_t k, void *out, int64_t ldo, void *hip_stream)
{
    using namespace dass;
    const char *fn = "dass_expert_gather";
    dass_status s = check_row_length(fn, d, dt);
    if (s == DASS_OK)
        s = check_pairs(fn, T, k);
    if (s == DASS_OK)
        s = check_rows(fn, "X", X, T, ldx, d, vec_elems(dt));
    if (s == DASS_OK)
        s = check_rows(fn, "out", out, T * k, ldo, d, vec_elems(dt));
    if (s != DASS_OK)
        return s;
    if (!place)
        return fail(DASS_ERR_NULL, "%s: place must not be NULL", fn);
    if (!aligned4(place))
        return fail(DASS_ERR_ALIGN, "%s: place must be 4-byte aligned", fn);
    const int64_t chunks = d / vec_elems(dt), e = elem_bytes(dt);
    const unsigned blocks = chunk_blocks(T * chunks);
    if (blocks == 0)
        return fail(DASS_ERR_SHAPE, "%s: too many rows for one launch; split the tokens", fn);
    s = check_apart(fn, "out", out, X);
    if (s != DASS_OK)
        return s;
    hipLaunchKernelGGL(gather_kernel, dim3(blocks), dim3(256), 0, static_cast<hipStream_t>(hip_stream),
                       static_cast<const char *>(X), ldx * e, (uint32_t)chunks, T * chunks, place, (int)k, T * k,
                       static_cast<char *>(out), ldo * e);
    return check_launch("gather kernel");
}

extern "C" dass_status dass_expert_combine(const void *Y, int64_t ldy, const int32_t *place, int64_t T, int64_t k,
                                           const float *weights, const void *residual, int64_t ldr, int64_t d,
                                           dass_dtype dt, void *out, int64_t ldo, void *hip_stream)
{
    using namespace dass;
    const char *fn = "dass_expert_combine";
    dass_status s = check_row_length(fn, d, dt);
    if (s == DASS_OK)
        s = check_pairs(fn, T, k);
    if (s == DASS_OK)
        s = check_rows(fn, "Y", Y, T * k, ldy, d, vec_elems(dt));
    if (s == DASS_OK && residual)
        s = check_rows(fn, "residual", residual, T, ldr, d, vec_elems(dt));
    if (s == DASS_OK)
        s = check_rows(fn, "out", out, T, ldo, d, vec_elems(dt));
    if (s != DASS_OK)
        return s;
    if (!place)
        return fail(DASS_ERR_NULL, "%s: place must not be NULL", fn);
    if (!aligned4(place) || !aligned4(weights))
        return fail(DASS_ERR_ALIGN, "%s: place and weights must be 4-byte aligned", fn);
    const int64_t chunks = d / vec_elems(dt);
    const unsigned blocks = chunk_blocks(T * chunks);
    if (blocks == 0)
        return fail(DASS_ERR_SHAPE, "%s: too many rows for one launch; split the tokens", fn);
    s = check_apart(fn, "out", out, Y);
    if (s == DASS_OK && ldr != ldo)
        s = check_apart(fn, "out with another stride", out, residual);
    if (s != DASS_OK)
        return s;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (dt == DASS_BF16)
        hipLaunchKernelGGL(combine_kernel<uint16_t>, dim3(blocks), dim3(256), 0, stream, static_cast<const uint16_t *>(Y), ldy,
                           place, (uint32_t)chunks, T * chunks, (int)k, T * k, weights,
                           static_cast<const uint16_t *>(residual), ldr, static_cast<uint16_t *>(out), ldo);
    else
        hipLaunchKernelGGL(combine_kernel<float>, dim3(blocks), dim3(256), 0, stream, static_cast<const float *>(Y), ldy, place,
                           (uint32_t)chunks, T * chunks, (int)k, T * k, weights, static_cast<const float *>(residual), ldr,
                           static_cast<float *>(out), ldo);
    return check_launch("combine kernel");
}

extern "C" dass_status dass_expert_combine_backward(const void *dout, int64_t ldg, const void *Y, int64_t ldy,
                                                    const int32_t *place, int64_t T, int64_t k, const float *weights,
                                                    int64_t d, dass_dtype dt, void *dY, int64_t lddy, float *dweights,
                                                    void *hip_stream)
{
    using namespace dass;
    const char *fn = "dass_expert_combine_backward";
    dass_status s = check_row_length(fn, d, dt);
    if (s == DASS_OK)
        s = check_pairs(fn, T, k);
    if (s == DASS_OK)
        s = check_rows(fn, "dout", dout, T, ldg, d, vec_elems(dt));
    if (s == DASS_OK)
        s = check_rows(fn, "Y", Y, T * k, ldy, d, vec_elems(dt));
    if (s == DASS_OK)
        s = check_rows(fn, "dY", dY, T * k, lddy, d, vec_elems(dt));
    if (s != DASS_OK)
        return s;
    if (!place || !weights || !dweights)
        return fail(DASS_ERR_NULL, "%s: place, weights and dweights must not be NULL", fn);
    if (!aligned4(place) || !aligned4(weights) || !aligned4(dweights))
        return fail(DASS_ERR_ALIGN, "%s: place, weights and dweights must be 4-byte aligned", fn);
    const int64_t blocks = (T + 3) / 4;
    if (blocks > 0xffffffffLL / 256)
        return fail(DASS_ERR_SHAPE, "%s: too many rows for one launch; split the tokens", fn);
    s = check_apart(fn, "dY", dY, dout);
    if (s == DASS_OK)
        s = check_apart(fn, "dY", dY, Y);
    if (s == DASS_OK)
        s = check_apart(fn, "dweights", dweights, weights);
    if (s != DASS_OK)
        return s;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const uint32_t chunks = (uint32_t)(d / vec_elems(dt));
    if (dt == DASS_BF16)
        hipLaunchKernelGGL(combine_grad_kernel<uint16_t>, dim3((unsigned)blocks), dim3(256), 0, stream,
                           static_cast<const uint16_t *>(dout), ldg, static_cast<const uint16_t *>(Y), ldy, place, T, (int)k,
                           T * k, weights, chunks, static_cast<uint16_t *>(dY), lddy, dweights);
    else
        hipLaunchKernelGGL(combine_grad_kernel<float>, dim3((unsigned)blocks), dim3(256), 0, stream,
                           static_cast<const float *>(dout), ldg, static_cast<const float *>(Y), ldy, place, T, (int)k, T * k,
                           weights, chunks, static_cast<float *>(dY), lddy, dweights);
    return check_launch("combine gradient kernel");
}
