// The products of dass_linear and dass_linear_backward on the matrix cores, tile by tile (bf16 and f32).
//
// A workgroup owns a tile of 32 RB rows x 32 CB columns of the output, its four wavefronts (2 x 2) a quarter each:
// RB x CB blocks of 16 x 16, for 8 x 8 all 256 accumulation registers of a lane.  Slabs of 128 bytes of k (64 bf16, 32 f32) go
// from global memory straight into LDS (16 bytes a lane, no registers in between).  Output columns are the
// instruction's M index and rows its N index, so a lane holds four neighbouring columns of a row.  bf16:
// v_mfma_f32_16x16x32_bf16; f32: four v_mfma_f32_16x16x4_f32, the i-th on the i-th of the four k that a lane holds of a row, so
// that it covers k = i, 4 + i, 8 + i, 12 + i of both operands.
//
// An operand comes in one of two forms, and LDS holds it in the form that it has in memory:
//   by rows   a wave-load is 8 rows x 128 bytes; a lane's 16 bytes of a row are one read.  16-byte chunk c of
//             row r lies in slot c ^ (r / 2 mod 8): 16 rows of one chunk meet 16 places of the banks.
//   k by k    a wave-load is 1 KB of lines of k.  bf16: ds_read_b64_tr_b16 reads a 4 x 16 block of k x rows for 16
//             lanes and gives each lane the four k of one row; two of them are a lane's eight k.  A block's 32 bytes
//             of line k lie in place piece ^ f(k), f(k) = (k mod 4) + 4 (k / 8 mod 2), so that the eight lines
//             that 32 lanes read at a time meet all 64 banks once.  f32: a lane's four k are four reads of 4 bytes; a block's 64
//             bytes of line k lie in place piece ^ (k / 4 mod 4), so that the four lines of a read meet all banks once.
// So no operand is transposed in memory: the three products (linear.h) differ in their operands' forms alone.
//
// LDS is two rings, ND parts of the operand that leads and NF of the one that follows, as many as 160 KB hold (in the short tiles
// 64 KB).  The places of slab s are free after the one barrier of the slab, which stands where every wavefront has read its
// last fragments of it, in the middle of its second K step; the loads of the follower's slab s + NF and the leader's s + ND
// are spread over the matrix instructions from there to the next barrier.  The wait before a barrier counts the loads that
// may still be on their way, so their order is pinned; only slabs that exist are requested, and the last slabs have bodies
// of their own with fewer to wait for.
//
// Reads outside a matrix: each operand is a raw buffer that starts at the tile's first row and ends with its last
// valid element; what lies beyond reads as 0.  Lane offsets are 32-bit registers, the scalar offset is at most a row
// (by rows) or none (k by k, whose buffer moves with the slab), so the length less the scalar offset is never negative.  By
// rows, chunks of the last slab that lie beyond k are given an offset outside the buffer.
//
// Grids of few tiles split k over blockIdx.z: each share writes its sums as f32 to a place of its own in the workspace, and a second
// launch adds them up in order and finishes the outputs (join_kernel).
#pragma once

#include "linear.h"
#include "tile_order.h"

#include <cstdlib>
#include <atomic>
#include <type_traits>
#include <utility>

namespace dass {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((address_space(3))) void *lds_ptr_t;
typedef __attribute__((address_space(3))) s16x4 *lds_s16x4_t;

// f(0), f(1), .. f(N - 1) with compile-time numbers.  (The loops of a slab are too large for the compiler's unrolling, and what is
// not unrolled leaves its registers in memory.)
template <typename F, int... I>
__device__ __forceinline__ void for_each_of(F &&f, std::integer_sequence<int, I...>)
{
    (f(std::integral_constant<int, I>{}), ...);
}
template <int FROM, int TO, typename F>
__device__ __forceinline__ void for_each(F &&f)
{
    if constexpr (TO > FROM)
        for_each_of([&](auto i) __attribute__((always_inline)) { f(std::integral_constant<int, FROM + decltype(i)::value>{}); },
                    std::make_integer_sequence<int, TO - FROM>{});
}

constexpr int kSlabBytes = 128;
template <bool SHORT>
constexpr int lds_bytes()
{
    return (SHORT ? 64 : 160) * 1024;
}
constexpr int kOutside = 0x7fffffff;

// A raw buffer: 48 bits of address, no stride, its length in bytes.  Its words, the same in every lane, are put into scalar registers
// here, as the loads by hand need them; left to itself the compiler does so with every optimisation on alone.
__device__ __forceinline__ u32x4 raw_buffer(const void *p, int bytes)
{
    const uint64_t a = reinterpret_cast<uint64_t>(p);
    const auto scalar = [](uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); };
    return u32x4{scalar((uint32_t)a), scalar((uint32_t)(a >> 32) & 0xffffu), scalar((uint32_t)bytes), 0x00020000u};
}

// One wave-load of 16 bytes a lane from a buffer straight into LDS: the builtin where both operands are by rows, and
// by hand where one is not.  Beside the builtin the compiler waits for every such load before each transposing LDS read (it takes the
// read to depend on them), which empties the pipeline once a load: dX and dW of 6000 rows of 4096 x 11008 1590 us, by
// hand 548 and 444; of products without such reads the builtin is 4 % ahead.  (Not a template: with arguments that depend on
// one, the host pass rejects the builtin.)  The block by hand writes no register; m0 is an operand of it, so that
// the compiler knows what it holds.  The waits for it are those before the barriers.  Its s_nop covers the wait states between a scalar register's last write and its use as an address.
__device__ __forceinline__ void load_to_lds(const u32x4 &buffer, char *dst, uint32_t lane_off, int off)
{
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(
        reinterpret_cast<void *>((uint64_t)buffer[1] << 32 | buffer[0]), 0, (int)buffer[2], (int)buffer[3]);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_ptr_t)dst, 16, lane_off, off, 0, 0);
}
__device__ __forceinline__ void load_to_lds_by_hand(const u32x4 &buffer, char *dst, uint32_t lane_off, int off)
{
    const uint32_t at = (uint32_t)(uintptr_t)(lds_ptr_t)dst;
    asm volatile("s_nop 4\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"{m0}"(at), "v"(lane_off), "s"(buffer), "s"(off) : "memory");
}

__device__ __forceinline__ void block_barrier()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// lgkmcnt(0) and at most N vector memory operations on their way
template <int N>
__device__ __forceinline__ void wait_loads()
{
    static_assert(N >= 0 && N < 64, "vmcnt is a 6-bit counter");
    __builtin_amdgcn_s_waitcnt(0x0070 | (N & 15) | ((N >> 4) << 14));
}

// One operand of a workgroup: its loads into LDS and its fragments from there.  B: blocks of 16 rows of a wavefront.
template <typename T_, bool BY_ROWS, int B, bool BY_HAND>
struct Part;

template <typename T_, int B, bool BY_HAND>
struct Part<T_, true, B, BY_HAND> {
    static constexpr int LOADS = B, READS = B, UNIT = 32 * B * 128, E = sizeof(T_);
    struct Frags {
        u32x4 v[B];
        __device__ __forceinline__ u32x4 get(int b) const { return v[b]; }
    };
    u32x4 buffer;
    uint32_t off[LOADS];
    int chunk[2], k_bytes, frag;

    __device__ __forceinline__ void init(const T_ *m, int64_t ld, int64_t row0, int64_t rows, int64_t k0, int64_t k, int wave, int lane, int part)
    {
        const int64_t n = rows - row0 < 32 * B ? rows - row0 : 32 * B;
        buffer = raw_buffer(m + row0 * ld + k0, (int)(((n - 1) * ld + k) * E));
        k_bytes = (int)(k * E);
        const int sub = lane >> 3;
        chunk[0] = ((lane & 7) ^ (sub >> 1)) * 16;
        chunk[1] = chunk[0] ^ 64;                          // rows 8 further on: r / 2 has changed by 4
#pragma unroll
        for (int q = 0; q < LOADS; ++q)
            off[q] = (uint32_t)(((wave * LOADS + q) * 8 + sub) * ld * E) + chunk[q & 1];
        const int r = part * 16 * B + (lane & 15);
        frag = r * 128 + (((lane >> 4) ^ (r >> 1)) & 7) * 16;
    }
    __device__ __forceinline__ void begin_slab(int) {}
    // LAST: the slab may be the last one, whose chunks may lie beyond k
    template <bool LAST>
    __device__ __forceinline__ void load(char *unit, int wave, int slab, int q) const
    {
        const int at = slab * kSlabBytes;
        const uint32_t lane_off = !LAST || at + chunk[q & 1] < k_bytes ? off[q] : (uint32_t)kOutside;
        if constexpr (BY_HAND)
            load_to_lds_by_hand(buffer, unit + (wave * LOADS + q) * 1024, lane_off, at);
        else
            load_to_lds(buffer, unit + (wave * LOADS + q) * 1024, lane_off, at);
    }
    // read x of the fragments of K step kk
    __device__ __forceinline__ void read(const char *unit, int kk, int x, Frags &f) const
    {
        f.v[x] = *reinterpret_cast<const u32x4 *>(unit + (frag ^ (kk * 64)) + x * 2048);
    }
};

// The lines of k of an operand that is stored k by k.
template <typename T_, int B, bool BY_HAND>
struct Lines {
    static constexpr int LOADS = B, UNIT = 32 * B * 128, E = sizeof(T_), SLAB = kSlabBytes / E;
    static constexpr int LINE = 32 * B * E, SLOTS = LINE / 16, LINES = 1024 / LINE;   // bytes, chunks; lines of a wave-load
    static_assert(LINES * LINE == 1024 && LINES > 0, "whole lines");
    const T_ *m;
    int64_t ld, depth, width, lo = 0;
    int first = 0, fold = 0x7fffffff;
    u32x4 buffer;
    uint32_t off[LOADS];

    // k runs over the same `slabs` slabs twice, this workgroup's beginning with the `begin`-th; the second time `lo_` elements further on.
    __device__ __forceinline__ void twice(int begin, int slabs, int64_t lo_)
    {
        first = begin;
        fold = slabs;
        lo = lo_;
    }
    // swap(line): what the place of a 16-byte chunk is XORed with
    template <typename F>
    __device__ __forceinline__ void init_lines(const T_ *base, int64_t ld_, int64_t row0, int64_t rows, int64_t k0, int64_t k, int wave, int lane, F swap)
    {
        m = base + k0 * ld_ + row0;
        ld = ld_;
        depth = k;
        width = rows - row0 < 32 * B ? rows - row0 : 32 * B;
#pragma unroll
        for (int q = 0; q < LOADS; ++q) {
            const int line = (wave * LOADS + q) * LINES + lane / SLOTS;
            off[q] = (uint32_t)(line * ld * E) + ((lane % SLOTS) ^ swap(line)) * 16;
        }
    }
    __device__ __forceinline__ void begin_slab(int slab)
    {
        const T_ *from = m;
        if constexpr (BY_HAND) {
            slab += first;
            if (slab >= fold) {
                slab -= fold;
                from += lo;
            }
        }
        const int64_t left = depth - (int64_t)slab * SLAB, lines = left < SLAB ? left : SLAB;
        buffer = raw_buffer(from + (int64_t)slab * SLAB * ld, (int)(((lines - 1) * ld + width) * E));
    }
    template <bool LAST>
    __device__ __forceinline__ void load(char *unit, int wave, int, int q) const
    {
        if constexpr (BY_HAND)
            load_to_lds_by_hand(buffer, unit + (wave * LOADS + q) * 1024, off[q], 0);
        else
            load_to_lds(buffer, unit + (wave * LOADS + q) * 1024, off[q], 0);
    }
};

template <int B, bool BY_HAND>
struct Part<uint16_t, false, B, BY_HAND> : Lines<uint16_t, B, BY_HAND> {
    static_assert(BY_HAND, "it is read by transposing reads");
    typedef Lines<uint16_t, B, BY_HAND> Base;
    static constexpr int READS = 2 * B;
    struct Frags {
        s16x4 v[2 * B];
        __device__ __forceinline__ u32x4 get(int b) const
        {
            return __builtin_bit_cast(u32x4, __builtin_shufflevector(v[2 * b], v[2 * b + 1], 0, 1, 2, 3, 4, 5, 6, 7));
        }
    };
    int frag;

    static __device__ __forceinline__ int f_of(int k) { return (k & 3) | (k >> 1 & 4); }
    __device__ __forceinline__ void init(const uint16_t *base, int64_t ld, int64_t row0, int64_t rows, int64_t k0, int64_t k, int wave, int lane, int part)
    {
        this->init_lines(base, ld, row0, rows, k0, k, wave, lane, [](int line) { return f_of(line) << 1; });
        const int g = lane >> 4, i = lane & 15, line = 8 * g + (i >> 2);
        frag = line * Base::LINE + (((part * B) ^ f_of(line)) * 32) + (i & 3) * 8;
    }
    __device__ __forceinline__ void read(const char *unit, int kk, int x, Frags &f) const
    {
        f.v[x] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (lds_s16x4_t)(unit + (frag ^ (x / 2 * 32)) + (x % 2 * 4 + kk * 32) * Base::LINE));
    }
};

template <int B, bool BY_HAND>
struct Part<float, false, B, BY_HAND> : Lines<float, B, BY_HAND> {
    typedef Lines<float, B, BY_HAND> Base;
    static constexpr int READS = 4 * B;
    struct Frags {
        uint32_t v[4 * B];
        __device__ __forceinline__ u32x4 get(int b) const { return u32x4{v[4 * b], v[4 * b + 1], v[4 * b + 2], v[4 * b + 3]}; }
    };
    int frag;

    static __device__ __forceinline__ int f_of(int k) { return k >> 2 & 3; }
    __device__ __forceinline__ void init(const float *base, int64_t ld, int64_t row0, int64_t rows, int64_t k0, int64_t k, int wave, int lane, int part)
    {
        this->init_lines(base, ld, row0, rows, k0, k, wave, lane, [](int line) { return f_of(line) << 2; });
        const int g = lane >> 4, line = 4 * g;
        frag = line * Base::LINE + (((part * B) ^ f_of(line)) * 64) + (lane & 15) * 4;
    }
    __device__ __forceinline__ void read(const char *unit, int kk, int x, Frags &f) const
    {
        f.v[x] = *reinterpret_cast<const uint32_t *>(unit + (frag ^ (x / 4 * 64)) + (x % 4 + kk * 16) * Base::LINE);
    }
};

__device__ __forceinline__ f32x4 multiply_add(const u32x4 &q, const u32x4 &p, const f32x4 &acc, uint16_t)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, q), __builtin_bit_cast(bf16x8, p), acc, 0, 0, 0);
}
__device__ __forceinline__ f32x4 multiply_add(const u32x4 &q, const u32x4 &p, f32x4 acc, float)
{
    const f32x4 a = __builtin_bit_cast(f32x4, q), b = __builtin_bit_cast(f32x4, p);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], acc, 0, 0, 0);
    return acc;
}

__device__ __forceinline__ void store(void *p, const u32x4 &v, bool streamed)
{
    if (streamed) {
        asm volatile("");   // on both sides, or the compiler makes one plain store of the two
        __builtin_nontemporal_store(v, static_cast<u32x4 *>(p));
        asm volatile("");
    } else {
        *static_cast<u32x4 *>(p) = v;
    }
}

// The epilogue of one 16-byte chunk of a row (8 bf16, 4 f32), with the chunks of mul and residual at hand; `col` is inside.
template <typename T_, int N = Chunk<T_>::N>
__device__ __forceinline__ void finish(const Epilogue<T_> &ep, bool streamed, int64_t row, int64_t col, const float (&bias)[N],
                                       const u32x4 &mul, const u32x4 &residual, float (&v)[N])
{
    typedef Chunk<T_> C;
    constexpr bool FAST = sizeof(T_) == 2;
    float w[N];
    if (ep.bias) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] += bias[i];
    }
    if (ep.pre)
        store(ep.pre + row * ep.ldp + col, C::narrow(v), streamed);
    act_values<FAST>(v, ep.act);
    if (ep.mul) {
        C::widen(mul, w);
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] *= w[i];
    }
    if (ep.residual) {
        C::widen(residual, w);
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] += w[i];
    }
    store(ep.out + row * ep.ldo + col, C::narrow(v), streamed);
}

// Every XCD one contiguous run of the tiles, as tile_order.h has them, for a number of row tiles that only the device knows.
__device__ __forceinline__ TileOrder order_runs(uint32_t tiles_r, uint32_t tiles_c, uint32_t max_band)
{
    const uint32_t bands = (tiles_r + max_band - 1) / max_band;
    TileOrder o = {};
    o.tiles_t = tiles_r;
    o.tiles_n = tiles_c;
    o.band = tiles_r > 0 ? (tiles_r + bands - 1) / bands : 1;
    o.per_xcd = (tiles_r * tiles_c + kXcds - 1) / kXcds;
    return o;
}

// SHORT: rings of two parts each, 64 KB in all, so that two workgroups share a compute unit and one's loads and stores go on
// beside the other's products: for k of few slabs.
// `block` is a place in the tile order, `nth` the share of k, `expert` is given for dW and found for the others.
template <typename T_, Product PRODUCT, int RB, int CB, bool SHORT>
__device__ __forceinline__ void product_tile(const Operands<T_> &a, const Epilogue<T_> &ep0, const TileOrder &order, const Split &split,
                                             uint32_t block, int expert, uint32_t nth)
{
    constexpr bool BY_HAND = sizeof(T_) == 2 && PRODUCT != kForward;   // transposing reads
    typedef Part<T_, PRODUCT != kWeightGrad, RB, BY_HAND> PartP;
    typedef Part<T_, PRODUCT == kForward, CB, BY_HAND> PartQ;
    constexpr int SLAB = kSlabBytes / sizeof(T_);
    constexpr int BR = 32 * RB, BC = 32 * CB;
    // Ring parts of the operand that leads and of the one that follows.  The weights lead in the large tiles of dX: 6000 rows of 4096 x
    // 11008 486 -> 475 us, over 8 experts 541 -> 533; in the forward product they do not (8192 rows of 4096 x 14336 690, with
    // them 699; over 8 experts 880 and 867).
    constexpr bool Q_LEADS = RB == 8 && PRODUCT == kInputGrad;
    constexpr int ND = SHORT ? 2 : RB == 8 ? 3 : CB == 8 ? 4 : 5, NF = SHORT || RB == 8 ? 2 : CB == 8 ? 3 : 5, LEAD = ND - NF;
    constexpr int LDS = lds_bytes<SHORT>();
    constexpr int NP = Q_LEADS ? NF : ND, NQ = Q_LEADS ? ND : NF;
    static_assert(NP * PartP::UNIT + NQ * PartQ::UNIT <= LDS && (LEAD == 0 || LEAD == 1), "the rings fit");
    constexpr int DL = Q_LEADS ? PartQ::LOADS : PartP::LOADS, FL = Q_LEADS ? PartP::LOADS : PartQ::LOADS, NL = DL + FL;
    constexpr int N = RB * CB;   // matrix instructions of a K step
    extern __shared__ __attribute__((aligned(1024))) char lds[];   // LDS bytes

    uint32_t tile_r, tile_c;   // tile_order.h
    int64_t r0, r_end, k0 = 0, depth = a.depth;
    if (PRODUCT == kWeightGrad || !a.seg.offsets) {
        if (!tile_of_block(order, block, tile_r, tile_c))
            return;
        r0 = (int64_t)tile_r * BR;
        r_end = PRODUCT == kWeightGrad ? a.out_rows : a.seg.rows;
        if constexpr (PRODUCT == kWeightGrad) {
            const Span k = segment(a.seg, expert);
            k0 = k.lo;
            depth = k.hi - k.lo;
        }
    } else {   // the order for the tiles that there are: runs
        const TileList list(a.seg, BR);
        const TileOrder runs = order_runs(list.total, order.tiles_n, BR < BC ? 8 : kPatchT);
        if (list.total == 0 || block / kXcds >= runs.per_xcd || !tile_of_block(runs, block, tile_r, tile_c))
            return;
        const Span r = list.rows(a.seg, BR, (int)tile_r, expert);
        r0 = r.lo;
        r_end = r.hi;
    }
    const int64_t c0 = (int64_t)tile_c * BC;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wr = wave >> 1, wc = wave & 1;

    f32x4 acc[CB][RB];
#pragma unroll
    for (int i = 0; i < CB; ++i)
#pragma unroll
        for (int j = 0; j < RB; ++j)
            acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    const int64_t once = depth;
    const bool two = BY_HAND && a.lo > 0;   // g in two parts: k runs over them one after the other, whole slabs of each
    const int fold = (int)((once + SLAB - 1) / SLAB);
    if (two)
        depth = 2 * (int64_t)fold * SLAB;
    int64_t from = 0;
    if (split.n > 1) {   // this workgroup's share of the slabs, perhaps none
        const int64_t share = ((depth + SLAB - 1) / SLAB + split.n - 1) / split.n * SLAB;
        from = share * nth;
        depth = from >= depth ? 0 : depth - from < share ? depth - from : share;
    }
    const int S = (int)((depth + SLAB - 1) / SLAB);
    if (S > 0) {
    PartP P;
    PartQ Q;
    const T_ *const q = PRODUCT == kWeightGrad ? a.Q : a.Q + (int64_t)expert * a.q_stride;
    const bool p_folds = two && PRODUCT == kWeightGrad;   // (by rows the parts are one row)
    P.init(a.P, a.ldp, r0, r_end, p_folds ? k0 : k0 + from, p_folds ? once : depth, wave, lane, wr);
    Q.init(q, a.ldq, c0, ep0.cols, two ? k0 : k0 + from, two ? once : depth, wave, lane, wc);
    if constexpr (BY_HAND) {
        if (two) {
            if constexpr (PRODUCT == kWeightGrad)
                P.twice((int)(from / SLAB), fold, a.lo);
            Q.twice((int)(from / SLAB), fold, 0);
        }
    }
    char *const p_ring = lds, *const q_ring = lds + NP * PartP::UNIT;

    // ---- the loads.  Iteration t (after the barrier of slab t) requests the follower's slab t + NF, then the leader's t + ND.
    auto load_p = [&](int unit, int slab, int q, auto last) __attribute__((always_inline)) {
        P.template load<decltype(last)::value>(p_ring + unit * PartP::UNIT, wave, slab, q);
        __builtin_amdgcn_sched_barrier(0);
    };
    auto load_q = [&](int unit, int slab, int q, auto last) __attribute__((always_inline)) {
        Q.template load<decltype(last)::value>(q_ring + unit * PartQ::UNIT, wave, slab, q);
        __builtin_amdgcn_sched_barrier(0);
    };
    auto load = [&](auto leader, int unit, int slab, int q, auto last) __attribute__((always_inline)) {
        if constexpr (decltype(leader)::value == Q_LEADS)
            load_q(unit, slab, q, last);
        else
            load_p(unit, slab, q, last);
    };
    auto begin_slab = [&](auto leader, int slab) __attribute__((always_inline)) {
        if constexpr (decltype(leader)::value == Q_LEADS)
            Q.begin_slab(slab);
        else
            P.begin_slab(slab);
    };
    constexpr std::true_type LEADER{};
    constexpr std::false_type FOLLOWER{};
    constexpr int AT_ONCE = (NL + 3) / 4;   // of an iteration's loads, those right after its barrier
    static_assert(AT_ONCE <= FL, "they are the follower's");
    auto whole_leader = [&](int slab) {
        if (slab < S) {
            begin_slab(LEADER, slab);
#pragma unroll
            for (int q = 0; q < DL; ++q)
                load(LEADER, slab % ND, slab, q, std::true_type{});
        }
    };
    if (LEAD == 1)
        whole_leader(0);
#pragma unroll
    for (int t = -NF; t < -1; ++t) {
        if (t + NF < S) {
            begin_slab(FOLLOWER, t + NF);
#pragma unroll
            for (int q = 0; q < FL; ++q)
                load(FOLLOWER, t + NF, t + NF, q, std::true_type{});
        }
        whole_leader(t + ND);
    }
    if (NF - 1 < S) {
        begin_slab(FOLLOWER, NF - 1);
#pragma unroll
        for (int q = 0; q < AT_ONCE; ++q)
            load(FOLLOWER, NF - 1, NF - 1, q, std::true_type{});
    }
    // The sums stay in accumulation registers: cleared while the loads are on their way, and held there between slabs (left to
    // itself the compiler moves some to and fro, or spills in the first slab).
    auto pin = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < CB; ++i)
#pragma unroll
            for (int j = 0; j < RB; ++j)
                asm volatile("" : "+a"(acc[i][j]));
    };
    pin();
    // slab 0 has landed: all but the first parts may be on their way
    auto begin = [&](auto slabs_tag) __attribute__((always_inline)) {
        constexpr int HAVE = decltype(slabs_tag)::value;   // slabs, at most ND
        constexpr int D_OUT = (HAVE < ND - 1 ? HAVE : ND - 1) - 1, F_OUT = (HAVE < NF - 1 ? HAVE : NF - 1) - 1;
        constexpr int OUT = D_OUT * DL + (F_OUT > 0 ? F_OUT : 0) * FL + (HAVE >= NF ? AT_ONCE : 0);
        wait_loads<OUT>();
    };
    static_assert(NF >= 2, "the follower's first part is requested whole");
    if (S >= ND)
        begin(std::integral_constant<int, ND>{});
    else if (ND > 4 && S == 4)
        begin(std::integral_constant<int, (ND > 4 ? 4 : 1)>{});
    else if (ND > 3 && S == 3)
        begin(std::integral_constant<int, (ND > 3 ? 3 : 1)>{});
    else if (S == 2)
        begin(std::integral_constant<int, 2>{});
    else
        begin(std::integral_constant<int, 1>{});
    block_barrier();

    // ---- fragments, in the order in which the matrix instructions want them: two of P, those of Q, the others of P
    struct Frags {
        typename PartP::Frags p;
        typename PartQ::Frags q;
    };
    constexpr int RP = PartP::READS / RB, READS = PartP::READS + PartQ::READS;
    auto read_one = [&](Frags &f, int pu, int qu, int kk, auto x) __attribute__((always_inline)) {
        constexpr int X = decltype(x)::value;
        if constexpr (X < 2 * RP)
            P.read(p_ring + pu * PartP::UNIT, kk, X, f.p);
        else if constexpr (X < 2 * RP + PartQ::READS)
            Q.read(q_ring + qu * PartQ::UNIT, kk, X - 2 * RP, f.q);
        else
            P.read(p_ring + pu * PartP::UNIT, kk, X - PartQ::READS, f.p);
    };
    // Instruction n of a K step: every one shares an operand with the one before.
    auto multiply = [&](const Frags &f, auto n) __attribute__((always_inline)) {
        constexpr int JP = decltype(n)::value / (2 * CB), X = decltype(n)::value % (2 * CB), I = X / 2, J = 2 * JP + ((X & 1) ^ (I & 1));
        acc[I][J] = multiply_add(f.q.get(I), f.p.get(J), acc[I][J], T_{});
    };

    Frags f0, f1;
    for_each<0, READS>([&](auto x) __attribute__((always_inline)) { read_one(f0, 0, 0, 0, x); });
    int du = 0, fu = 0, du_old = ND - 1, fu_old = NF - 1;   // ring places of slab s and of slab s - 1
    // LEFT: how many slabs follow; STEADY stands for that and more, and never requests the last slab.
    constexpr int STEADY = LEAD == 0 ? ND + 1 : ND;
    auto slab_body = [&](int s, auto left_tag) __attribute__((always_inline)) {
        constexpr int LEFT = decltype(left_tag)::value;
        constexpr auto LAST = std::integral_constant<bool, (LEFT < STEADY)>{};
        constexpr bool OLD_F = LEFT >= NF - 1, OLD_D = LEFT >= ND - 1, NEW_F = LEFT >= NF;   // what iterations s - 1 and s request
        const int du1 = du + 1 == ND ? 0 : du + 1, fu1 = fu + 1 == NF ? 0 : fu + 1;
        const int pu = Q_LEADS ? fu : du, qu = Q_LEADS ? du : fu, pu1 = Q_LEADS ? fu1 : du1, qu1 = Q_LEADS ? du1 : fu1;
        // what goes with instruction POS of the 2 N since a barrier: its share of the loads, in their order
        auto old_loads = [&](auto pos) __attribute__((always_inline)) {
            constexpr int POS = decltype(pos)::value;
            for_each<(POS * NL + 2 * N - 1) / (2 * N), ((POS + 1) * NL + 2 * N - 1) / (2 * N)>([&](auto x) __attribute__((always_inline)) {
                constexpr int X = decltype(x)::value;
                if constexpr (X < FL) {
                    if constexpr (OLD_F)
                        load(FOLLOWER, fu_old, s - 1 + NF, X, LAST);
                } else if constexpr (OLD_D) {
                    load(LEADER, du_old, s - 1 + ND, X - FL, LAST);
                }
            });
        };
        if (OLD_F)
            begin_slab(FOLLOWER, s - 1 + NF);
        if (OLD_D)
            begin_slab(LEADER, s - 1 + ND);
        for_each<0, N>([&](auto n) __attribute__((always_inline)) {   // K step 0
            constexpr int I = decltype(n)::value;
            old_loads(std::integral_constant<int, N / 2 + I>{});
            for_each<(I * READS + N - 1) / N, ((I + 1) * READS + N - 1) / N>([&](auto x) __attribute__((always_inline)) { read_one(f1, pu, qu, 1, x); });
            multiply(f0, n);
            __builtin_amdgcn_sched_barrier(0);
        });
        for_each<0, N / 2>([&](auto n) __attribute__((always_inline)) {   // K step 1, first half
            old_loads(std::integral_constant<int, N / 2 + N + decltype(n)::value>{});
            multiply(f1, n);
            __builtin_amdgcn_sched_barrier(0);
        });
        if constexpr (LEFT > 0) {
            // slab s + 1 has landed, and this wavefront holds its last fragments of slab s
            constexpr int F_OUT = (LEFT < NF - 1 ? LEFT : NF - 1) - 1, D_OUT = (LEFT < ND - 1 ? LEFT : ND - 1) - 1;
            wait_loads<F_OUT * FL + D_OUT * DL>();
            block_barrier();
            if (NEW_F)
                begin_slab(FOLLOWER, s + NF);
        }
        for_each<0, N / 2>([&](auto n) __attribute__((always_inline)) {   // K step 1, second half
            constexpr int I = decltype(n)::value;
            if constexpr (NEW_F)
                for_each<(I * NL + 2 * N - 1) / (2 * N), ((I + 1) * NL + 2 * N - 1) / (2 * N)>(
                    [&](auto x) __attribute__((always_inline)) { load(FOLLOWER, fu, s + NF, x, LAST); });
            if constexpr (LEFT > 0)
                for_each<(I * READS + N / 2 - 1) / (N / 2), ((I + 1) * READS + N / 2 - 1) / (N / 2)>(
                    [&](auto x) __attribute__((always_inline)) { read_one(f0, pu1, qu1, 0, x); });
            multiply(f1, std::integral_constant<int, N / 2 + I>{});
            __builtin_amdgcn_sched_barrier(0);
        });
        du_old = du;
        fu_old = fu;
        du = du1;
        fu = fu1;
    };
    // (the first slab on its own: with one loop the compiler gives the accumulators other registers in every slab and moves
    // them back)
    int s = 0;
    if (S > STEADY) {
        slab_body(s++, std::integral_constant<int, STEADY>{});
        pin();
        for (; s + STEADY < S; ++s) {
            slab_body(s, std::integral_constant<int, STEADY>{});
            pin();
        }
    }
    auto last = [&](auto left_tag) {
        constexpr int LEFT = decltype(left_tag)::value;
        if constexpr (LEFT < STEADY) {
            if (s + LEFT < S) {
                slab_body(s++, left_tag);
                pin();
            }
        }
    };
    last(std::integral_constant<int, 5>{});
    last(std::integral_constant<int, 4>{});
    last(std::integral_constant<int, 3>{});
    last(std::integral_constant<int, 2>{});
    last(std::integral_constant<int, 1>{});
    last(std::integral_constant<int, 0>{});
    static_assert(ND <= 5, "every number of slabs left has its body");
    }

    // ---- epilogue.  A wavefront passes strips of 16 rows through LDS of its own, as f32, so that a lane finishes 16 bytes
    // of neighbouring columns and rows are read and written in whole 128-byte lines.  Up to four strips lie there at a time,
    // and a loop that is not unrolled goes over them: all of it unrolled, with five activations, was 200 KB of code that each tile
    // fetched anew (4096 rows of 512 x 4096 37 us).  mul and residual are requested a strip ahead.
    constexpr int N_CHUNK = Chunk<T_>::N;
    constexpr int SROW = 16 * CB * 4 + 16, LANES = 16 * CB / N_CHUNK, ROWS = 64 / LANES;   // lanes of a row; rows of a read
    constexpr int READS_16 = 16 / ROWS, HELD = SHORT ? 2 : 4;
    static_assert(ROWS * LANES == 64 && HELD * 16 * SROW <= LDS / 4 && RB % HELD == 0, "strips");
    Epilogue<T_> ep = ep0;
    char *const strips = lds + wave * (LDS / 4);
    const int fr = lane & 15, g = lane >> 4;
    int64_t row = r0 + wr * 16 * RB + lane / LANES;
    const int64_t col = c0 + wc * 16 * CB + lane % LANES * N_CHUNK;
    int64_t share = nth * split.stride;   // where this share's sums begin
    if constexpr (PRODUCT == kWeightGrad) {
        ep.out += (int64_t)expert * a.out_stride;
        share += (int64_t)expert * a.out_rows * ep.cols;
    }
    const bool whole = split.n == 1;
    // Stores that bypass the caches leave L2 to the operands (dW of 6000 rows over 8 experts of 4096 x 11008 536 us, 559 without;
    // 8192 rows of 128 x 4096 28.3, 31.3), but write a row's ends in pieces where it does not begin and end on lines, and those
    // cost more than a line that L2 puts together (dW of 7 rows over 18 experts of 3496 x 7456 416 us, 218 through L2).
    const uint64_t begins = reinterpret_cast<uintptr_t>(ep.out) | reinterpret_cast<uintptr_t>(ep.pre) | (ep.ldo | ep.ldp) * sizeof(T_);
    const bool streamed = begins % 128 == 0;
    float bias[N_CHUNK];
#pragma unroll
    for (int i = 0; i < N_CHUNK; ++i)
        bias[i] = 0.0f;
    u32x4 mul[READS_16], residual[READS_16];
    auto request = [&](int64_t first) __attribute__((always_inline)) {
        if constexpr (PRODUCT == kForward) {
#pragma unroll
            for (int t = 0; t < READS_16; ++t) {
                const int64_t r = first + t * ROWS;
                if (whole && r < r_end && col < ep.cols) {
                    if (ep.mul)
                        mul[t] = *reinterpret_cast<const u32x4 *>(ep.mul + r * ep.ldm + col);
                    if (ep.residual)
                        residual[t] = *reinterpret_cast<const u32x4 *>(ep.residual + r * ep.ldr + col);
                }
            }
        }
    };
    request(row);
    if (PRODUCT == kForward && whole && ep.bias && col < ep.cols)
        Chunk<T_>::widen(*reinterpret_cast<const u32x4 *>(ep.bias + (int64_t)expert * ep.cols + col), bias);
    block_barrier();   // the rings are about to be used again
    for_each<0, RB / HELD>([&](auto phase) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < HELD; ++j)
#pragma unroll
            for (int i = 0; i < CB; ++i)
                *reinterpret_cast<f32x4 *>(strips + (j * 16 + fr) * SROW + (i * 16 + 4 * g) * 4) = acc[i][decltype(phase)::value * HELD + j];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll 1
        for (int j = 0; j < HELD; ++j, row += 16) {
            u32x4 mul_now[READS_16], residual_now[READS_16];
#pragma unroll
            for (int t = 0; t < READS_16; ++t) {
                mul_now[t] = mul[t];
                residual_now[t] = residual[t];
            }
            request(row + 16);
#pragma unroll
            for (int t = 0; t < READS_16; ++t) {
                const char *at = strips + (j * 16 + t * ROWS + lane / LANES) * SROW + lane % LANES * N_CHUNK * 4;
                f32x4 part[N_CHUNK / 4];
                float v[N_CHUNK];
#pragma unroll
                for (int i = 0; i < N_CHUNK; ++i) {
                    if (i % 4 == 0)
                        part[i / 4] = *reinterpret_cast<const f32x4 *>(at + i * 4);
                    v[i] = part[i / 4][i % 4];
                }
                const int64_t r = row + t * ROWS;
                if (r < r_end && col < ep.cols) {
                    if (!whole) {
#pragma unroll
                        for (int i = 0; i < N_CHUNK / 4; ++i)
                            *reinterpret_cast<f32x4 *>(split.partial + share + r * ep.cols + col + 4 * i) = part[i];
                    } else if constexpr (PRODUCT == kForward) {
                        finish(ep, streamed, r, col, bias, mul_now[t], residual_now[t], v);
                    } else {
                        store(ep.out + r * ep.ldo + col, Chunk<T_>::narrow(v), streamed);
                    }
                }
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    });
}

template <typename T_, Product PRODUCT, int RB, int CB, bool SHORT>
__global__ __launch_bounds__(256) void product_tile_kernel(const Operands<T_> a, const Epilogue<T_> ep, const TileOrder order, const Split split)
{
    product_tile<T_, PRODUCT, RB, CB, SHORT>(a, ep, order, split, blockIdx.x, blockIdx.y, blockIdx.z);
}

// The outputs of a product whose k was split: the shares' sums are added in their order and finished.  A thread owns 16
// bytes of a row of the output, a workgroup 256 of them in 256 / lanes rows of one expert.
template <typename T_, Product PRODUCT>
__global__ __launch_bounds__(256) void join_kernel(const Operands<T_> a, const Epilogue<T_> ep, const Split split, uint32_t strips)
{
    constexpr int N = Chunk<T_>::N;
    const uint32_t tile = blockIdx.x / strips, strip = blockIdx.x - tile * strips;
    const int64_t col = ((int64_t)strip * 32 + threadIdx.x % 32) * N;
    int expert = 0;
    int64_t row, out_row;
    bool in = col < ep.cols;
    T_ *out = ep.out;
    if constexpr (PRODUCT == kWeightGrad) {   // rows of all experts in a row
        row = (int64_t)tile * 8 + threadIdx.x / 32;
        in = in && row < a.out_rows * a.seg.n;
        const int64_t e = row / a.out_rows;
        out_row = row - e * a.out_rows;
        out += e * a.out_stride;
    } else {
        Span r;
        if (!rows_of_tile(a.seg, tile, 8, expert, r))
            return;
        row = out_row = r.lo + threadIdx.x / 32;
        in = in && row < r.hi;
    }
    if (!in)
        return;
    u32x4 mul, residual;
    float bias[N], v[N];
    if constexpr (PRODUCT == kForward) {
        if (ep.mul)
            mul = *reinterpret_cast<const u32x4 *>(ep.mul + row * ep.ldm + col);
        if (ep.residual)
            residual = *reinterpret_cast<const u32x4 *>(ep.residual + row * ep.ldr + col);
        if (ep.bias)
            Chunk<T_>::widen(*reinterpret_cast<const u32x4 *>(ep.bias + (int64_t)expert * ep.cols + col), bias);
    }
    f32x4 sum[N / 4];
    const float *p = split.partial + row * ep.cols + col;
#pragma unroll
    for (int i = 0; i < N / 4; ++i)
        sum[i] = *reinterpret_cast<const f32x4 *>(p + 4 * i);
#pragma unroll 4
    for (int z = 1; z < split.n; ++z) {
#pragma unroll
        for (int i = 0; i < N / 4; ++i)
            sum[i] += *reinterpret_cast<const f32x4 *>(p + z * split.stride + 4 * i);
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
        v[i] = sum[i / 4][i % 4];
    if constexpr (PRODUCT == kForward)
        finish(ep, false, row, col, bias, mul, residual, v);
    else
        *reinterpret_cast<u32x4 *>(out + out_row * ep.ldo + col) = Chunk<T_>::narrow(v);
}

// ------------------------------------------------------------------ host side --
// More LDS than a launch gets without asking: asked for once a kernel and device (0.9 us of a call otherwise).
template <auto KERNEL, int BYTES>
static dass_status reserve_lds(const char *fn)
{
    static std::atomic<uint64_t> done{0};
    int device = 0;
    hipError_t e = hipGetDevice(&device);
    const uint64_t bit = device >= 0 && device < 64 ? 1ull << device : 0;
    if (e == hipSuccess && (done.load(std::memory_order_relaxed) & bit))
        return DASS_OK;
    if (e == hipSuccess)
        e = hipFuncSetAttribute(reinterpret_cast<const void *>(KERNEL), hipFuncAttributeMaxDynamicSharedMemorySize, BYTES);
    if (e != hipSuccess)
        return fail(DASS_ERR_HIP, "%s: cannot reserve %d bytes of LDS: %s", fn, BYTES, hipGetErrorString(e));
    done.fetch_or(bit, std::memory_order_relaxed);
    return DASS_OK;
}

// The order of a product's tiles (for dW of one expert's); blocks: 0 if they are too many for a launch.
template <typename T_, Product PRODUCT, int BR, int BC>
static TileOrder order_tiles(const Operands<T_> &a, const Epilogue<T_> &ep)
{
    const int64_t tiles_r = PRODUCT == kWeightGrad ? (a.out_rows + BR - 1) / BR : tile_numbers(a.seg, BR);
    const int64_t tiles_c = (ep.cols + BC - 1) / BC;
    const int64_t q_bytes = (PRODUCT == kWeightGrad ? a.seg.rows : a.depth) * ep.cols * (int64_t)sizeof(T_);
    TileOrder order = make_tile_order(tiles_r, tiles_c, q_bytes <= (256LL << 20), BR < BC ? 8 : kPatchT);
    if (PRODUCT != kWeightGrad && a.seg.offsets) {   // the kernel orders the tiles that there are
        const int64_t n = (tiles_r * tiles_c + kXcds - 1) / kXcds * kXcds;
        order.blocks = n <= 0x7fffffffLL ? (unsigned)n : 0;
        order.tiles_n = (unsigned)tiles_c;
    }
    return order;
}

template <typename T_, Product PRODUCT, int RB, int CB, bool SHORT = false>
static dass_status launch_tiles(const char *fn, const Operands<T_> &a, const Epilogue<T_> &ep, const Split &split, hipStream_t stream)
{
    const TileOrder order = order_tiles<T_, PRODUCT, 32 * RB, 32 * CB>(a, ep);
    const unsigned experts = PRODUCT == kWeightGrad ? a.seg.n : 1;
    if (order.blocks == 0 || (int64_t)order.blocks * 256 > 0xffffffffLL / experts / split.n)
        return fail(DASS_ERR_SHAPE, "%s: too many tiles for one launch; split the rows", fn);
    dass_status s = reserve_lds<product_tile_kernel<T_, PRODUCT, RB, CB, SHORT>, lds_bytes<SHORT>()>(fn);
    if (s != DASS_OK)
        return s;
    hipLaunchKernelGGL((product_tile_kernel<T_, PRODUCT, RB, CB, SHORT>), dim3(order.blocks, experts, split.n), dim3(256),
                       lds_bytes<SHORT>(), stream, a, ep, order, split);
    s = check_launch("product kernel");
    if (s != DASS_OK || split.n == 1)
        return s;
    constexpr int N = Chunk<T_>::N;
    const int64_t strips = (ep.cols + 32 * N - 1) / (32 * N);
    const int64_t rows = PRODUCT == kWeightGrad ? (a.out_rows * a.seg.n + 7) / 8 : tile_numbers(a.seg, 8);
    if (rows > 0xffffffffLL / 256 / strips)
        return fail(DASS_ERR_SHAPE, "%s: too many rows for one launch; split the rows", fn);
    hipLaunchKernelGGL((join_kernel<T_, PRODUCT>), dim3((unsigned)(rows * strips)), dim3(256), 0, stream, a, ep, split, (uint32_t)strips);
    return check_launch("join kernel");
}

template <typename T_, Product PRODUCT>
static dass_status launch_plan(const char *fn, const Plan &plan, const Operands<T_> &a, const Epilogue<T_> &ep, const Split &split,
                               hipStream_t stream)
{
    if constexpr (sizeof(T_) == 2) {
        if (plan.tile == 0)
            return launch_tiles<T_, PRODUCT, 8, 8>(fn, a, ep, split, stream);
        if (plan.tile == 1)
            return launch_tiles<T_, PRODUCT, 4, 8>(fn, a, ep, split, stream);
        if (plan.tile == 3)
            return launch_tiles<T_, PRODUCT, 4, 4, true>(fn, a, ep, split, stream);
    }
    return launch_tiles<T_, PRODUCT, 4, 4>(fn, a, ep, split, stream);
}

}  // namespace dass
