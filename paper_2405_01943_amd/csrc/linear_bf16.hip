// dass_linear and dass_linear_backward in bf16 on the matrix cores.
//
// A workgroup owns a tile of 32 RB rows x 32 CB columns of the output, its four wavefronts (2 x 2) a quarter each:
// RB x CB blocks of v_mfma_f32_16x16x32_bf16, for 8 x 8 all 256 accumulation registers of a lane.  Slabs of 64 k go
// from global memory straight into LDS (16 bytes a lane, no registers in between).  Output columns are the
// instruction's M index and rows its N index, so a lane holds four neighbouring columns of a row.
//
// An operand comes in one of two forms, and LDS holds it in the form that it has in memory:
//   by rows   a wave-load is 8 rows x 128 bytes; a lane's eight k of a row are one 16-byte read.  16-byte chunk c of
//             row r lies in slot c ^ (r / 2 mod 8): 16 rows of one chunk meet 16 places of the banks.
//   k by k    a wave-load is 2 (4) lines of k of 256 (128) rows.  ds_read_b64_tr_b16 reads a 4 x 16 block of k x rows for 16
//             lanes and gives each lane the four k of one row; two of them are a lane's eight k.  A block's 32 bytes
//             of line k lie in place piece ^ f(k), f(k) = (k mod 4) + 4 (k / 8 mod 2), so that the eight lines
//             that 32 lanes read at a time meet all 64 banks once.
// So no operand is transposed in memory: the three products (linear.h) differ in their operands' forms alone.
//
// LDS is two rings, NP parts of P and NQ of Q, as many as 160 KB hold.  The places of slab s are free after the one
// barrier of the slab, which stands where every wavefront has read its last fragments of it, in the middle of its second
// K step; the loads of Q's slab s + NQ and P's slab s + NP are spread over the matrix instructions from there to the
// next barrier.  The wait before a barrier counts the loads that may still be on their way, so their order is
// pinned; only slabs that exist are requested, and the last slabs have bodies of their own with fewer to wait for.
//
// Reads outside a matrix: each operand is a raw buffer that starts at the tile's first row and ends with its last
// valid element; what lies beyond reads as 0.  Lane offsets are 32-bit registers, the scalar offset is at most a row
// (by rows) or none (k by k, whose buffer moves with the slab), so the length less the scalar offset is never negative.  By rows, chunks of
// the last slab that lie beyond k are given an offset outside the buffer.
#include "linear.h"
#include "tile_order.h"

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

constexpr int kLds = 160 * 1024, kSlab = 64;
constexpr int kOutside = 0x7fffffff;

// A raw buffer: 48 bits of address, no stride, its length in bytes.
__device__ __forceinline__ u32x4 raw_buffer(const void *p, int bytes)
{
    const uint64_t a = reinterpret_cast<uint64_t>(p);
    return u32x4{(uint32_t)a, (uint32_t)(a >> 32) & 0xffffu, (uint32_t)bytes, 0x00020000u};
}

// One wave-load of 16 bytes a lane from a buffer straight into LDS: the builtin where both operands are by rows, and
// by hand where one is not.  Beside the builtin the compiler waits for every such load before each transposing LDS read (it takes the
// read to depend on them), which empties the pipeline once a load: dX and dW of 6000 rows of 4096 x 11008 1590 us, by
// hand 548 and 444; of products without such reads the builtin is 4 % ahead.  (Not a template: with arguments that depend on
// one, the host pass rejects the builtin.)  The block by hand writes no register but m0; the waits for it are
// those before the barriers.  Its s_nop covers the wait states between a scalar register's last write and its use as an address.
__device__ __forceinline__ void load_to_lds(const u32x4 &buffer, char *dst, uint32_t lane_off, int off)
{
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(
        reinterpret_cast<void *>((uint64_t)buffer[1] << 32 | buffer[0]), 0, (int)buffer[2], (int)buffer[3]);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_ptr_t)dst, 16, lane_off, off, 0, 0);
}
__device__ __forceinline__ void load_to_lds_by_hand(const u32x4 &buffer, char *dst, uint32_t lane_off, int off)
{
    const uint32_t at = (uint32_t)(uintptr_t)(lds_ptr_t)dst;
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(at), "v"(lane_off), "s"(buffer),
                 "s"(off) : "m0", "memory");
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
template <bool BY_ROWS, int B, bool BY_HAND>
struct Part;

template <int B, bool BY_HAND>
struct Part<true, B, BY_HAND> {
    static constexpr int LOADS = B, READS = B, UNIT = 32 * B * 128;
    struct Frags {
        bf16x8 v[B];
        __device__ __forceinline__ bf16x8 get(int b) const { return v[b]; }
    };
    u32x4 buffer;
    uint32_t off[LOADS];
    int chunk[2], k_bytes, frag;

    __device__ __forceinline__ void init(const uint16_t *m, int64_t ld, int64_t row0, int64_t rows, int64_t k0, int64_t k, int wave, int lane,
                                         int part)
    {
        const int64_t n = rows - row0 < 32 * B ? rows - row0 : 32 * B;
        buffer = raw_buffer(m + row0 * ld + k0, (int)(((n - 1) * ld + k) * 2));
        k_bytes = (int)(k * 2);
        const int sub = lane >> 3;
        chunk[0] = ((lane & 7) ^ (sub >> 1)) * 16;
        chunk[1] = chunk[0] ^ 64;                          // rows 8 further on: r / 2 has changed by 4
#pragma unroll
        for (int q = 0; q < LOADS; ++q)
            off[q] = (uint32_t)(((wave * LOADS + q) * 8 + sub) * ld * 2) + chunk[q & 1];
        const int r = part * 16 * B + (lane & 15);
        frag = r * 128 + (((lane >> 4) ^ (r >> 1)) & 7) * 16;
    }
    __device__ __forceinline__ void begin_slab(int) {}
    // LAST: the slab may be the last one, whose chunks may lie beyond k
    template <bool LAST>
    __device__ __forceinline__ void load(char *unit, int wave, int slab, int q) const
    {
        const int at = slab * (kSlab * 2);
        const uint32_t lane_off = !LAST || at + chunk[q & 1] < k_bytes ? off[q] : (uint32_t)kOutside;
        if constexpr (BY_HAND)
            load_to_lds_by_hand(buffer, unit + (wave * LOADS + q) * 1024, lane_off, at);
        else
            load_to_lds(buffer, unit + (wave * LOADS + q) * 1024, lane_off, at);
    }
    // read x of the fragments of K step kk
    __device__ __forceinline__ void read(const char *unit, int kk, int x, Frags &f) const
    {
        f.v[x] = *reinterpret_cast<const bf16x8 *>(unit + (frag ^ (kk * 64)) + x * 2048);
    }
};

template <int B, bool BY_HAND>
struct Part<false, B, BY_HAND> {
    static constexpr int LOADS = B, READS = 2 * B, UNIT = 32 * B * 128;
    struct Frags {
        s16x4 v[2 * B];
        __device__ __forceinline__ bf16x8 get(int b) const
        {
            return __builtin_bit_cast(bf16x8, __builtin_shufflevector(v[2 * b], v[2 * b + 1], 0, 1, 2, 3, 4, 5, 6, 7));
        }
    };
    static constexpr int LINE = 32 * B * 2, SLOTS = LINE / 16, LINES = 1024 / LINE;   // bytes, chunks; lines of a wave-load
    const uint16_t *m;
    int64_t ld, depth, width;
    u32x4 buffer;
    uint32_t off[LOADS];
    int frag;

    static __device__ __forceinline__ int f_of(int k) { return (k & 3) | (k >> 1 & 4); }
    __device__ __forceinline__ void init(const uint16_t *base, int64_t ld_, int64_t row0, int64_t rows, int64_t k0, int64_t k, int wave, int lane,
                                         int part)
    {
        m = base + k0 * ld_ + row0;
        ld = ld_;
        depth = k;
        width = rows - row0 < 32 * B ? rows - row0 : 32 * B;
#pragma unroll
        for (int q = 0; q < LOADS; ++q) {
            const int line = wave * 16 + q * LINES + lane / SLOTS;
            off[q] = (uint32_t)(line * ld * 2) + ((lane % SLOTS) ^ (f_of(line) << 1)) * 16;
        }
        const int g = lane >> 4, i = lane & 15, line = 8 * g + (i >> 2);
        frag = line * LINE + (((part * B) ^ f_of(line)) * 32) + (i & 3) * 8;
    }
    __device__ __forceinline__ void begin_slab(int slab)
    {
        const int64_t left = depth - (int64_t)slab * kSlab, lines = left < kSlab ? left : kSlab;
        buffer = raw_buffer(m + (int64_t)slab * kSlab * ld, (int)(((lines - 1) * ld + width) * 2));
    }
    template <bool LAST>
    __device__ __forceinline__ void load(char *unit, int wave, int, int q) const
    {
        static_assert(BY_HAND, "it is read by transposing reads");
        load_to_lds_by_hand(buffer, unit + (wave * LOADS + q) * 1024, off[q], 0);
    }
    __device__ __forceinline__ void read(const char *unit, int kk, int x, Frags &f) const
    {
        f.v[x] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (lds_s16x4_t)(unit + (frag ^ (x / 2 * 32)) + (x % 2 * 4 + kk * 32) * LINE));
    }
};

// Eight neighbouring columns of one row, with the chunks of mul and residual at hand; `col` is a multiple of 8 and inside.
__device__ __forceinline__ void finish8(const Epilogue<uint16_t> &ep, int64_t row, int64_t col, const float (&bias)[8], const u32x4 &mul,
                                        const u32x4 &residual, float (&v)[8])
{
    typedef Chunk<uint16_t> C;
    float w[8];
    if (ep.bias) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] += bias[i];
    }
    if (ep.pre)
        *reinterpret_cast<u32x4 *>(ep.pre + row * ep.ldp + col) = C::narrow(v);
    if (ep.act != DASS_ACT_NONE) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] = act_value<true>(v[i], ep.act);
    }
    if (ep.mul) {
        C::widen(mul, w);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] *= w[i];
    }
    if (ep.residual) {
        C::widen(residual, w);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] += w[i];
    }
    *reinterpret_cast<u32x4 *>(ep.out + row * ep.ldo + col) = C::narrow(v);
}

template <Product PRODUCT, int RB, int CB>
__global__ __launch_bounds__(256) void product_bf16_kernel(const Operands<uint16_t> a, const Epilogue<uint16_t> ep0, const TileOrder order)
{
    typedef Part<PRODUCT != kWeightGrad, RB, PRODUCT != kForward> PartP;
    typedef Part<PRODUCT == kForward, CB, PRODUCT != kForward> PartQ;
    constexpr int BR = 32 * RB, BC = 32 * CB;
    constexpr int NP = RB == 8 ? 3 : CB == 8 ? 4 : 5, NQ = RB == 8 ? 2 : CB == 8 ? 3 : 5, LEAD = NP - NQ;
    static_assert(NP * PartP::UNIT + NQ * PartQ::UNIT <= kLds && (LEAD == 0 || LEAD == 1), "the rings fit");
    constexpr int PL = PartP::LOADS, QL = PartQ::LOADS, NL = PL + QL;
    constexpr int N = RB * CB;   // matrix instructions of a K step
    extern __shared__ __attribute__((aligned(1024))) char lds[];   // kLds bytes

    uint32_t tile_r, tile_c;   // tile_order.h
    if (!tile_of_block(order, blockIdx.x, tile_r, tile_c))
        return;
    int expert;
    int64_t r0, r_end, k0 = 0, depth = a.depth;
    if constexpr (PRODUCT == kWeightGrad) {
        expert = blockIdx.y;
        const Span k = segment(a.seg, expert);
        k0 = k.lo;
        depth = k.hi - k.lo;
        r0 = (int64_t)tile_r * BR;
        r_end = a.out_rows;
    } else {
        Span r;
        if (!rows_of_tile(a.seg, tile_r, BR, expert, r))
            return;
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

    const int S = (int)((depth + kSlab - 1) / kSlab);
    if (PRODUCT != kWeightGrad || S > 0) {
    PartP P;
    PartQ Q;
    P.init(a.P, a.ldp, r0, r_end, k0, depth, wave, lane, wr);
    Q.init(PRODUCT == kWeightGrad ? a.Q : a.Q + (int64_t)expert * a.q_stride, a.ldq, c0, ep0.cols, k0, depth, wave, lane, wc);
    char *const p_ring = lds, *const q_ring = lds + NP * PartP::UNIT;

    // ---- the loads.  Iteration t (after the barrier of slab t) requests Q's slab t + NQ, then P's slab t + NP.
    auto load_p = [&](int unit, int slab, int q, auto last) __attribute__((always_inline)) {
        P.template load<decltype(last)::value>(p_ring + unit * PartP::UNIT, wave, slab, q);
        __builtin_amdgcn_sched_barrier(0);
    };
    auto load_q = [&](int unit, int slab, int q, auto last) __attribute__((always_inline)) {
        Q.template load<decltype(last)::value>(q_ring + unit * PartQ::UNIT, wave, slab, q);
        __builtin_amdgcn_sched_barrier(0);
    };
    constexpr int AT_ONCE = (NL + 3) / 4;   // of an iteration's loads, those right after its barrier
    static_assert(AT_ONCE <= QL, "they are Q's");
    auto all_p = [&](int slab) {
        if (slab < S) {
            P.begin_slab(slab);
#pragma unroll
            for (int q = 0; q < PL; ++q)
                load_p(slab % NP, slab, q, std::true_type{});
        }
    };
    if (LEAD == 1)
        all_p(0);
#pragma unroll
    for (int t = -NQ; t < -1; ++t) {
        if (t + NQ < S) {
            Q.begin_slab(t + NQ);
#pragma unroll
            for (int q = 0; q < QL; ++q)
                load_q(t + NQ, t + NQ, q, std::true_type{});
        }
        all_p(t + NP);
    }
    if (NQ - 1 < S) {
        Q.begin_slab(NQ - 1);
#pragma unroll
        for (int q = 0; q < AT_ONCE; ++q)
            load_q(NQ - 1, NQ - 1, q, std::true_type{});
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
    // slab 0 has landed: all but the first part of P and of Q may be on their way
    auto begin = [&](auto slabs_tag) __attribute__((always_inline)) {
        constexpr int HAVE = decltype(slabs_tag)::value;   // slabs, at most NP
        constexpr int P_OUT = (HAVE < NP - 1 ? HAVE : NP - 1) - 1, Q_OUT = (HAVE < NQ - 1 ? HAVE : NQ - 1) - 1;
        constexpr int OUT = P_OUT * PL + (Q_OUT > 0 ? Q_OUT : 0) * QL + (HAVE >= NQ ? AT_ONCE : 0);
        wait_loads<OUT>();
    };
    static_assert(NQ >= 2, "the first part of Q is requested whole");
    if (S >= NP)
        begin(std::integral_constant<int, NP>{});
    else if (NP > 4 && S == 4)
        begin(std::integral_constant<int, (NP > 4 ? 4 : 1)>{});
    else if (NP > 3 && S == 3)
        begin(std::integral_constant<int, (NP > 3 ? 3 : 1)>{});
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
        acc[I][J] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.q.get(I), f.p.get(J), acc[I][J], 0, 0, 0);
    };

    Frags f0, f1;
    for_each<0, READS>([&](auto x) __attribute__((always_inline)) { read_one(f0, 0, 0, 0, x); });
    int pu = 0, qu = 0, pu_old = NP - 1, qu_old = NQ - 1;   // ring places of slab s and of slab s - 1
    // LEFT: how many slabs follow; STEADY stands for that and more, and never requests the last slab.
    constexpr int STEADY = LEAD == 0 ? NP + 1 : NP;
    auto slab_body = [&](int s, auto left_tag) __attribute__((always_inline)) {
        constexpr int LEFT = decltype(left_tag)::value;
        constexpr auto LAST = std::integral_constant<bool, (LEFT < STEADY)>{};
        constexpr bool OLD_Q = LEFT >= NQ - 1, OLD_P = LEFT >= NP - 1, NEW_Q = LEFT >= NQ;   // what iterations s - 1 and s request
        const int pu1 = pu + 1 == NP ? 0 : pu + 1, qu1 = qu + 1 == NQ ? 0 : qu + 1;
        // what goes with instruction POS of the 2 N since a barrier: its share of the loads, in their order
        auto old_loads = [&](auto pos) __attribute__((always_inline)) {
            constexpr int POS = decltype(pos)::value;
            for_each<(POS * NL + 2 * N - 1) / (2 * N), ((POS + 1) * NL + 2 * N - 1) / (2 * N)>([&](auto x) __attribute__((always_inline)) {
                constexpr int X = decltype(x)::value;
                if constexpr (X < QL) {
                    if constexpr (OLD_Q)
                        load_q(qu_old, s - 1 + NQ, X, LAST);
                } else if constexpr (OLD_P) {
                    load_p(pu_old, s - 1 + NP, X - QL, LAST);
                }
            });
        };
        if (OLD_Q)
            Q.begin_slab(s - 1 + NQ);
        if (OLD_P)
            P.begin_slab(s - 1 + NP);
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
            constexpr int Q_OUT = (LEFT < NQ - 1 ? LEFT : NQ - 1) - 1, P_OUT = (LEFT < NP - 1 ? LEFT : NP - 1) - 1;
            wait_loads<Q_OUT * QL + P_OUT * PL>();
            block_barrier();
            if (NEW_Q)
                Q.begin_slab(s + NQ);
        }
        for_each<0, N / 2>([&](auto n) __attribute__((always_inline)) {   // K step 1, second half
            constexpr int I = decltype(n)::value;
            if constexpr (NEW_Q)
                for_each<(I * NL + 2 * N - 1) / (2 * N), ((I + 1) * NL + 2 * N - 1) / (2 * N)>(
                    [&](auto x) __attribute__((always_inline)) { load_q(qu, s + NQ, x, LAST); });
            if constexpr (LEFT > 0)
                for_each<(I * READS + N / 2 - 1) / (N / 2), ((I + 1) * READS + N / 2 - 1) / (N / 2)>(
                    [&](auto x) __attribute__((always_inline)) { read_one(f0, pu1, qu1, 0, x); });
            multiply(f1, std::integral_constant<int, N / 2 + I>{});
            __builtin_amdgcn_sched_barrier(0);
        });
        pu_old = pu;
        qu_old = qu;
        pu = pu1;
        qu = qu1;
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
    static_assert(NP <= 5, "every number of slabs left has its body");
    }

    // ---- epilogue.  A wavefront passes strips of 16 rows through LDS of its own, as f32, so that a lane finishes eight
    // neighbouring columns and rows are read and written in whole 128-byte lines.  mul and residual are requested
    // AHEAD strips before they are needed, the first while the last sums are still being finished.
    Epilogue<uint16_t> ep = ep0;
    if constexpr (PRODUCT == kWeightGrad)
        ep.out += (int64_t)expert * a.out_stride;
    constexpr int SROW = 16 * CB * 4 + 16, LANES = 2 * CB, ROWS = 64 / LANES;   // lanes of a row; rows of a read
    constexpr int READS_16 = 16 / ROWS, AHEAD = 3;
    char *const strips = lds + wave * (kLds / 4);
    const int fr = lane & 15, g = lane >> 4;
    const int64_t row0 = r0 + wr * 16 * RB + lane / LANES, col = c0 + wc * 16 * CB + lane % LANES * 8;
    float bias[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    u32x4 mul[AHEAD + 1][READS_16], residual[AHEAD + 1][READS_16];
    auto request = [&](auto j_tag) __attribute__((always_inline)) {
        constexpr int J = decltype(j_tag)::value;
        if constexpr (J < RB && PRODUCT == kForward) {
#pragma unroll
            for (int t = 0; t < READS_16; ++t) {
                const int64_t r = row0 + J * 16 + t * ROWS;
                if (r < r_end && col < ep.cols) {
                    if (ep.mul)
                        mul[J % (AHEAD + 1)][t] = *reinterpret_cast<const u32x4 *>(ep.mul + r * ep.ldm + col);
                    if (ep.residual)
                        residual[J % (AHEAD + 1)][t] = *reinterpret_cast<const u32x4 *>(ep.residual + r * ep.ldr + col);
                }
            }
        }
    };
    for_each<0, AHEAD>(request);
    if (PRODUCT == kForward && ep.bias && col < ep.cols)
        Chunk<uint16_t>::widen(*reinterpret_cast<const u32x4 *>(ep.bias + (int64_t)expert * ep.cols + col), bias);
    block_barrier();   // the rings are about to be used again
    for_each<0, RB>([&](auto j_tag) __attribute__((always_inline)) {
        constexpr int J = decltype(j_tag)::value;
        char *const strip = strips + (J & 1) * 16 * SROW;
        request(std::integral_constant<int, J + AHEAD>{});
#pragma unroll
        for (int i = 0; i < CB; ++i)
            *reinterpret_cast<f32x4 *>(strip + fr * SROW + (i * 16 + 4 * g) * 4) = acc[i][J];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int t = 0; t < READS_16; ++t) {
            const char *at = strip + (t * ROWS + lane / LANES) * SROW + lane % LANES * 32;
            const f32x4 lo = *reinterpret_cast<const f32x4 *>(at), hi = *reinterpret_cast<const f32x4 *>(at + 16);
            float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
            const int64_t r = row0 + J * 16 + t * ROWS;
            if (r < r_end && col < ep.cols) {
                if constexpr (PRODUCT == kForward)
                    finish8(ep, r, col, bias, mul[J % (AHEAD + 1)][t], residual[J % (AHEAD + 1)][t], v);
                else
                    *reinterpret_cast<u32x4 *>(ep.out + r * ep.ldo + col) = Chunk<uint16_t>::narrow(v);
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    });
}

// ------------------------------------------------------------------ host side --
template <Product PRODUCT, int RB, int CB>
static dass_status launch_tile(const char *fn, const Operands<uint16_t> &a, const Epilogue<uint16_t> &ep, bool q_cached, hipStream_t stream)
{
    constexpr int BR = 32 * RB, BC = 32 * CB;
    const int64_t tiles_r = PRODUCT == kWeightGrad ? (a.out_rows + BR - 1) / BR : tile_numbers(a.seg, BR);
    const int64_t tiles_c = (ep.cols + BC - 1) / BC;
    const TileOrder order = make_tile_order(tiles_r, tiles_c, q_cached, BR < BC ? 8 : kPatchT);
    const unsigned experts = PRODUCT == kWeightGrad ? a.seg.n : 1;
    if (order.blocks == 0 || (int64_t)order.blocks * 256 * experts > 0xffffffffLL)
        return fail(DASS_ERR_SHAPE, "%s: too many tiles for one launch; split the rows", fn);
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(product_bf16_kernel<PRODUCT, RB, CB>),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
    if (e != hipSuccess)
        return fail(DASS_ERR_HIP, "%s: cannot reserve %d bytes of LDS: %s", fn, kLds, hipGetErrorString(e));
    hipLaunchKernelGGL((product_bf16_kernel<PRODUCT, RB, CB>), dim3(order.blocks, experts), dim3(256), kLds, stream, a, ep, order);
    return check_launch("bf16 product kernel");
}

template <Product PRODUCT>
static dass_status launch_any(const char *fn, const Operands<uint16_t> &a, const Epilogue<uint16_t> &ep, hipStream_t stream)
{
    // 32-bit byte offsets inside a tile: 256 rows (by rows), 64 lines of k (k by k)
    if (256 * a.ldp * 2 >= 0x7fffffffLL || 256 * a.ldq * 2 >= 0x7fffffffLL)
        return fail(DASS_ERR_SHAPE, "%s: rows too long for the tile addressing", fn);
    // each expert's tiles count as if its rows were an even share
    const int64_t groups = PRODUCT == kWeightGrad ? 1 : a.seg.n;
    const int64_t rows = PRODUCT == kWeightGrad ? a.out_rows : (a.seg.rows + groups - 1) / groups;
    const TileShape shape = dense_tile_shape(rows, ep.cols * groups, false);
    const int64_t q_bytes = (PRODUCT == kWeightGrad ? a.seg.rows : a.depth) * ep.cols * 2;
    const bool cached = q_bytes <= (256LL << 20);
    if (shape.which == 0)
        return launch_tile<PRODUCT, 8, 8>(fn, a, ep, cached, stream);
    if (shape.which == 1)
        return launch_tile<PRODUCT, 4, 8>(fn, a, ep, cached, stream);
    return launch_tile<PRODUCT, 4, 4>(fn, a, ep, cached, stream);
}

dass_status launch_product_bf16(const char *fn, Product product, const Operands<uint16_t> &a, const Epilogue<uint16_t> &ep,
                                hipStream_t stream)
{
    if (product == kForward)
        return launch_any<kForward>(fn, a, ep, stream);
    if (product == kInputGrad)
        return launch_any<kInputGrad>(fn, a, ep, stream);
    return launch_any<kWeightGrad>(fn, a, ep, stream);
}

}  // namespace dass
