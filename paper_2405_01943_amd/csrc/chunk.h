// One 16-byte chunk of a row (8 bf16 or 4 f32) as f32 values and back.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace dass {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

template <typename T_>
struct Chunk;
template <>
struct Chunk<uint16_t> {
    static constexpr int N = 8;
    static __device__ __forceinline__ void widen(const u32x4 &c, float (&v)[8])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __builtin_bit_cast(float, c[i] << 16);
            v[2 * i + 1] = __builtin_bit_cast(float, c[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ u32x4 narrow(const float (&v)[8])
    {
        typedef __attribute__((ext_vector_type(2))) float f2;
        typedef __attribute__((ext_vector_type(2))) __bf16 b2;
        u32x4 c;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            c[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{v[2 * i], v[2 * i + 1]}, b2));
        return c;
    }
};
template <>
struct Chunk<float> {
    typedef __attribute__((ext_vector_type(4))) float f32x4;
    static constexpr int N = 4;
    static __device__ __forceinline__ void widen(const u32x4 &c, float (&v)[4])
    {
        const f32x4 f = __builtin_bit_cast(f32x4, c);   // whole: the cast of one element of a vector takes its first
#pragma unroll
        for (int i = 0; i < 4; ++i)
            v[i] = f[i];
    }
    static __device__ __forceinline__ u32x4 narrow(const float (&v)[4])
    {
        return __builtin_bit_cast(u32x4, f32x4{v[0], v[1], v[2], v[3]});
    }
};

}  // namespace dass
