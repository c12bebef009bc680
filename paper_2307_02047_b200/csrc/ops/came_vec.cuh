// Wide loads and stores of fp32 and bf16 for the operators beside the step: N consecutive elements
// in one or two accesses.
#pragma once
#include "came_ops.cuh"

namespace came_ops {

// N elements as they are stored: accesses of up to 32 bytes.  (Volatile, so that the loads of a batch
// stay together in front of what uses them.)
template <typename T, int N>
struct Vec {
    static constexpr int B = N * static_cast<int>(sizeof(T));
    static constexpr int W = B < 4 ? 1 : B / 4;
    uint32_t w[W];

    __device__ __forceinline__ void load(const T* p)
    {
        if constexpr (B >= 32) {
#pragma unroll
            for (int j = 0; j < W; j += 8)
                asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                             : "=r"(w[j]), "=r"(w[j + 1]), "=r"(w[j + 2]), "=r"(w[j + 3]),
                               "=r"(w[j + 4]), "=r"(w[j + 5]), "=r"(w[j + 6]), "=r"(w[j + 7])
                             : "l"(reinterpret_cast<const char*>(p) + 4 * j));
        } else if constexpr (B == 16) {
            asm volatile("ld.global.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(p));
        } else if constexpr (B == 8) {
            asm volatile("ld.global.v2.b32 {%0,%1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(p));
        } else if constexpr (B == 4) {
            asm volatile("ld.global.b32 %0, [%1];" : "=r"(w[0]) : "l"(p));
        } else if constexpr (B == 2) {
            uint16_t h;
            asm volatile("ld.global.b16 %0, [%1];" : "=h"(h) : "l"(p));
            w[0] = h;
        } else {
            uint32_t h;
            asm volatile("ld.global.u8 %0, [%1];" : "=r"(h) : "l"(p));
            w[0] = h;
        }
    }

    __device__ __forceinline__ void store(T* p) const
    {
        if constexpr (B >= 32) {
#pragma unroll
            for (int j = 0; j < W; j += 8)
                asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                             :: "l"(reinterpret_cast<char*>(p) + 4 * j), "r"(w[j]), "r"(w[j + 1]), "r"(w[j + 2]), "r"(w[j + 3]),
                                "r"(w[j + 4]), "r"(w[j + 5]), "r"(w[j + 6]), "r"(w[j + 7]) : "memory");
        } else if constexpr (B == 16) {
            *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
        } else if constexpr (B == 8) {
            *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
        } else if constexpr (B == 4) {
            *reinterpret_cast<uint32_t*>(p) = w[0];
        } else if constexpr (B == 2) {
            *reinterpret_cast<uint16_t*>(p) = static_cast<uint16_t>(w[0]);
        } else {
            *reinterpret_cast<uint8_t*>(p) = static_cast<uint8_t>(w[0]);
        }
    }

    // element k of fp32 or bf16 as fp32
    __device__ __forceinline__ float value(int k) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[k]);
        else return __uint_as_float(k & 1 ? w[k >> 1] & 0xffff0000u : w[k >> 1] << 16);
    }

    __device__ __forceinline__ void set(const float (&x)[N])
    {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int k = 0; k < N; ++k) w[k] = __float_as_uint(x[k]);
        } else if constexpr (N == 1) {
            w[0] = __bfloat16_as_ushort(__float2bfloat16_rn(x[0]));
        } else {
#pragma unroll
            for (int k = 0; k < N; k += 2)
                asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[k >> 1]) : "f"(x[k + 1]), "f"(x[k]));
        }
    }
};

}  // namespace came_ops
