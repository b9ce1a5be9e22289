// rows.hpp -- eight neighbouring values of a row of bf16 or fp32.
#pragma once

#include "fp8.hpp"

namespace echo {

// Eight values as they lie in memory
template <bool F32>
struct Eight {
    fp8::u32x4 a[F32 ? 2 : 1];
    __device__ __forceinline__ void load(const void *x, int64_t e) {
        const fp8::u32x4 *q = (const fp8::u32x4 *)((const uint8_t *)x + e * (F32 ? 4 : 2));
#pragma unroll
        for (int i = 0; i < (F32 ? 2 : 1); ++i) a[i] = q[i];
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < (F32 ? 2 : 1); ++i) a[i] = (fp8::u32x4){0u, 0u, 0u, 0u};
    }
    __device__ __forceinline__ float get(int i) const {
        if constexpr (F32) return __uint_as_float(a[i / 4][i % 4]);
        return __uint_as_float(i & 1 ? a[0][i / 2] & 0xFFFF0000u : a[0][i / 2] << 16);
    }
    // bits of the largest magnitude, as fp32: above infinity's with a NaN
    __device__ __forceinline__ uint32_t top() const {
        uint32_t m = 0;
        if constexpr (F32) {
#pragma unroll
            for (int i = 0; i < 8; ++i) m = max(m, a[i / 4][i % 4] & 0x7FFFFFFFu);
            return m;
        }
        typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
        u16x2 two = {0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i)
            two = __builtin_elementwise_max(two, __builtin_bit_cast(u16x2, a[0][i] & 0x7FFF7FFFu));
        return (uint32_t)max(two[0], two[1]) << 16;
    }
};

}  // namespace echo
