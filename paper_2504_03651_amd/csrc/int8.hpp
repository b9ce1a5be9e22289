// int8.hpp -- device pieces shared by the kernels of products in 8-bit integers.
#pragma once

#include "fp8_tiled.hpp"
#include "int8_cut.hpp"

namespace echo {
namespace int8 {

using fp8::any_f32x4;
using fp8::any_u32x2;
using fp8::any_u32x4;
using fp8::bf2f;
using fp8::cdiv;
using fp8::f2bf;
using fp8::f2bf2;
using fp8::f32x4;
using fp8::kZeros;
using fp8::landed_but;
using fp8::launch_lds;
using fp8::lds_void;
using fp8::u32x2;
using fp8::u32x4;
using fp8::wave_lds;

typedef int i32x4 __attribute__((ext_vector_type(4)));

// What a product's kernel reads and writes.
struct Product {
    const uint8_t *x, *w;    // codes [T][K], [N][K]
    const float *xs, *ws;    // [T], [N]
    const float *bias;       // [N] or null
    const void *residual;    // of y's type and stride, or null
    void *y;
    int64_t y_stride;
    int T, N, K, KB;         // KB: steps of K
    int32_t *part;           // [ranges][T][part_pitch], for products over ranges of K
    int part_pitch;
};

// c[16 rows of a][16 rows of b] += of 64 contraction steps.  Each lane holds 16 codes
// of row lane % 16 of each operand; which of the 64 steps they are is free as long as
// both operands agree (here bytes 16 (lane / 16) ..).  The lane gets column lane % 16
// (a row of b) and rows 4 (lane / 16) .. + 3 (of a).
__device__ __forceinline__ i32x4 mfma64(u32x4 a, u32x4 b, i32x4 c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
}

// A scale as a fraction in [0.5, 1) and a power of two, so that the scaled sum leaves
// fp32's range only where it has to, whatever the two scales' product does.  The sum's
// conversion and the two products by fractions round, three halves of 2^-23 at most.
struct Scale {
    float m;
    int e;
};
__device__ __forceinline__ Scale split(float s) {
    return {__builtin_amdgcn_frexp_mantf(s), __builtin_amdgcn_frexp_expf(s)};
}
__device__ __forceinline__ float scaled(int sum, Scale x, Scale w) {
    return __builtin_amdgcn_ldexpf((float)sum * x.m * w.m, x.e + w.e);
}

// The residual of E columns from n, at element `at`
template <bool F32, int E>
struct Rest {
    static constexpr int WORDS = F32 ? E : E / 2;
    uint32_t b[WORDS];
    __device__ __forceinline__ void load(const Product &p, int64_t at, int n) {
        if (n + E <= p.N) {
            if constexpr (WORDS == 4) {
                const u32x4 r = F32 ? __builtin_bit_cast(u32x4, *(const any_f32x4 *)((const float *)p.residual + at))
                                    : (u32x4)*(const any_u32x4 *)((const uint16_t *)p.residual + at);
#pragma unroll
                for (int i = 0; i < 4; ++i) b[i] = r[i];
            } else {
                static_assert(!F32 && WORDS == 2);
                const u32x2 r = *(const any_u32x2 *)((const uint16_t *)p.residual + at);
                b[0] = r[0], b[1] = r[1];
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < WORDS; ++i) {
            if constexpr (F32) {
                b[i] = n + i < p.N ? __float_as_uint(((const float *)p.residual)[at + i]) : 0u;
            } else {
                const uint16_t *r = (const uint16_t *)p.residual + at + 2 * i;
                b[i] = (n + 2 * i < p.N ? r[0] : 0u) | (n + 2 * i + 1 < p.N ? (uint32_t)r[1] << 16 : 0u);
            }
        }
    }
    __device__ __forceinline__ void add(float (&v)[E]) const {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) {
            if constexpr (F32) v[i] += __uint_as_float(b[i]);
            else v[2 * i] += bf2f(b[i] & 0xFFFFu), v[2 * i + 1] += bf2f(b[i] >> 16);
        }
    }
};

// y of E columns from n of row t; PAST: past the caches
template <bool F32, int E, bool PAST = false>
__device__ __forceinline__ void put(const Product &p, int64_t t, int n, const float (&v)[E]) {
    static_assert(E == 4 || (E == 8 && !F32));
    const int64_t at = t * p.y_stride + n;
    if (n + E <= p.N) {
        if constexpr (F32) {
            const f32x4 o = {v[0], v[1], v[2], v[3]};
            if (PAST) __builtin_nontemporal_store(o, (any_f32x4 *)((float *)p.y + at));
            else *(any_f32x4 *)((float *)p.y + at) = o;
        } else {
            uint32_t o[E / 2];
#pragma unroll
            for (int e = 0; e < E / 2; ++e) o[e] = f2bf2(v[2 * e], v[2 * e + 1]);
            if constexpr (E == 8 && PAST)
                __builtin_nontemporal_store((u32x4){o[0], o[1], o[2], o[3]}, (any_u32x4 *)((uint16_t *)p.y + at));
            else if constexpr (E == 8)
                *(any_u32x4 *)((uint16_t *)p.y + at) = (u32x4){o[0], o[1], o[2], o[3]};
            else
                *(any_u32x2 *)((uint16_t *)p.y + at) = (u32x2){o[0], o[1]};
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
        if (n + e >= p.N) continue;
        if constexpr (F32) ((float *)p.y)[at + e] = v[e];
        else ((uint16_t *)p.y)[at + e] = (uint16_t)f2bf(v[e]);
    }
}

// the same with the residual, if any
template <bool F32, int E, bool PAST = false>
__device__ __forceinline__ void put_sum(const Product &p, int64_t t, int n, float (&v)[E]) {
    if (p.residual) {
        Rest<F32, E> r;
        r.load(p, t * p.y_stride + n, n);
        r.add(v);
    }
    put<F32, E, PAST>(p, t, n, v);
}

// Scales and bias of E columns from n
template <int E>
struct Columns {
    Scale w[E];
    float bias[E];
    __device__ __forceinline__ void load(const Product &p, int n) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int at = min(n + e, p.N - 1);
            w[e] = split(p.ws[at]);
            bias[e] = p.bias ? p.bias[at] : 0.f;
        }
    }
    // the columns of a row with scale x: bias is added where there is one, so that a
    // sum of -0 stays one without
    __device__ __forceinline__ void apply(const Product &p, const int (&sum)[E], Scale x, float (&v)[E]) const {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = scaled(sum[e], x, w[e]);
        if (p.bias) {
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] += bias[e];
        }
    }
};

}  // namespace int8
}  // namespace echo
