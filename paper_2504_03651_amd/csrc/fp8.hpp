// fp8.hpp -- device pieces shared by the e4m3 kernels (fp8.hip, moe.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace echo {
namespace fp8 {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kQ = 128;   // values of a row under one scale

__host__ __device__ inline int cdiv(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

__device__ __forceinline__ float bf2f(uint32_t b) { return __uint_as_float(b << 16); }

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// fp32 -> bf16, round to nearest even (a NaN stays one): one instruction
__device__ __forceinline__ uint32_t f2bf(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
__device__ __forceinline__ uint32_t f2bf2(float x, float y) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){x, y}, bf16x2));
}

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// Two fp32 -> two fp16, round to nearest even
__device__ __forceinline__ uint32_t f2h2(float x, float y) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){x, y}, f16x2));
}

// Two fp32 -> two e4m3fn codes in the low 16 bits, round to nearest even,
// saturating at 448, NaN to 0x7F (v_cvt_pk_fp8_f32 on clamped values).
__device__ __forceinline__ uint32_t e4m3x2(float x, float y) {
    const uint32_t w = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(
        __builtin_amdgcn_fmed3f(x, -448.f, 448.f), __builtin_amdgcn_fmed3f(y, -448.f, 448.f), 0, false);
    const uint32_t nan = (x != x ? 0x7Fu : 0u) | (y != y ? 0x7F00u : 0u);
    const uint32_t keep = (x != x ? 0u : 0xFFu) | (y != y ? 0u : 0xFF00u);
    return (w & keep) | nan;
}

// The scale of a block whose largest magnitude is amax
__device__ __forceinline__ float scale_of(float amax) {
    const float s = amax / 448.0f;
    return s == 0.f ? 1.f : s;
}

// A block's sum is scaled by the product x w of its two scales, rounded to fp32.  Where
// that is no normal number (subnormal, zero, infinite, NaN) the sum may be one that
// makes the result an ordinary number all the same: it is then multiplied by one
// scale after the other, the larger first under a small product, the smaller first
// under a large one, so that the first product stays in range wherever the second
// does.  Few tokens do that beside the step, tiles by taking a wave's sums again
// (a test of each step's scales: 5% of 100 x 4096 x 4096, up to 1.5% from 137 tokens on;
// decided step by step it cost twice that).
constexpr uint32_t kOddClass = 2u << 24;
__device__ __forceinline__ uint32_t scale_class(float s) {   // below kOddClass: not normal
    return (__float_as_uint(s) << 1) + (1u << 24);   // exponents 255 and 0 become 0 and 1
}
__device__ __forceinline__ bool odd_scale(float s) { return scale_class(s) < kOddClass; }
__device__ __forceinline__ f32x4 scaled(f32x4 v, float x, float w) {
    const bool x_less = fabsf(x) < fabsf(w);
    const float less = x_less ? x : w, more = x_less ? w : x;
    const bool small = fabsf(x * w) < 1.f && less != 0.f;   // 0 first: it leaves no infinity
    return v * (small ? more : less) * (small ? less : more);
}

// Eight e4m3 codes as bf16, exact (every e4m3 value is a bf16 value)
__device__ __forceinline__ bf16x8 widen8(int lo, int hi) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)lo, 1.0f, false);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)lo, 1.0f, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)hi, 1.0f, false);
    const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)hi, 1.0f, true);
    return (bf16x8){a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// P[16 rows of a][16 rows of b] of 128 contraction steps, from zero.  Each lane
// holds 32 codes of row lane % 16 of each operand; which of the 128 steps they
// are is free as long as both operands agree (here bytes 16 g .. and 64 + 16 g ..,
// g = lane / 16, two 16-byte loads).  The lane gets column lane % 16 (a row of
// b) and rows 4 g .. 4 g + 3 (of a).
//
// The e4m3 instruction adds its products at fewer bits than fp32 holds: those of
// eight neighbours along K are cut off, towards zero, at 2^-13 of the power of two
// below the largest of the eight (found with single small products beside large
// ones that cancel).  Over 200 tiles of N(0, 1) operands a sum of 128 was 1.5e-5 off
// in the 2-norm, the 16x16x32 form the same to the bit.  Under a result that is
// rounded to bf16 (2^-9) that is little; fp32 results (WIDE) take the products in
// bf16, where they are exact and the sum is 1e-8 off, at half the rate.  (Products
// of up to 32 tokens, which wait for their weights, would be 1 to 4% slower that way.)
template <bool WIDE>
__device__ __forceinline__ f32x4 mfma128(i32x8 a, i32x8 b) {
    f32x4 z = {0.f, 0.f, 0.f, 0.f};
    if constexpr (WIDE) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(a[2 * i], a[2 * i + 1]),
                                                        widen8(b[2 * i], b[2 * i + 1]), z, 0, 0, 0);
        return z;
    }
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, z, 0, 0, 0, 0, 0, 0);
}

__device__ __forceinline__ i32x8 pair(u32x4 lo, u32x4 hi) {
    return (i32x8){(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3],
                   (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
}

// ---------------------------------------------------------------- products

// What a product's kernel reads and writes.
//   Plain   y[t][n] (+)= x[t] . w[n]
//   GateUp  rows are (token, expert) pairs in order of expert; a tile's pair p
//           reads token order[p] / top_k and writes codes and scales of row p of
//           SiLU(x . w[n]) * (x . w[N + n]), n < N = I
//   Down    pair p reads row p and writes row order[p] of y, fp16 times powers of
//           two whose exponents, of groups of a wave's columns, go to ye
enum class Mode { Plain, GateUp, Down };

struct Tile {
    int expert, row0, rows, pad;
};

struct ProductArgs {
    const uint8_t *x;      // codes [rows][K]
    const float *xs;       // [rows][KB]
    const uint8_t *w;      // codes of the first expert
    const float *ws;
    int64_t w_expert, ws_expert;   // elements from one expert to the next
    int T, N, K, KB;
    // Plain, Down
    const void *residual;
    void *y;
    int64_t y_stride;
    float *part;           // [splits][T][part_pitch], for products over ranges of K
    int part_pitch;
    // GateUp
    uint8_t *hc;           // [pairs][N]
    float *hs;             // [pairs][ceil(N / 128)]
    // GateUp, Down
    const int *num_tiles;
    const Tile *tiles;
    const int *order;      // pair of each place
    int top_k;
    // Down
    int8_t *ye;            // [pairs][y_groups]
    int y_groups;
};

// LDS written by lanes of this wave is there for its other lanes
__device__ __forceinline__ void wave_lds() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Memory that need not be aligned to more than its elements: the hardware takes such
// accesses of 8 and 16 bytes, which the compiler emits for these types.
typedef u32x4 __attribute__((aligned(2))) any_u32x4;
typedef u32x2 __attribute__((aligned(2))) any_u32x2;
typedef f32x4 __attribute__((aligned(4))) any_f32x4;

// v plus the residual of a lane's four columns n .. n + 3 at element `at`
template <bool F32>
__device__ __forceinline__ f32x4 plus_residual(const ProductArgs &p, int64_t at, int n, f32x4 v) {
    if constexpr (F32) {
        const float *r = (const float *)p.residual + at;
        if (n + 4 <= p.N) return v + *(const any_f32x4 *)r;
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (n + e < p.N) v[e] += r[e];
    } else {
        const uint16_t *r = (const uint16_t *)p.residual + at;
        if (n + 4 <= p.N) {
            const u32x2 q = *(const any_u32x2 *)r;
#pragma unroll
            for (int e = 0; e < 2; ++e) v[2 * e] += bf2f(q[e] & 0xFFFFu), v[2 * e + 1] += bf2f(q[e] >> 16);
            return v;
        }
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (n + e < p.N) v[e] += bf2f(r[e]);
    }
    return v;
}

// y of a lane's four columns n .. n + 3 of row t, the residual added
template <bool F32>
__device__ __forceinline__ void store4(const ProductArgs &p, int64_t t, int n, f32x4 v) {
    const int64_t at = t * p.y_stride + n;
    if (p.residual) v = plus_residual<F32>(p, at, n, v);
    if constexpr (F32) {
        float *y = (float *)p.y + at;
        if (n + 4 <= p.N) {
            *(any_f32x4 *)y = v;
            return;
        }
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (n + e < p.N) y[e] = v[e];
    } else {
        uint16_t *y = (uint16_t *)p.y + at;
        if (n + 4 <= p.N) {
            *(any_u32x2 *)y = (u32x2){f2bf2(v[0], v[1]), f2bf2(v[2], v[3])};
            return;
        }
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (n + e < p.N) y[e] = (uint16_t)f2bf(v[e]);
    }
}

}  // namespace fp8
}  // namespace echo
