// fp8_stream.hpp -- e4m3 products for few tokens: weights streamed from memory
// into registers.
#pragma once

#include "fp8.hpp"

namespace echo {
namespace fp8 {

// 32 codes of a lane's row in block kb (rows at p, which includes 16 g); ONCE:
// past the caches, for weights that one workgroup reads
template <bool ONCE>
__device__ __forceinline__ i32x8 load_block(const uint8_t *p, int kb) {
    const u32x4 *q = (const u32x4 *)(p + kQ * kb);
    if constexpr (ONCE) return pair(__builtin_nontemporal_load(q), __builtin_nontemporal_load(q + 4));
    return pair(q[0], q[4]);
}
// codes at or past K are zeros
__device__ __forceinline__ i32x8 load_tail(const uint8_t *p, int kb, int K, int g) {
    const u32x4 z = {0u, 0u, 0u, 0u};
    const int k = kQ * kb + 16 * g;
    return pair(k < K ? *(const u32x4 *)(p + kQ * kb) : z,
                k + 64 < K ? *(const u32x4 *)(p + kQ * kb + 64) : z);
}

// acc[i][j] += the products of weight rows w[i] and token rows x[j] over blocks
// kb0 .. kb1 - 1 of K, U of them in flight at a time; each block's sum is scaled
// on its way into acc.
template <bool WIDE, bool ONCE, int U, int NT, int TT>
__device__ __forceinline__ void stream_blocks(const uint8_t *const (&w)[NT],
                                              const float *const (&ws)[NT],
                                              const uint8_t *const (&x)[TT],
                                              const float *const (&xs)[TT], int kb0, int kb1,
                                              int K, int g, f32x4 (&acc)[NT][TT]) {
    const int full = min(kb1, K / kQ);
    for (int kb = kb0; kb < full; kb += U) {
        i32x8 a[U][NT], b[U][TT];
        float sw[U][NT], sx[U][TT];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = min(kb + u, full - 1);
#pragma unroll
            for (int i = 0; i < NT; ++i) a[u][i] = load_block<ONCE>(w[i], k), sw[u][i] = ws[i][k];
#pragma unroll
            for (int j = 0; j < TT; ++j) b[u][j] = load_block<false>(x[j], k), sx[u][j] = xs[j][k];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (kb + u >= full) break;
#pragma unroll
            for (int j = 0; j < TT; ++j)
#pragma unroll
                for (int i = 0; i < NT; ++i)
                    acc[i][j] += mfma128<WIDE>(a[u][i], b[u][j]) * (sx[u][j] * sw[u][i]);
        }
    }
    if (full < kb1) {   // a last block of less than 128
        i32x8 a[NT];
#pragma unroll
        for (int i = 0; i < NT; ++i) a[i] = load_tail(w[i], full, K, g);
#pragma unroll
        for (int j = 0; j < TT; ++j) {
            const i32x8 b = load_tail(x[j], full, K, g);
            const float s = xs[j][full];
#pragma unroll
            for (int i = 0; i < NT; ++i) acc[i][j] += mfma128<WIDE>(a[i], b) * (s * ws[i][full]);
        }
    }
}

// One workgroup: 16 NT weight rows, 16 TT tokens, its KS waves taking equal
// ranges of K; their sums meet in LDS in the waves' order.
template <bool F32, bool ONCE, int NT, int TT, int KS, int U>
__global__ __launch_bounds__(64 * KS) void stream_kernel(ProductArgs p, int n_tiles) {
    __shared__ f32x4 part[KS][NT * TT][64];
    const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int ti = blockIdx.x / n_tiles, n0 = 16 * NT * (blockIdx.x - ti * n_tiles);
    const int row0 = 16 * TT * ti, rows = p.T - row0;
    const uint8_t *w[NT];
    const float *ws[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        w[i] = p.w + (int64_t)min(n0 + 16 * i + c, p.N - 1) * p.K + 16 * g;
        ws[i] = p.ws + (int64_t)min((n0 + 16 * i) / kQ, (p.N - 1) / kQ) * p.KB;
    }
    const uint8_t *x[TT];
    const float *xs[TT];
#pragma unroll
    for (int j = 0; j < TT; ++j) {
        const int64_t r = row0 + min(16 * j + c, rows - 1);
        x[j] = p.x + r * p.K + 16 * g;
        xs[j] = p.xs + r * p.KB;
    }
    f32x4 acc[NT][TT] = {};
    stream_blocks<F32, ONCE, U, NT, TT>(w, ws, x, xs, p.KB * wave / KS, p.KB * (wave + 1) / KS, p.K, g, acc);
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int j = 0; j < TT; ++j) part[wave][i * TT + j][lane] = acc[i][j];
    __syncthreads();
    for (int q = wave; q < NT * TT; q += KS) {
        f32x4 v = part[0][q][lane];
#pragma unroll
        for (int k = 1; k < KS; ++k) v += part[k][q][lane];
        const int i = q / TT, r = 16 * (q % TT) + c;
        if (r < rows) store4<F32>(p, row0 + r, n0 + 16 * i + 4 * g, v);
    }
}

}  // namespace fp8
}  // namespace echo
