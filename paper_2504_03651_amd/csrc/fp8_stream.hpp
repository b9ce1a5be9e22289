// fp8_stream.hpp -- e4m3 products for few tokens: weights streamed from memory
// into registers.
#pragma once

#include "fp8.hpp"

namespace echo {
namespace fp8 {

// 32 codes of a lane's row in block kb (rows at p, which includes 16 g);
// codes at or past K are zeros.
__device__ __forceinline__ i32x8 load_block(const uint8_t *p, int kb) {
    return pair(*(const u32x4 *)(p + kQ * kb), *(const u32x4 *)(p + kQ * kb + 64));
}
__device__ __forceinline__ i32x8 load_tail(const uint8_t *p, int kb, int K, int g) {
    const u32x4 z = {0u, 0u, 0u, 0u};
    const int k = kQ * kb + 16 * g;
    return pair(k < K ? *(const u32x4 *)(p + kQ * kb) : z,
                k + 64 < K ? *(const u32x4 *)(p + kQ * kb + 64) : z);
}

// acc[i][j] += the products of weight rows w[i] and token rows x[j] over blocks
// kb0, kb0 + step, ... of K; each block's sum is scaled on its way into acc.
template <bool WIDE, int NT, int TT>
__device__ __forceinline__ void stream_blocks(const uint8_t *const (&w)[NT],
                                              const float *const (&ws)[NT],
                                              const uint8_t *const (&x)[TT],
                                              const float *const (&xs)[TT], int kb0, int step,
                                              int K, int KB, int g, f32x4 (&acc)[NT][TT]) {
    const int full = K / kQ;
    int kb = kb0;
#pragma unroll 4
    for (; kb < full; kb += step) {
        i32x8 a[NT];
#pragma unroll
        for (int i = 0; i < NT; ++i) a[i] = load_block(w[i], kb);
#pragma unroll
        for (int j = 0; j < TT; ++j) {
            const i32x8 b = load_block(x[j], kb);
            const float s = xs[j][kb];
#pragma unroll
            for (int i = 0; i < NT; ++i) acc[i][j] += mfma128<WIDE>(a[i], b) * (s * ws[i][kb]);
        }
    }
    if (kb == full && full < KB) {
        i32x8 a[NT];
#pragma unroll
        for (int i = 0; i < NT; ++i) a[i] = load_tail(w[i], kb, K, g);
#pragma unroll
        for (int j = 0; j < TT; ++j) {
            const i32x8 b = load_tail(x[j], kb, K, g);
            const float s = xs[j][kb];
#pragma unroll
            for (int i = 0; i < NT; ++i) acc[i][j] += mfma128<WIDE>(a[i], b) * (s * ws[i][kb]);
        }
    }
}

// One workgroup: 16 weight rows, 16 TT tokens, its KS waves taking every KS-th
// block of K; their sums meet in LDS in the waves' order.
template <Mode M, bool F32, int TT, int KS>
__global__ __launch_bounds__(64 * KS) void stream_kernel(ProductArgs p, int n_tiles) {
    __shared__ f32x4 part[KS][TT][64];
    const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int ti = blockIdx.x / n_tiles, n0 = 16 * (blockIdx.x - ti * n_tiles);
    int row0 = 16 * TT * ti, rows = p.T - row0;
    const uint8_t *wbase = p.w;
    const float *sbase = p.ws;
    if constexpr (M == Mode::Down) {
        if (ti >= *p.num_tiles) return;
        const Tile t = p.tiles[ti];
        row0 = t.row0;
        rows = t.rows;
        wbase += t.expert * p.w_expert;
        sbase += t.expert * p.ws_expert;
    }
    const uint8_t *w[1] = {wbase + (int64_t)min(n0 + c, p.N - 1) * p.K + 16 * g};
    const float *ws[1] = {sbase + (int64_t)(n0 / kQ) * p.KB};
    const uint8_t *x[TT];
    const float *xs[TT];
#pragma unroll
    for (int j = 0; j < TT; ++j) {
        const int64_t r = row0 + min(16 * j + c, rows - 1);
        x[j] = p.x + r * p.K + 16 * g;
        xs[j] = p.xs + r * p.KB;
    }
    f32x4 acc[1][TT] = {};
    stream_blocks<F32, 1, TT>(w, ws, x, xs, wave, KS, p.K, p.KB, g, acc);
#pragma unroll
    for (int j = 0; j < TT; ++j) part[wave][j][lane] = acc[0][j];
    __syncthreads();
    for (int j = wave; j < TT; j += KS) {
        f32x4 v = part[0][j][lane];
#pragma unroll
        for (int k = 1; k < KS; ++k) v += part[k][j][lane];
        const int r = 16 * j + c;
        if (r < rows) {
            const int64_t t = M == Mode::Down ? p.order[row0 + r] : row0 + r;
            store4<F32>(p, t, n0 + 4 * g, v);
        }
    }
}

// One workgroup of 8 waves: 128 columns of an expert's activation for 16 TT of
// its pairs; wave v has the gate and the up rows 16 v .. 16 v + 15 of the block.
template <int TT>
__global__ __launch_bounds__(512) void stream_gate_up_kernel(ProductArgs p, int n_tiles) {
    __shared__ float peak[8][16 * TT];
    const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int ti = blockIdx.x / n_tiles, nb = blockIdx.x - ti * n_tiles;
    if (ti >= *p.num_tiles) return;
    const Tile t = p.tiles[ti];
    const int n0 = kQ * nb + 16 * wave;
    const int64_t nr = min(n0 + c, p.N - 1);
    const uint8_t *wbase = p.w + t.expert * p.w_expert + 16 * g;
    const float *sbase = p.ws + t.expert * p.ws_expert + (int64_t)nb * p.KB;
    const uint8_t *w[2] = {wbase + nr * p.K, wbase + (p.N + nr) * p.K};
    const float *ws[2] = {sbase, sbase + (int64_t)n_tiles * p.KB};
    const uint8_t *x[TT];
    const float *xs[TT];
#pragma unroll
    for (int j = 0; j < TT; ++j) {
        const int64_t r = p.order[t.row0 + min(16 * j + c, t.rows - 1)] / p.top_k;
        x[j] = p.x + r * p.K + 16 * g;
        xs[j] = p.xs + r * p.KB;
    }
    f32x4 acc[2][TT] = {};
    stream_blocks<false, 2, TT>(w, ws, x, xs, 0, 1, p.K, p.KB, g, acc);
    f32x4 h[TT];
#pragma unroll
    for (int j = 0; j < TT; ++j) {
        float m = 0.f;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float a = acc[0][j][r];
            h[j][r] = n0 + 4 * g + r < p.N ? a / (1.f + expf(-a)) * acc[1][j][r] : 0.f;
            m = fmaxf(m, fabsf(h[j][r]));   // a NaN keeps out
        }
        m = fmaxf(m, __shfl_xor(m, 16));
        m = fmaxf(m, __shfl_xor(m, 32));
        if (g == 0) peak[wave][16 * j + c] = m;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < TT; ++j) {
        const int r = 16 * j + c;
        if (r >= t.rows) continue;
        float m = peak[0][r];
#pragma unroll
        for (int v = 1; v < 8; ++v) m = fmaxf(m, peak[v][r]);
        const float s = scale_of(m);
        const int64_t row = t.row0 + r;
        if (wave == 0 && g == 0) p.hs[row * n_tiles + nb] = s;
        if (n0 + 4 * g < p.N)   // N a multiple of 16
            *(uint32_t *)(p.hc + row * p.N + n0 + 4 * g) =
                e4m3x2(h[j][0] / s, h[j][1] / s) | (e4m3x2(h[j][2] / s, h[j][3] / s) << 16);
    }
}

}  // namespace fp8
}  // namespace echo
