// int8_stream.hpp -- products in 8-bit integers for few tokens: every wave streams its
// own weights.
#pragma once

#include "int8_tiled.hpp"

namespace echo {
namespace int8 {

// One workgroup: 16 NT weight rows and up to 16 TT tokens; its eight waves take
// equal ranges of K and their sums meet in LDS.  A wave copies its 128 bytes of the
// weight rows and of XR token rows straight into a ring of D stages of its own and
// waits for nobody.  XR 8: at most 8 tokens, the operand's other columns repeat them.
// Bound by memory and a launch: 8 x 6144 x 4096 takes 6.1 us with weights from the
// caches, 6.4 a call with weights from memory (25 MB, 4.0 TB/s).
constexpr int kStreamWaves = 8;

constexpr int stream_stage(int NT, int XR) { return (16 * NT + XR) * kStep; }

template <bool F32, bool ONCE, int NT, int XR, int D>
__global__ __launch_bounds__(64 * kStreamWaves) void stream_kernel(Product p, int n_tiles) {
    constexpr int TT = XR > 16 ? 2 : 1, COPIES = 2 * NT + XR / 8, STAGE = stream_stage(NT, XR);
    __shared__ __align__(16) uint8_t lds[kStreamWaves * D * STAGE];
    static_assert(kStreamWaves * NT * TT * 1024 <= sizeof lds);
    const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int ti = blockIdx.x / n_tiles, n0 = 16 * NT * (blockIdx.x - ti * n_tiles);
    const int row0 = 16 * TT * ti, rows = min(16 * TT, p.T - row0);
    const int kb0 = p.KB * wave / kStreamWaves, kb1 = p.KB * (wave + 1) / kStreamWaves;
    uint8_t *ring = lds + wave * D * STAGE;
    const int piece = (lane & 7) ^ (lane >> 3);
    const uint8_t *src[COPIES];
#pragma unroll
    for (int i = 0; i < COPIES; ++i) {
        const int r = 8 * i + (lane >> 3);
        src[i] = (i < 2 * NT ? p.w + (int64_t)min(n0 + r, p.N - 1) * p.K
                             : p.x + (int64_t)(row0 + min(r - 16 * NT, rows - 1)) * p.K) + 16 * piece;
    }
    auto copy = [&](int kb, int slot) {
        uint8_t *dst = ring + slot * STAGE;
        const bool in = kStep * kb + 16 * piece < p.K;
#pragma unroll
        for (int i = 0; i < COPIES; ++i) {
            const uint8_t *from = in ? src[i] + (int64_t)kStep * kb : kZeros;
            if (ONCE && i < 2 * NT)
                __builtin_amdgcn_global_load_lds((const void *)from, (lds_void *)(dst + 1024 * i), 16, 0, 2);   // nt
            else
                __builtin_amdgcn_global_load_lds((const void *)from, (lds_void *)(dst + 1024 * i), 16, 0, 0);
        }
    };
    i32x4 acc[NT][TT] = {};
    const int at = 16 * (g ^ (c & 7));
    int slot = 0;
    auto step = [&](int kb) {
        const uint8_t *stage = ring + slot * STAGE;
        u32x4 a[2][NT], x[2][TT];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int i = 0; i < NT; ++i) a[h][i] = *(const u32x4 *)(stage + (16 * i + c) * kStep + (at ^ (64 * h)));
#pragma unroll
            for (int t = 0; t < TT; ++t)
                x[h][t] = *(const u32x4 *)(stage + (16 * NT + (XR == 8 ? c & 7 : 16 * t + c)) * kStep + (at ^ (64 * h)));
        }
        // the stage has been read: its operands are in registers
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (kb + D < kb1) copy(kb + D, slot);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int t = 0; t < TT; ++t) acc[i][t] = mfma64(a[h][i], x[h][t], acc[i][t]);
        slot = slot + 1 == D ? 0 : slot + 1;
    };
#pragma unroll
    for (int i = 0; i < D; ++i)
        if (kb0 + i < kb1) copy(kb0 + i, i);
    int kb = kb0;
    for (; kb + D <= kb1; ++kb) {   // D - 1 stages are in flight behind this one
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((D - 1) * COPIES) : "memory");
        step(kb);
    }
    for (; kb < kb1; ++kb) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        step(kb);
    }
    __syncthreads();   // all waves are done with their rings
    i32x4 *part = (i32x4 *)lds;   // [waves][NT TT][64]
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int t = 0; t < TT; ++t) part[(wave * NT * TT + i * TT + t) * 64 + lane] = acc[i][t];
    __syncthreads();
    if (wave < NT * TT) {
        i32x4 s = part[wave * 64 + lane];
#pragma unroll
        for (int k = 1; k < kStreamWaves; ++k) s += part[(k * NT * TT + wave) * 64 + lane];
        const int r = 16 * (wave % TT) + c, n = n0 + 16 * (wave / TT) + 4 * g;
        if (r < rows && n < p.N) {
            Columns<4> cols;
            cols.load(p, n);
            const int sum[4] = {s[0], s[1], s[2], s[3]};
            float v[4];
            cols.apply(p, sum, split(p.xs[row0 + r]), v);
            put_sum<F32, 4>(p, row0 + r, n, v);
        }
    }
}

template <bool F32, bool ONCE, int NT, int XR, int D>
hipError_t launch_stream(const Product &p, hipStream_t st) {
    const int n_tiles = cdiv(p.N, 16 * NT), t_tiles = cdiv(p.T, XR > 16 ? 32 : 16);
    hipLaunchKernelGGL((stream_kernel<F32, ONCE, NT, XR, D>), dim3((unsigned)(n_tiles * t_tiles)), dim3(64 * kStreamWaves),
                       0, st, p, n_tiles);
    return hipSuccess;
}

}  // namespace int8
}  // namespace echo
