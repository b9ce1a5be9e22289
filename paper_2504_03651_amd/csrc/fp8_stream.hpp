// fp8_stream.hpp -- e4m3 products for few tokens: every wave streams its own
// weights.
#pragma once

#include "fp8_tiled.hpp"

namespace echo {
namespace fp8 {

// One workgroup: 16 NT weight rows and up to 16 TT tokens; its eight waves take
// equal ranges of K and their sums meet in LDS in the waves' order.  A wave copies
// its 128 columns of the weight rows and of XR token rows straight into a ring of D
// stages of its own and waits for nobody.  (Loads into registers took a request
// for every 16 bytes, as neighbouring lanes of a matrix operand are rows apart; copies
// have eight lanes a row.  8 x 6144 x 4096, calls back to back: 8.5 us with weights
// from memory, 3.0 TB/s, 8.0 over the same ones.)  XR 8: at most 8 tokens, the
// operand's other columns repeat them.  The scales of the whole range come first.
constexpr int kStreamWaves = 8;

__host__ __device__ constexpr int stream_stage(int NT, int XR) { return (16 * NT + XR) * kQ; }

// LDS bytes of a wave: its ring, and the scales of `blocks` blocks of K
__host__ __device__ inline int stream_bytes(int NT, int XR, int D, int blocks) {
    const int four = (blocks + 3) / 4 * 4;
    return D * stream_stage(NT, XR) + four * (XR > 16 ? 128 : 64) + (blocks + 63) / 64 * 256;
}

template <bool F32, bool ONCE, int NT, int XR, int D>
__global__ __launch_bounds__(64 * kStreamWaves) void stream_kernel(ProductArgs p, int n_tiles, int wave_bytes) {
    constexpr int TT = XR > 16 ? 2 : 1, COPIES = 2 * NT + XR / 8;
    extern __shared__ __align__(16) uint8_t lds[];
    const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int ti = blockIdx.x / n_tiles, n0 = 16 * NT * (blockIdx.x - ti * n_tiles);
    const int row0 = 16 * TT * ti, rows = min(16 * TT, p.T - row0);
    const int kb0 = p.KB * wave / kStreamWaves, kb1 = p.KB * (wave + 1) / kStreamWaves, blocks = kb1 - kb0;
    uint8_t *ring = lds + wave * wave_bytes;
    float *xsl = (float *)(ring + D * stream_stage(NT, XR));     // [blocks][16 TT]
    float *wsl = xsl + (blocks + 3) / 4 * 4 * 16 * TT;           // [blocks]

    // scales: four blocks of sixteen tokens, or 64 blocks of the rows, a copy
    const float *xs = p.xs + (int64_t)row0 * p.KB, *ws = p.ws + (int64_t)(n0 / kQ) * p.KB;
    for (int b = 0; b < blocks; b += 4)
#pragma unroll
        for (int t = 0; t < TT; ++t)
            // TT 2: the copy of tokens 16 .. 31 lies behind that of 0 .. 15
            __builtin_amdgcn_global_load_lds(
                (const void *)(xs + (int64_t)min(16 * t + c, rows - 1) * p.KB + min(kb0 + b + g, p.KB - 1)),
                (lds_void *)(xsl + (b / 4 * TT + t) * 64), 4, 0, 0);
    for (int b = 0; b < blocks; b += 64)
        __builtin_amdgcn_global_load_lds((const void *)(ws + min(kb0 + b + lane, p.KB - 1)),
                                         (lds_void *)(wsl + b), 4, 0, 0);

    const int piece = (lane & 7) ^ (lane >> 3);
    const uint8_t *src[COPIES];
#pragma unroll
    for (int i = 0; i < COPIES; ++i) {
        const int r = 8 * i + (lane >> 3);
        src[i] = (i < 2 * NT ? p.w + (int64_t)min(n0 + r, p.N - 1) * p.K
                             : p.x + (int64_t)(row0 + min(r - 16 * NT, rows - 1)) * p.K) + 16 * piece;
    }
    auto copy = [&](int kb, int slot) {
        uint8_t *dst = ring + slot * stream_stage(NT, XR);
        const bool in = kQ * kb + 16 * piece < p.K;
#pragma unroll
        for (int i = 0; i < COPIES; ++i) {
            const uint8_t *from = in ? src[i] + (int64_t)kQ * kb : kZeros;
            if (ONCE && i < 2 * NT)
                __builtin_amdgcn_global_load_lds((const void *)from, (lds_void *)(dst + 1024 * i), 16, 0, 2);   // nt
            else
                __builtin_amdgcn_global_load_lds((const void *)from, (lds_void *)(dst + 1024 * i), 16, 0, 0);
        }
    };
    f32x4 acc[NT][TT] = {};
    const int at = 16 * (g ^ (c & 7));
    int slot = 0;
    auto step = [&](int kb) {
        const uint8_t *stage = ring + slot * stream_stage(NT, XR);
        auto read = [&](int row) {
            const uint8_t *l = stage + row * kQ;
            return pair(*(const u32x4 *)(l + at), *(const u32x4 *)(l + (at ^ 64)));
        };
        const int b = kb - kb0;
        const float sw = wsl[b];
        i32x8 a[NT], x[TT];
        float s[TT], sx[TT];
        bool odd = false;
#pragma unroll
        for (int i = 0; i < NT; ++i) a[i] = read(16 * i + c);
#pragma unroll
        for (int t = 0; t < TT; ++t) {
            x[t] = read(16 * NT + (XR == 8 ? c & 7 : 16 * t + c));
            sx[t] = xsl[(b / 4 * TT + t) * 64 + b % 4 * 16 + c];
            s[t] = sx[t] * sw;
            odd |= odd_scale(s[t]);
        }
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int t = 0; t < TT; ++t) acc[i][t] += mfma128<F32>(a[i], x[t]) * (odd_scale(s[t]) ? 0.f : s[t]);
        if (__any(odd)) {
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int t = 0; t < TT; ++t) {
                    const f32x4 v = scaled(mfma128<F32>(a[i], x[t]), sx[t], sw);
                    if (odd_scale(s[t])) acc[i][t] += v;
                }
        }
        // the stage has been read: its operands are in registers
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (kb + D < kb1) copy(kb + D, slot);
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
    f32x4 *part = (f32x4 *)lds;   // [waves][NT TT][64]
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int t = 0; t < TT; ++t) part[(wave * NT * TT + i * TT + t) * 64 + lane] = acc[i][t];
    __syncthreads();
    if (wave < NT * TT) {
        f32x4 v = part[wave * 64 + lane];
#pragma unroll
        for (int k = 1; k < kStreamWaves; ++k) v += part[(k * NT * TT + wave) * 64 + lane];
        const int i = wave / TT, r = 16 * (wave % TT) + c;
        if (r < rows) store4<F32>(p, row0 + r, n0 + 16 * i + 4 * g, v);
    }
}

template <bool F32, bool ONCE, int NT, int XR, int D>
hipError_t launch_stream(const ProductArgs &p, hipStream_t st) {
    static std::atomic<int> resident[64];
    const int n_tiles = cdiv(p.N, 16 * NT), t_tiles = cdiv(p.T, XR > 16 ? 32 : 16);
    const int wave_bytes = stream_bytes(NT, XR, D, cdiv(p.KB, kStreamWaves));
    const int sums = kStreamWaves * NT * (XR > 16 ? 2 : 1) * 1024;
    const int bytes = wave_bytes * kStreamWaves > sums ? wave_bytes * kStreamWaves : sums;
    return launch_lds(stream_kernel<F32, ONCE, NT, XR, D>, resident, 160 * 1024, bytes, (int64_t)n_tiles * t_tiles,
                      false, 64 * kStreamWaves, st, p, n_tiles, wave_bytes);
}

}  // namespace fp8
}  // namespace echo
