// fp8_tiled.hpp -- e4m3 products for many tokens: operand tiles in LDS.
#pragma once

#include "fp8.hpp"

namespace echo {
namespace fp8 {

typedef __attribute__((address_space(3))) void lds_void;

// where 16-byte pieces past the end of a row come from
__device__ __align__(16) const uint8_t kZeros[16] = {};

// s_waitcnt immediate: vmcnt n, everything else unconstrained
constexpr int wait_vm(int n) { return (n & 15) | ((n >> 4) << 14) | (7 << 4) | (15 << 8); }

// One workgroup of WN x WT waves: BN weight rows (GateUp: BN / 2 gate rows and
// the up rows of the same columns) by BT tokens, K in steps of 128 through two
// LDS buffers that are filled straight from memory.  A row's 128 codes are eight
// 16-byte pieces; piece q of row r lies at place q ^ (r & 7), so that the eight
// lanes that read one piece of eight rows meet eight different places.  Each
// step's sum comes out of the matrix instruction alone and is scaled on its way
// into the accumulators: one FMA a value, beside the products of the next tiles.
template <Mode M, bool F32, int BN, int BT, int WN, int WT>
__global__ __launch_bounds__(64 * WN *WT) void tiled_kernel(ProductArgs p, int n_tiles, int t_tiles) {
    constexpr int W = WN * WT, NW = BN / WN, TW = BT / WT;   // a wave's rows and tokens
    constexpr int NI = NW / 16, NJ = TW / 16;
    constexpr int STAGE = (BN + BT) * kQ;
    constexpr int COPIES = STAGE / 1024 / W;   // 1 KiB copies of a wave per step
    static_assert(COPIES * 1024 * W == STAGE && NI >= 2);
    extern __shared__ __align__(16) uint8_t lds[];
    const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wn = wave % WN, wt = wave / WN;

    const int ti = blockIdx.x / n_tiles, nb = blockIdx.x - ti * n_tiles;
    int row0 = BT * ti, rows = min(BT, p.T - row0);
    const uint8_t *wbase = p.w;
    const float *sbase = p.ws;
    if constexpr (M != Mode::Plain) {
        if (ti >= *p.num_tiles) return;
        const Tile t = p.tiles[ti];
        row0 = t.row0;
        rows = t.rows;
        wbase += t.expert * p.w_expert;
        sbase += t.expert * p.ws_expert;
    }
    const int n0 = (M == Mode::GateUp ? BN / 2 : BN) * nb;

    // sources of this lane's copies: rows of weights, then of tokens
    const uint8_t *src[COPIES];
#pragma unroll
    for (int i = 0; i < COPIES; ++i) {
        const int r = 8 * (wave * COPIES + i) + (lane >> 3);   // row of the stage
        int64_t at;
        if (r < BN) {
            if constexpr (M == Mode::GateUp) {
                const int q = r % NW, n = min(n0 + (r / NW) * (NW / 2) + q % (NW / 2), p.N - 1);
                at = (int64_t)(q < NW / 2 ? n : p.N + n) * p.K;
            } else {
                at = (int64_t)min(n0 + r, p.N - 1) * p.K;
            }
            src[i] = wbase + at;
        } else {
            int64_t t = row0 + min(r - BN, rows - 1);
            if constexpr (M == Mode::GateUp) t = p.order[t] / p.top_k;
            src[i] = p.x + t * p.K;
        }
    }
    const int piece = (lane & 7) ^ (lane >> 3);
    auto copy = [&](int kb, int buf) {
        const int k = kQ * kb + 16 * piece;
        uint8_t *dst = lds + buf * STAGE + wave * COPIES * 1024;
        if (kQ * (kb + 1) <= p.K) {
#pragma unroll
            for (int i = 0; i < COPIES; ++i)
                __builtin_amdgcn_global_load_lds((const void *)(src[i] + k), (lds_void *)(dst + 1024 * i), 16, 0, 0);
        } else {
#pragma unroll
            for (int i = 0; i < COPIES; ++i)
                __builtin_amdgcn_global_load_lds((const void *)(k < p.K ? src[i] + k : kZeros),
                                                 (lds_void *)(dst + 1024 * i), 16, 0, 0);
        }
    };

    // scales: one of each token column, one (GateUp: two) of the wave's weight rows
    const float *xs[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
        int64_t t = row0 + min(wt * TW + 16 * j + c, rows - 1);
        if constexpr (M == Mode::GateUp) t = p.order[t] / p.top_k;
        xs[j] = p.xs + t * p.KB;
    }
    const float *ws0, *ws1;
    if constexpr (M == Mode::GateUp) {
        ws0 = sbase + (int64_t)nb * p.KB;
        ws1 = ws0 + (int64_t)n_tiles * p.KB;
    } else {
        ws0 = ws1 = sbase + (int64_t)min((n0 + wn * NW) / kQ, (p.N - 1) / kQ) * p.KB;
    }

    f32x4 acc[NI][NJ];
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[i][j] = (f32x4){0.f, 0.f, 0.f, 0.f};

    const int at = 16 * (g ^ (c & 7));   // place of piece g; piece g + 4 at the same ^ 64
    copy(0, 0);
    for (int kb = 0; kb < p.KB; ++kb) {
        float s0[NJ], s1[NJ];
        const float w0 = ws0[kb], w1 = ws1[kb];
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            const float v = xs[j][kb];
            s0[j] = v * w0;
            s1[j] = M == Mode::GateUp ? v * w1 : s0[j];
        }
        __builtin_amdgcn_s_waitcnt(wait_vm(0));
        __builtin_amdgcn_s_barrier();
        if (kb + 1 < p.KB) copy(kb + 1, (kb + 1) & 1);
        const uint8_t *wl = lds + (kb & 1) * STAGE + (wn * NW + c) * kQ;
        const uint8_t *xl = lds + (kb & 1) * STAGE + (BN + wt * TW + c) * kQ;
        i32x8 b[NJ];
#pragma unroll
        for (int j = 0; j < NJ; ++j)
            b[j] = pair(*(const u32x4 *)(xl + 16 * kQ * j + at), *(const u32x4 *)(xl + 16 * kQ * j + (at ^ 64)));
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const i32x8 a = pair(*(const u32x4 *)(wl + 16 * kQ * i + at), *(const u32x4 *)(wl + 16 * kQ * i + (at ^ 64)));
            f32x4 v[NJ];
#pragma unroll
            for (int j = 0; j < NJ; ++j) v[j] = mfma128<F32>(a, b[j]);
#pragma unroll
            for (int j = 0; j < NJ; ++j) acc[i][j] += v[j] * (i < NI / 2 ? s0[j] : s1[j]);
        }
    }

    if constexpr (M == Mode::GateUp) {
        float *peak = (float *)lds;   // [WN][BT]
        __builtin_amdgcn_s_barrier();   // the last step's reads are done
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            float m = 0.f;
#pragma unroll
            for (int i = 0; i < NI / 2; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float a = acc[i][j][r];
                    const float h = n0 + wn * (NW / 2) + 16 * i < p.N
                                        ? a / (1.f + expf(-a)) * acc[NI / 2 + i][j][r] : 0.f;
                    acc[i][j][r] = h;
                    m = fmaxf(m, fabsf(h));   // a NaN keeps out
                }
            m = fmaxf(m, __shfl_xor(m, 16));
            m = fmaxf(m, __shfl_xor(m, 32));
            if (g == 0) peak[wn * BT + wt * TW + 16 * j + c] = m;
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            const int r = wt * TW + 16 * j + c;
            if (r >= rows) continue;
            float m = peak[r];
#pragma unroll
            for (int v = 1; v < WN; ++v) m = fmaxf(m, peak[v * BT + r]);
            const float s = scale_of(m);
            const int64_t row = row0 + r;
            if (wn == 0 && g == 0) p.hs[row * n_tiles + nb] = s;
#pragma unroll
            for (int i = 0; i < NI / 2; ++i) {
                const int n = n0 + wn * (NW / 2) + 16 * i + 4 * g;
                const f32x4 h = acc[i][j];
                if (n < p.N)   // N a multiple of 16
                    *(uint32_t *)(p.hc + row * p.N + n) =
                        e4m3x2(h[0] / s, h[1] / s) | (e4m3x2(h[2] / s, h[3] / s) << 16);
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            const int r = wt * TW + 16 * j + c;
            if (r >= rows) continue;
            const int64_t t = M == Mode::Down ? p.order[row0 + r] : row0 + r;
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const int n = n0 + wn * NW + 16 * i + 4 * g;
                store4<F32>(p, t, n, acc[i][j]);
            }
        }
    }
}

template <Mode M, bool F32, int BN, int BT, int WN, int WT>
hipError_t launch_tiled(const ProductArgs &p, int t_tiles, hipStream_t st) {
    constexpr int bytes = 2 * (BN + BT) * kQ;
    const auto kernel = tiled_kernel<M, F32, BN, BT, WN, WT>;
    static std::atomic<uint64_t> ready{0};   // devices whose LDS limit is raised
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    if (dev >= 64 || !(ready.load() >> dev & 1)) {
        e = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e != hipSuccess) return e;
        if (dev < 64) ready.fetch_or(1ull << dev);
    }
    const int n_tiles = cdiv(p.N, M == Mode::GateUp ? BN / 2 : BN);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(n_tiles * t_tiles)), dim3(64 * WN * WT), bytes, st, p,
                       n_tiles, t_tiles);
    return hipSuccess;
}

}  // namespace fp8
}  // namespace echo
