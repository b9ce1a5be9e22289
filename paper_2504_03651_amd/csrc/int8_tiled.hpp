// int8_tiled.hpp -- products in 8-bit integers for many tokens: operand tiles in LDS.
#pragma once

#include "int8.hpp"

namespace echo {
namespace int8 {

// Where the units of a launch lie.  Workgroup b runs on XCD b % 8; each XCD takes a
// run of the units in the order (range of K, band of token tiles, tile of weights,
// tile of the band), so that the 32 that run on it at once are a block of about
// 8 x 4 tiles which share their operands in its L2.
struct Units {
    int n_tiles, t_tiles, ranges, band;   // band: token tiles of a band
    int all;
};

struct Place {
    int ni, ti, range;
};

__device__ __forceinline__ Place place_of(const Units &u, int i) {
    const int per = u.n_tiles * u.t_tiles;
    const int range = i / per;
    i -= range * per;
    const int full = u.n_tiles * u.band, b = i / full;
    i -= b * full;
    const int tall = min(u.band, u.t_tiles - b * u.band);
    const int ni = i / tall;
    return {ni, b * u.band + i - ni * tall, range};
}

// One workgroup of WN x WT waves: BN weight rows by BT tokens, K in steps of 128 bytes
// through a ring of S LDS stages that are filled straight from memory, S - 1 steps
// ahead.  A row's 128 codes are eight 16-byte pieces; piece q of row r lies at place
// q ^ (r & 7), so that the eight lanes that read one piece of eight rows meet eight
// different places.  Sums stay in the matrix instructions' accumulators to the end.
// No more workgroups are launched than run at once: each goes on to a next tile.
template <bool F32, bool ONCE, int BN, int BT, int WN, int WT, int S>
__global__ __launch_bounds__(64 * WN * WT, 1) void tiled_kernel(Product p, Units u) {
    constexpr int W = WN * WT, NW = BN / WN, TW = BT / WT;   // a wave's rows and tokens
    constexpr int NI = NW / 16, NJ = TW / 16;
    constexpr int STAGE = (BN + BT) * kStep;
    constexpr int PIECES = STAGE / 1024;                     // 1 KiB copies of a stage
    constexpr int COPIES = (PIECES + W - 1) / W, EXTRA = PIECES % W;
    // the epilogue: columns of a lane, lanes of a row, rows of a pass and their bytes, the
    // next one's four banks on
    constexpr int E = F32 ? 4 : 8, Q = NW / E, ROWS = Q < 4 ? 64 / Q : 16, PITCH = NW * 4 + 16;
    constexpr int SUMS = W * ROWS * PITCH;
    static_assert(!ONCE || BN / 8 % W == 0, "a copy is of weights in all waves or none");
    static_assert(NW % 16 == 0 && TW % ROWS == 0 && S >= 2 && SUMS <= S * STAGE);
    extern __shared__ __align__(16) uint8_t lds[];
    const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wn = wave % WN, wt = wave / WN;
    const bool more = EXTRA == 0 || wave < EXTRA;
    const int piece = (lane & 7) ^ (lane >> 3);

    const int xcd = blockIdx.x & 7, groups = (gridDim.x + 7 - xcd) / 8;
    const int end = (int)((int64_t)u.all * (xcd + 1) / 8);
    for (int unit = (int)((int64_t)u.all * xcd / 8) + (int)(blockIdx.x >> 3); unit < end; unit += groups) {
        const Place at_ = place_of(u, unit);
        const int n0 = BN * at_.ni, row0 = BT * at_.ti, rows = min(BT, p.T - row0);
        const int kb0 = (int)((int64_t)p.KB * at_.range / u.ranges);
        const int kb1 = (int)((int64_t)p.KB * (at_.range + 1) / u.ranges);
        const uint8_t *wsrc = p.w + (int64_t)n0 * p.K, *xsrc = p.x + (int64_t)row0 * p.K;
        uint32_t src[COPIES];   // this lane's bytes from the tile's weights or tokens
#pragma unroll
        for (int i = 0; i < COPIES; ++i) {
            const int r = min(8 * (W * i + wave), BN + BT - 8) + (lane >> 3);
            const int row = W * i + wave >= BN / 8 ? min(r - BN, rows - 1) : min(r, p.N - 1 - n0);
            src[i] = (uint32_t)row * (uint32_t)p.K + 16 * piece;
        }
        auto copy = [&](int kb, int slot) {
            uint8_t *dst = lds + slot * STAGE + 1024 * wave;
            const uint8_t *w = wsrc + (int64_t)kStep * kb, *x = xsrc + (int64_t)kStep * kb;
            const bool whole = kStep * (kb + 1) <= p.K, in = kStep * kb + 16 * piece < p.K;
#pragma unroll
            for (int i = 0; i < COPIES; ++i) {
                if (i + 1 == COPIES && !more) break;
                const uint8_t *from = (W * i + wave < BN / 8 ? w : x) + src[i];
                if (!(whole || in)) from = kZeros;
                lds_void *to = (lds_void *)(dst + 1024 * W * i);
                if (ONCE && W * i < BN / 8) __builtin_amdgcn_global_load_lds((const void *)from, to, 16, 0, 2);   // 2: nt
                else __builtin_amdgcn_global_load_lds((const void *)from, to, 16, 0, 0);
            }
        };
        constexpr int AHEAD = S - 2;   // stages that may be in flight behind the next one
        auto landed = [&](int kb) {
            if (kb + AHEAD >= kb1 || AHEAD == 0) landed_but<0>();
            else if (more) landed_but<AHEAD * COPIES>();
            else landed_but<AHEAD * (COPIES - 1)>();
        };
        i32x4 acc[NI][NJ];
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
            for (int j = 0; j < NJ; ++j) acc[i][j] = (i32x4){0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < S - 1; ++i)
            if (kb0 + i < kb1) copy(kb0 + i, i);
        const int at = 16 * (g ^ (c & 7));   // place of piece g; piece g + 4 at the same ^ 64
        int slot = 0;
        for (int kb = kb0; kb < kb1; ++kb) {
            landed(kb);
            if (kb + S - 1 < kb1) copy(kb + S - 1, slot == 0 ? S - 1 : slot - 1);
            if (WT == 1 || wt * TW < rows) {   // this wave has tokens
                const uint8_t *stage = lds + slot * STAGE;
                const uint8_t *wl = stage + (wn * NW + c) * kStep, *xl = stage + (BN + wt * TW + c) * kStep;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    u32x4 b[NJ];
#pragma unroll
                    for (int j = 0; j < NJ; ++j) b[j] = *(const u32x4 *)(xl + 16 * kStep * j + (at ^ (64 * h)));
#pragma unroll
                    for (int i = 0; i < NI; ++i) {
                        const u32x4 a = *(const u32x4 *)(wl + 16 * kStep * i + (at ^ (64 * h)));
#pragma unroll
                        for (int j = 0; j < NJ; ++j) acc[i][j] = mfma64(a, b[j], acc[i][j]);
                    }
                }
            }
            slot = slot + 1 == S ? 0 : slot + 1;
        }

        // Sums leave through LDS, ROWS tokens at a time, so that a store instruction
        // writes whole pieces of rows: the tile has them by columns, four of a row a lane.
        __syncthreads();   // the last step's reads are done
        if (u.ranges > 1) {
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                const int r = wt * TW + 16 * j + c;
                if (r >= rows) continue;
                int32_t *to = p.part + (at_.range * (int64_t)p.T + row0 + r) * p.part_pitch;
#pragma unroll
                for (int i = 0; i < NI; ++i) {
                    const int n = n0 + wn * NW + 16 * i + 4 * g;
                    if (n < p.part_pitch) *(i32x4 *)(to + n) = acc[i][j];
                }
            }
            continue;
        }
        uint8_t *mine = lds + wave * (ROWS * PITCH);
        const int q = lane % Q, n = n0 + wn * NW + E * q;
        Columns<E> cols;
        cols.load(p, n);
#pragma unroll
        for (int j0 = 0; j0 < NJ; j0 += ROWS / 16) {
#pragma unroll
            for (int j = 0; j < ROWS / 16; ++j)
#pragma unroll
                for (int i = 0; i < NI; ++i)
                    *(i32x4 *)(mine + (16 * j + c) * PITCH + (16 * i + 4 * g) * 4) = acc[i][j0 + j];
            wave_lds();
#pragma unroll
            for (int r0 = 0; r0 < ROWS; r0 += 64 / Q) {
                const int r = r0 + lane / Q, row = wt * TW + 16 * j0 + r;
                if (row >= rows || n >= p.N) continue;
                int sum[E];
#pragma unroll
                for (int e = 0; e < E; e += 4) {
                    const i32x4 s = *(const i32x4 *)(mine + r * PITCH + (E * q + e) * 4);
#pragma unroll
                    for (int k = 0; k < 4; ++k) sum[e + k] = s[k];
                }
                float v[E];
                cols.apply(p, sum, split(p.xs[row0 + row]), v);
                put<F32, E>(p, row0 + row, n, v);
            }
            wave_lds();
        }
        __syncthreads();   // the next tile's copies may land
    }
}

template <bool F32, bool ONCE, int BN, int BT, int WN, int WT, int S>
hipError_t launch_tiled(const Product &p, int ranges, hipStream_t st) {
    constexpr int bytes = S * (BN + BT) * kStep;
    static_assert(bytes <= 160 * 1024);
    static std::atomic<int> resident[64];
    Units u;
    u.n_tiles = cdiv(p.N, BN);
    u.t_tiles = cdiv(p.T, BT);
    u.ranges = ranges;
    u.band = cdiv(u.t_tiles, cdiv(u.t_tiles, 4));
    const int64_t all = (int64_t)u.n_tiles * u.t_tiles * ranges;
    u.all = (int)all;
    // workgroups beyond an XCD's units end at once
    return launch_lds(tiled_kernel<F32, ONCE, BN, BT, WN, WT, S>, resident, bytes, bytes, (all + 7) / 8 * 8, true,
                      64 * WN * WT, st, p, u);
}

}  // namespace int8
}  // namespace echo
