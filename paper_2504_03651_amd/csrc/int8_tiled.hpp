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

// All but the last `left` stages of C copies, N at most, of this wave have landed and
// its reads of LDS are done; then all waves'.
template <int N, int C>
__device__ __forceinline__ void landed_but_stages(int left) {
    if constexpr (N == 0) {
        landed_but<0>();
    } else {
        if (left >= N) landed_but<N * C>();
        else landed_but_stages<N - 1, C>(left);
    }
}

// Scales and bias of a tile in LDS, in whole copies of 64
constexpr int scale_room(int BN, int BT) { return (2 * BN + BT + 63) / 64 * 64; }

// LDS of a workgroup: two share a CU where it holds them
constexpr int lds_bytes(int BN, int BT, int S) { return S * (BN + BT) * kStep + 8 * scale_room(BN, BT); }

// One workgroup of WN x WT waves: BN weight rows by BT tokens, K in steps of 128
// through a ring of S LDS stages that are filled straight from memory.  A row's
// 16-byte pieces lie in an order that turns with the row, so that the lanes that read
// one piece of neighbouring rows meet different banks.  A step's operands are read into
// registers as the matrix instructions of the step before are done with theirs: a stage
// is free again as soon as it has been read, and S - 1 stages are under way.  Sums stay in
// the matrix instructions' accumulators to the end.
// No more workgroups are launched than run at once: each goes on to a next tile, whose
// first copies it starts before it writes the last one's results through one stage.
// 4,640 x 28672 x 4096 in tiles of 256 x 192 takes 532 us, 2.05 PetaOp/s (a library's
// product of 8,192^3: 2.02): copies alone 374, products with their reads of LDS alone 345,
// everything but the results 460.  Matrix instructions are busy 51% of the time at the
// 1.97 GHz that the card then holds, three in four requests of the copies hit an XCD's
// L2, LDS reads have no conflicts.  137 x 4096 x 14336, tiles of 128 x 160 in six ranges
// of K: 20.7 us, 2.8 TB/s of weights, behind its copies.  What was tried: a step's copies
// asked for at once, ahead of its products, hold the waves up (two stages of 256 x 256:
// 548 us and more); rows of 64 bytes halve what a request of the L2 brings (copies of 13
// TB/s in the place of 20); instructions of 32 x 32 x 32 (products alone 12% slower); four
// waves of 128 x 128 spill; workgroups that start apart, so that one's results meet others'
// products, 3% at best.
template <bool F32, bool ONCE, int BN, int BT, int WN, int WT, int S>
__global__ __launch_bounds__(64 * WN * WT, WN * WT * (2 * lds_bytes(BN, BT, S) <= 160 * 1024 ? 2 : 1) / 4) void tiled_kernel(Product p, Units u) {
    constexpr int W = WN * WT, NW = BN / WN, TW = BT / WT;   // a wave's rows and tokens
    constexpr int NI = NW / 16, NJ = TW / 16, NH = kStep / 64;
    constexpr int STAGE = (BN + BT) * kStep;
    constexpr int PIECES = STAGE / 1024;                     // 1 KiB copies of a stage
    constexpr int COPIES = (PIECES + W - 1) / W, EXTRA = PIECES % W;
    constexpr int RC = 1024 / kStep, PR = kStep / 16;        // rows of a copy, pieces of a row
    // the epilogue: sums of ROWS tokens and CP columns of each wave at a time; E columns
    // and Q lanes of a row
    constexpr int E = F32 ? 4 : 8, ROOM = STAGE / W;
    constexpr int CP = NW % 64 == 0 && ROOM >= 4096 ? 64 : NW % 32 == 0 ? 32 : 16;
    // ranges of K, and a residual that is asked for early: where registers allow it
    constexpr bool CUTS = BN * BT <= 128 * 256;
    constexpr bool REST = BN * BT * (F32 ? 2 : 1) <= 128 * 256 && (W <= 4 || 2 * lds_bytes(BN, BT, S) > 160 * 1024);
    constexpr int Q = CP / E, ROWS = Q < 4 ? 64 / Q : 16, CHUNKS = CP / 4;
    static_assert(!ONCE || BN / RC % W == 0, "a copy is of weights in all waves or none");
    static_assert(STAGE % 1024 == 0 && BN % RC == 0 && NW % CP == 0 && TW % ROWS == 0 && S >= 2);
    static_assert(ROWS * CP * 4 <= ROOM && (ROOM % 16) == 0);
    extern __shared__ __align__(16) uint8_t lds[];
    const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wn = wave % WN, wt = wave / WN;
    const bool more = EXTRA == 0 || wave < EXTRA;
    // the place of piece q of row r: rows whose places start at the same bank differ
    auto turn = [](int r) { return r & (PR - 1); };
    const int piece = (lane % PR) ^ turn(lane / PR);

    const int xcd = blockIdx.x & 7, groups = (gridDim.x + 7 - xcd) / 8;
    const int end = (int)((int64_t)u.all * (xcd + 1) / 8);
    int unit = (int)((int64_t)u.all * xcd / 8) + (int)(blockIdx.x >> 3);
    if (unit >= end) return;

    int n0, row0, rows, range, kb0, kb1;
    const uint8_t *wsrc, *xsrc;
    uint32_t src[COPIES];   // this lane's bytes from the tile's weights or tokens
    auto take = [&](int unit) {
        const Place at = place_of(u, unit);
        range = at.range;
        n0 = BN * at.ni;
        row0 = BT * at.ti;
        rows = min(BT, p.T - row0);
        kb0 = (int)((int64_t)p.KB * range / u.ranges);
        kb1 = (int)((int64_t)p.KB * (range + 1) / u.ranges);
        wsrc = p.w + (int64_t)n0 * p.K;
        xsrc = p.x + (int64_t)row0 * p.K;
#pragma unroll
        for (int i = 0; i < COPIES; ++i) {
            const int r = min(RC * (W * i + wave), BN + BT - RC) + lane / PR;
            const int row = W * i + wave >= BN / RC ? min(r - BN, rows - 1) : min(r, p.N - 1 - n0);
            src[i] = (uint32_t)row * (uint32_t)p.K + 16 * piece;
        }
    };
    // copy i of stage kb: a wave's own 1 KiB of it
    auto copy = [&](int kb, int slot, int i) {
        if (i + 1 == COPIES && !more) return;
        const bool in = kStep * (kb + 1) <= p.K || kStep * kb + 16 * piece < p.K;
        const uint8_t *from = (W * i + wave < BN / RC ? wsrc : xsrc) + (int64_t)kStep * kb + src[i];
        if (!in) from = kZeros;
        lds_void *to = (lds_void *)(lds + slot * STAGE + 1024 * (W * i + wave));
        if (ONCE && W * i < BN / RC) __builtin_amdgcn_global_load_lds((const void *)from, to, 16, 0, 2);   // 2: nt
        else __builtin_amdgcn_global_load_lds((const void *)from, to, 16, 0, 0);
    };
    auto copies = [&](int kb, int slot) {
#pragma unroll
        for (int i = 0; i < COPIES; ++i) copy(kb, slot, i);
    };
    // The scales of a tile's rows and tokens and its bias go to LDS ahead of its first
    // stage, so that nothing that is loaded stands between the results' stores.  Two
    // tiles take turns.
    constexpr int SCALES = scale_room(BN, BT), SCALE_COPIES = (SCALES + 64 * W - 1) / (64 * W);
    static_assert(BN % 64 == 0, "a copy is of one kind");
    int side = 0;
    auto copy_scales = [&] {
        float *to = (float *)(lds + S * STAGE) + side * SCALES;
#pragma unroll
        for (int i = 0; i < SCALE_COPIES; ++i) {
            const int at = 64 * (W * i + wave), e = at + lane;   // weights' scales, bias, tokens' scales
            if (at >= SCALES) break;
            const float *from = e < BN       ? p.ws + min(n0 + e, p.N - 1)
                                : e < 2 * BN ? (p.bias ? p.bias : p.ws) + min(n0 + e - BN, p.N - 1)
                                             : p.xs + row0 + min(e - 2 * BN, rows - 1);
            __builtin_amdgcn_global_load_lds((const void *)from, (lds_void *)(to + at), 4, 0, 0);
        }
    };
    auto next = [](int slot) { return slot + 1 == S ? 0 : slot + 1; };
    // Stage kb has landed and all waves have read the one before.  What a wave has
    // asked for behind it may be under way: S - 2 stages, fewer at the end.
    auto landed = [&](int kb) {
        if (more) landed_but_stages<S - 2, COPIES>(kb1 - 1 - kb);
        else landed_but_stages<S - 2, COPIES - 1>(kb1 - 1 - kb);
    };
    int at[NH];   // places of this lane's pieces
#pragma unroll
    for (int h = 0; h < NH; ++h) at[h] = 16 * ((g + 4 * h) ^ turn(c));
    u32x4 x[NJ], w[NI];   // the operands of 64 of K
    i32x4 acc[NI][NJ];
    auto read_x = [&](int slot, int h, int j) {
        return *(const u32x4 *)(lds + slot * STAGE + (BN + wt * TW + 16 * j + c) * kStep + at[h]);
    };
    auto read_w = [&](int slot, int h, int i) {
        return *(const u32x4 *)(lds + slot * STAGE + (wn * NW + 16 * i + c) * kStep + at[h]);
    };

    int slot = 0;   // of the tile's first stage, then of the last one read
    auto start = [&] {
        copy_scales();
        int s = slot;
#pragma unroll
        for (int i = 0; i < S - 1; ++i, s = next(s))
            if (kb0 + i < kb1) copies(kb0 + i, s);
    };
    take(unit);
    start();
    while (true) {
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
            for (int j = 0; j < NJ; ++j) acc[i][j] = (i32x4){0, 0, 0, 0};
        const bool busy = WT == 1 || wt * TW < rows;   // this wave has tokens
        landed(kb0);
        if (kb0 + S - 1 < kb1) copies(kb0 + S - 1, slot == 0 ? S - 1 : slot - 1);
        if (busy) {
#pragma unroll
            for (int j = 0; j < NJ; ++j) x[j] = read_x(slot, 0, j);
#pragma unroll
            for (int i = 0; i < NI; ++i) w[i] = read_w(slot, 0, i);
        }
        for (int kb = kb0; kb < kb1; ++kb) {
#pragma unroll
            for (int h = 0; h < NH; ++h) {
                // the next 64 of K: of this stage, or of the next one (behind the last, of
                // that one again), which frees this one for a copy
                const int now = slot, ahead = kb + S;
                const bool last = h + 1 == NH, more_k = last && ahead < kb1;
                if (last && kb + 1 < kb1) {
                    landed(kb + 1);
                    slot = next(slot);
                }
                if (busy) {
                    u32x4 then[NJ];
#pragma unroll
                    for (int j = 0; j < NJ; ++j) then[j] = read_x(slot, (h + 1) % NH, j);
#pragma unroll
                    for (int i = 0; i < NI; ++i) {
#pragma unroll
                        for (int j = 0; j < NJ; ++j) acc[i][j] = mfma64(w[i], x[j], acc[i][j]);
                        w[i] = read_w(slot, (h + 1) % NH, i);
                        // copies stand between the products: asked for at once they would hold
                        // the wave up until the last of them is taken
#pragma unroll
                        for (int k = i * COPIES / NI; k < (i + 1) * COPIES / NI; ++k)
                            if (more_k) copy(ahead, now, k);
                        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);            // LDS reads
                        __builtin_amdgcn_sched_group_barrier(0x008, NJ / 2, 0);       // matrix instructions
                        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                        __builtin_amdgcn_sched_group_barrier(0x008, NJ - NJ / 2, 0);
                        __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);            // copies
                    }
#pragma unroll
                    for (int j = 0; j < NJ; ++j) x[j] = then[j];
                } else if (more_k) {
                    copies(ahead, now);
                }
            }
        }

        // The residual is asked for ahead of the next tile's copies and of all stores, which
        // it would wait for: memory answers in order.
        constexpr int PARTS = NI / (CP / 16), READS = TW / (64 / Q);   // of a wave's columns, of its rows
        Rest<F32, E> rest[REST ? PARTS : 1][REST ? READS : 1];
        const bool early = REST && p.residual && u.ranges == 1 && busy;
        if (early) {
#pragma unroll
            for (int i = 0; i < (REST ? PARTS : 1); ++i)
#pragma unroll
                for (int k = 0; k < (REST ? READS : 1); ++k) {
                    const int row = wt * TW + k * (64 / Q) + lane / Q, n = n0 + wn * NW + CP * i + E * (lane % Q);
                    if (row < rows && n < p.N) rest[i][k].load(p, (row0 + row) * p.y_stride + n, n);
                }
        }

        // the next unit's first stages go to the slots behind the one that the epilogue
        // takes, the last one read
        const int n0_ = n0, row0_ = row0, rows_ = rows, range_ = range;
        const float *scales = (const float *)(lds + S * STAGE) + side * SCALES;
        side ^= 1;
        uint8_t *free = lds + slot * STAGE;
        unit += groups;
        const bool again = unit < end;
        landed_but<0>();   // all waves have read the last stage
        slot = next(slot);
        if (again) {
            take(unit);
            start();
        }
        if (busy) {
            // Sums leave through LDS, so that a store instruction writes whole pieces of rows:
            // the tile has them by columns, four of a row a lane.  A row's 16-byte chunks
            // lie in an order that turns with the row.
            uint8_t *mine = free + wave * ROOM;
            const int q = lane % Q;
#pragma unroll
            for (int i0 = 0; i0 < NI; i0 += CP / 16) {
                const int col = wn * NW + 16 * i0 + E * q, n = n0_ + col;
                int32_t *part = p.part + (range_ * (int64_t)p.T + row0_) * p.part_pitch + n;
                Columns<E> cols;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    cols.w[e] = split(scales[col + e]);
                    cols.bias[e] = scales[BN + col + e];
                }
#pragma unroll
                for (int j0 = 0; j0 < NJ; j0 += ROWS / 16) {
#pragma unroll
                    for (int j = 0; j < ROWS / 16; ++j)
#pragma unroll
                        for (int i = 0; i < CP / 16; ++i)
                            *(i32x4 *)(mine + (16 * j + c) * (CP * 4) + 16 * ((4 * i + g) ^ (c & (CHUNKS - 1)))) =
                                acc[i0 + i][j0 + j];
                    wave_lds();
#pragma unroll
                    for (int r0 = 0; r0 < ROWS; r0 += 64 / Q) {
                        const int r = r0 + lane / Q, row = wt * TW + 16 * j0 + r;
                        int sum[E];
#pragma unroll
                        for (int e = 0; e < E; e += 4) {
                            const i32x4 s = *(const i32x4 *)(mine + r * (CP * 4) +
                                                             16 * ((E / 4 * q + e / 4) ^ (r & 15 & (CHUNKS - 1))));
#pragma unroll
                            for (int k = 0; k < 4; ++k) sum[e + k] = s[k];
                        }
                        if (CUTS && u.ranges > 1) {
#pragma unroll
                            for (int e = 0; e < E; e += 4)
                                if (row < rows_ && n + e < p.part_pitch)
                                    *(i32x4 *)(part + row * (int64_t)p.part_pitch + e) =
                                        (i32x4){sum[e], sum[e + 1], sum[e + 2], sum[e + 3]};
                            continue;
                        }
                        float v[E];
                        cols.apply(p, sum, split(scales[2 * BN + row]), v);
                        if (row >= rows_ || n >= p.N) continue;
                        if constexpr (REST) {
                            if (early) rest[i0 / (CP / 16)][(16 * j0 + r0) / (64 / Q)].add(v);
                            put<F32, E>(p, row0_ + row, n, v);
                        } else {
                            put_sum<F32, E, !CUTS>(p, row0_ + row, n, v);
                        }
                    }
                    wave_lds();
                }
            }
        }
        if (!again) break;
    }
}

template <bool F32, bool ONCE, int BN, int BT, int WN, int WT, int S>
hipError_t launch_tiled(const Product &p, int ranges, hipStream_t st) {
    constexpr int bytes = lds_bytes(BN, BT, S);
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
