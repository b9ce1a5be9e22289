// fp8_tiled.hpp -- e4m3 products for many tokens: operand tiles in LDS.
#pragma once

#include <algorithm>
#include <atomic>

#include "fp8.hpp"

namespace echo {
namespace fp8 {

typedef __attribute__((address_space(3))) void lds_void;

// where 16-byte pieces past the end of a row come from
__device__ __align__(16) const uint8_t kZeros[16] = {};

// All but the last n of this wave's copies into LDS have landed and its reads of
// LDS are done; then all waves'.
template <int N>
__device__ __forceinline__ void landed_but() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// What a tile's workgroup does with its sums.  Results of 16 bits and codes go
// through LDS, so that a store instruction writes whole pieces of rows: the tile
// has them by columns, four values of a row a lane.
// Uses at most ROOM bytes of LDS, in PASSES where the whole tile needs more.
// An expert's outputs (Down) keep 11 bits in fp16 under an exponent of their own for
// each row's NW columns: no more than 2^-11 of the value off, or 2^-39 of the
// largest of those columns, at half the bytes of fp32.
template <Mode M, bool F32, int BN, int BT, int WN, int WT, int ROOM>
__device__ __forceinline__ void finish(const ProductArgs &p, uint8_t *lds,
                                       f32x4 (&acc)[BN / WN / 16][BT / WT / 16],
                                       const int (&to)[BT / WT / 16], int n_tiles, int nb,
                                       int n0, int row0, int rows, int splits, int split) {
    constexpr int NW = BN / WN, TW = BT / WT, NI = NW / 16, NJ = TW / 16;
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));   // addresses are computed here, not kept over the steps
    const int g = lane >> 4, c = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wn = wave % WN, wt = wave / WN;
    if constexpr (M == Mode::GateUp) {
        static_assert(BT * (kQ + 4 * WN) <= ROOM);
        float *peak = (float *)(lds + BT * kQ);   // [WN][BT]
        __syncthreads();   // the last step's reads are done
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            float m = 0.f;
#pragma unroll
            for (int i = 0; i < NI / 2; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    // a / (1 + e^-a) u; columns past N repeat the last one.  The
                    // exponential is |a| 2^-24 off, the reciprocal 2^-23: no
                    // more than the sums behind a, under codes of 2^-4.
                    const float a = acc[i][j][r];
                    const float h = a * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504f * a)) *
                                    acc[NI / 2 + i][j][r];
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
            float m = peak[r];
#pragma unroll
            for (int v = 1; v < WN; ++v) m = fmaxf(m, peak[v * BT + r]);
            const float s = scale_of(m);
            if (wn == 0 && g == 0 && r < rows) p.hs[(int64_t)(row0 + r) * n_tiles + nb] = s;
            // h / s by the reciprocal: at most 448 (1 + 2^-21), which rounds to 448,
            // but for scales below 2^-126, which are coarser than that
            float inv = __builtin_amdgcn_rcpf(s);
            if (s < 0x1p-100f) {
                inv = 1.f / (s * 0x1p64f);
#pragma unroll
                for (int i = 0; i < NI / 2; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float h = acc[i][j][e] * 0x1p64f * inv;
                        acc[i][j][e] = h > 448.f ? 448.f : h < -448.f ? -448.f : h;
                    }
                inv = 1.f;
            }
#pragma unroll
            for (int i = 0; i < NI / 2; ++i) {
                const f32x4 h = acc[i][j] * inv;
                // 16-byte piece q of row r at place q ^ (r & 7)
                const int at = wn * (NW / 2) + 16 * i + 4 * g;
                *(uint32_t *)(lds + r * kQ + 16 * ((at >> 4) ^ (r & 7)) + (at & 15)) =
                    __builtin_amdgcn_cvt_pk_fp8_f32(
                        h[2], h[3], __builtin_amdgcn_cvt_pk_fp8_f32(h[0], h[1], 0, false), true);
            }
        }
        __syncthreads();
        for (int e = threadIdx.x; e < 8 * rows; e += 64 * WN * WT) {
            const int r = e >> 3, q = e & 7;
            if (n0 + 16 * q < p.N)   // N a multiple of 16
                *(u32x4 *)(p.hc + (int64_t)(row0 + r) * p.N + n0 + 16 * q) =
                    *(const u32x4 *)(lds + r * kQ + 16 * (q ^ (r & 7)));
        }
    } else if (splits > 1 || F32) {
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            const int r = wt * TW + 16 * j + c;
            if (r >= rows) continue;
            const int64_t t = row0 + r;
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const int n = n0 + wn * NW + 16 * i + 4 * g;
                if (splits > 1) {
                    if (n < p.part_pitch)
                        *(f32x4 *)(p.part + (split * (int64_t)p.T + t) * p.part_pitch + n) = acc[i][j];
                } else {
                    store4<F32>(p, t, n, acc[i][j]);
                }
            }
        }
    } else {
        constexpr int Q = NW / 8;   // 16-byte pieces of a row of this wave
        constexpr int PASSES = (BN * BT * 2 + ROOM - 1) / ROOM, TP = TW / PASSES;
        static_assert(TP % 16 == 0 && TP * PASSES == TW);
        uint8_t *mine = lds + wave * (NW * TP * 2);
        __syncthreads();   // the last step's reads are done
#pragma unroll
        for (int pass = 0; pass < PASSES; ++pass) {
            const int t0 = wt * TW + pass * TP;   // the pass's first row
#pragma unroll
            for (int j = 0; j < TP / 16; ++j) {
                const int r = 16 * j + c;
                const bool live = t0 + r < rows;
                int up = 0;
                if constexpr (M == Mode::Down) {
                    float m = 0.f;
#pragma unroll
                    for (int i = 0; i < NI; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float a = fabsf(acc[i][pass * (TP / 16) + j][e]);
                            m = fmaxf(m, a < INFINITY ? a : 0.f);   // not a NaN either
                        }
                    m = fmaxf(m, __shfl_xor(m, 16));
                    m = fmaxf(m, __shfl_xor(m, 32));
                    up = min(15 - __builtin_amdgcn_frexp_expf(m), 127);   // m 2^up below 2^15
                    if (live && g == 0 && n0 + wn * NW < p.N)
                        p.ye[to[pass * (TP / 16) + j] * (int64_t)p.y_groups + (n0 + wn * NW) / NW] = (int8_t)-up;
                }
#pragma unroll
                for (int i = 0; i < NI; ++i) {
                    f32x4 v = acc[i][pass * (TP / 16) + j];
                    const int n = 16 * i + 4 * g;
                    if (M == Mode::Plain && p.residual && live)
                        v = plus_residual<false>(p, (row0 + t0 + r) * p.y_stride + n0 + wn * NW + n,
                                                 n0 + wn * NW + n, v);
                    u32x2 two;
                    if constexpr (M == Mode::Down) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[e] = __builtin_amdgcn_ldexpf(v[e], up);
                        two = (u32x2){f2h2(v[0], v[1]), f2h2(v[2], v[3])};
                    } else {
                        two = (u32x2){f2bf2(v[0], v[1]), f2bf2(v[2], v[3])};
                    }
                    *(u32x2 *)(mine + (r * Q + ((n >> 3) ^ (r & (Q - 1)))) * 16 + (n & 4) * 2) = two;
                }
            }
            wave_lds();
            const int q = lane % Q, n = n0 + wn * NW + 8 * q;
#pragma unroll
            for (int r0 = 0; r0 < TP; r0 += 64 / Q) {
                const int r = r0 + lane / Q, row = t0 + r;
                // sixteen rows of one j at most, but for waves of sixteen rows in all
                static_assert(M != Mode::Down || 64 / Q <= 16 || TW == 16);
                int64_t t = row0 + row;
                if constexpr (M == Mode::Down) t = __shfl(to[(pass * TP + r0) / 16], r & 15);
                if (row >= rows || n >= p.N) continue;
                const u32x4 *from = (const u32x4 *)(mine + (r * Q + (q ^ (r & (Q - 1)))) * 16);
                uint16_t *y = (uint16_t *)p.y + t * p.y_stride + n;
                if (M == Mode::Down) *(u32x4 *)y = *from;   // N a multiple of 16
                else if (n + 8 <= p.N) *(any_u32x4 *)y = *from;
                else
                    for (int e = 0; e < p.N - n; ++e) y[e] = ((const uint16_t *)from)[e];
            }
            if (pass + 1 < PASSES) wave_lds();
        }
    }
}

// One workgroup of WN x WT waves: BN weight rows (GateUp: BN / 2 gate rows and
// the up rows of the same columns) by BT tokens, K in steps of 128 through a ring
// of S LDS stages that are filled straight from memory, S - 1 steps ahead.  A
// row's 128 codes are eight 16-byte pieces; piece q of row r lies at place
// q ^ (r & 7), so that the eight lanes that read one piece of eight rows meet
// eight different places.  Behind a stage's codes lie each wave's scales: one of
// each of its tokens, and one (GateUp: two) of its weight rows.  Each step's sum
// comes out of the matrix instruction alone and is scaled on its way into the
// accumulators, one FMA a value.
// Bound by the copies into LDS: 4,640 x 28672 x 4096 takes 600 us, 1.82 PFLOP/s, its
// copies alone 484 (9.2 TB/s over all CUs), all the rest without them 407; 137 x 4096 x
// 14336 34, 32 and 29; 4,640 tokens through 64 experts of 2048 x 1024 497, 401 and 387.
// A step of 256 x 256 copies 64 KB in 1.9 us, one of 256 x 128 48 KB in 1.3.  Matrix
// instructions are busy 39% of the first one's time, vector instructions 35%, LDS 18%,
// with no conflicts in the steps.  Waves of 128 x 64 are the largest whose sums fit
// the registers that FMAs reach.
// No more workgroups are launched than run at once: each goes on to a next tile,
// whose first copies it starts before it writes the last one's results (4,640 tokens
// through 64 experts 509 -> 497 us).
// ONCE: weights past the caches, where one tile of tokens reads them (8 tokens
// through 64 experts of 2048 x 1024 65.7 -> 60.2 us, 64 tokens 93 -> 84; 64 x 28672
// x 4096 35.2 -> 33; but two tiles of 64, 100 x 4096 x 4096: 15.5 -> 16.3).
// F32: products are exact (mfma128), and Plain's results fp32.
// part: fp32 sums of one of `splits` equal ranges of K go to part[split][t][n],
// rows part_pitch apart, instead of y.
template <Mode M, bool F32, bool ONCE, int BN, int BT, int WN, int WT, int S>
__global__ __launch_bounds__(64 * WN * WT, 512 / (64 * WN * WT)) void tiled_kernel(ProductArgs p, int n_tiles, int t_tiles, int splits) {
    constexpr int W = WN * WT, NW = BN / WN, TW = BT / WT;   // a wave's rows and tokens
    constexpr int NI = NW / 16, NJ = TW / 16;
    constexpr int CODES = (BN + BT) * kQ, STAGE = CODES + 512 * W;
    constexpr int PIECES = CODES / 1024;                     // 1 KiB copies of a stage
    constexpr int COPIES = (PIECES + W - 1) / W, EXTRA = PIECES % W;
    static_assert(!ONCE || BN / 8 % W == 0, "a copy is of weights in all waves or none");
    static_assert(NW % (M == Mode::GateUp ? 32 : 16) == 0 && TW % 16 == 0 && TW <= 64 && S >= 2);
    extern __shared__ __align__(16) uint8_t lds[];
    const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wn = wave % WN, wt = wave / WN;

    // copies of a wave: COPIES, or one less where the stage's pieces run out
    const bool more = EXTRA == 0 || wave < EXTRA;
    const int piece = (lane & 7) ^ (lane >> 3);
    const int units = (M == Mode::Plain ? t_tiles : *p.num_tiles) * n_tiles * splits;
    // The unit of work: rows n0 .. of the weights by rows row0 .. of the tokens,
    // steps kb0 to kb1; and the sources of this lane's copies, in bytes from the
    // tile's weights (rows of the stage below BN) and from its tokens.
    int split, nb, n0, row0, rows, kb0, kb1;
    const uint8_t *wsrc, *xsrc;
    const float *xscale, *ws;   // ws: lanes below 32 the (gate) rows' scales, above the up rows'
    uint32_t src[COPIES], xs;
    auto take = [&](int b) {
        int lane = threadIdx.x & 63;
        asm volatile("" : "+v"(lane));   // computed here, not kept over the steps
        const int piece = (lane & 7) ^ (lane >> 3);
        split = b % splits;
        b /= splits;
        const int ti = b / n_tiles;
        nb = b - ti * n_tiles;
        n0 = (M == Mode::GateUp ? BN / 2 : BN) * nb;
        kb0 = (int)((int64_t)p.KB * split / splits);
        kb1 = (int)((int64_t)p.KB * (split + 1) / splits);
        wsrc = p.w;
        const float *sbase = p.ws;
        if constexpr (M == Mode::Plain) {
            row0 = BT * ti;
            rows = min(BT, p.T - row0);
        } else {
            const Tile t = p.tiles[ti];
            row0 = t.row0;
            rows = t.rows;
            wsrc += t.expert * p.w_expert;
            sbase += t.expert * p.ws_expert;
        }
        xsrc = p.x;
        xscale = p.xs;
        if constexpr (M != Mode::GateUp) {
            wsrc += (int64_t)n0 * p.K;
            xsrc += (int64_t)row0 * p.K;
            xscale += (int64_t)row0 * p.KB;
        }
        auto token = [&](int r) -> uint32_t {   // row of x that the tile's row r reads
            r = min(r, rows - 1);
            return M == Mode::GateUp ? (uint32_t)p.order[row0 + r] / (uint32_t)p.top_k : (uint32_t)r;
        };
#pragma unroll
        for (int i = 0; i < COPIES; ++i) {
            const int r = min(8 * (W * i + wave), BN + BT - 8) + (lane >> 3);
            uint32_t row;
            if (W * i + wave >= BN / 8) {
                row = token(r - BN);
            } else if constexpr (M == Mode::GateUp) {
                const int q = r % NW, n = min(n0 + (r / NW) * (NW / 2) + q % (NW / 2), p.N - 1);
                row = q < NW / 2 ? n : p.N + n;
            } else {
                row = min(r, p.N - 1 - n0);
            }
            src[i] = row * (uint32_t)p.K + 16 * piece;
        }
        xs = token(wt * TW + lane % TW) * (uint32_t)p.KB;
        if constexpr (M == Mode::GateUp) ws = sbase + (int64_t)(lane < 32 ? nb : n_tiles + nb) * p.KB;
        else ws = sbase + (int64_t)min((n0 + wn * NW) / kQ, (p.N - 1) / kQ) * p.KB;
    };
    auto copy = [&](int kb, int slot) {
        uint8_t *stage = lds + slot * STAGE, *dst = stage + 1024 * wave;
        const uint8_t *w = wsrc + (int64_t)kQ * kb, *x = xsrc + (int64_t)kQ * kb;
        const bool whole = kQ * (kb + 1) <= p.K, in = kQ * kb + 16 * piece < p.K;
#pragma unroll
        for (int i = 0; i < COPIES; ++i) {
            if (i + 1 == COPIES && !more) break;
            const uint8_t *from = (W * i + wave < BN / 8 ? w : x) + src[i];
            if (!(whole || in)) from = kZeros;
            lds_void *to = (lds_void *)(dst + 1024 * W * i);
            if (ONCE && W * i < BN / 8) __builtin_amdgcn_global_load_lds((const void *)from, to, 16, 0, 2);   // 2: nt
            else __builtin_amdgcn_global_load_lds((const void *)from, to, 16, 0, 0);
        }
        float *sc = (float *)(stage + CODES) + 128 * wave;
        __builtin_amdgcn_global_load_lds((const void *)(xscale + kb + xs), (lds_void *)sc, 4, 0, 0);
        __builtin_amdgcn_global_load_lds((const void *)(ws + kb), (lds_void *)(sc + 64), 4, 0, 0);
    };
    constexpr int AHEAD = S - 2;   // stages that may be in flight behind the next one
    auto landed = [&](int kb) {
        if (kb + AHEAD >= kb1 || AHEAD == 0) landed_but<0>();
        else if (more) landed_but<AHEAD * (COPIES + 2)>();
        else landed_but<AHEAD * (COPIES + 1)>();
    };

    const int at = 16 * (g ^ (c & 7));   // place of piece g; piece g + 4 at the same ^ 64
    int slot = 0;
    auto start = [&] {
#pragma unroll
        for (int i = 0; i < S - 1; ++i)
            if (kb0 + i < kb1) copy(kb0 + i, slot + i < S ? slot + i : slot + i - S);
    };
    int unit = blockIdx.x;
    if (unit >= units) return;
    take(unit);
    start();
    while (true) {
        f32x4 acc[NI][NJ];
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
            for (int j = 0; j < NJ; ++j) acc[i][j] = (f32x4){0.f, 0.f, 0.f, 0.f};
        int to[NJ] = {};   // Down: the pairs of this lane's rows
        if constexpr (M == Mode::Down)
#pragma unroll
            for (int j = 0; j < NJ; ++j) to[j] = p.order[row0 + min(wt * TW + 16 * j + c, rows - 1)];
        uint32_t least = kOddClass;   // of the scales that this lane's sums took
        for (int kb = kb0; kb < kb1; ++kb) {
            landed(kb);
            const int free = slot == 0 ? S - 1 : slot - 1;
            if (kb + S - 1 < kb1) copy(kb + S - 1, free);
            if (WT == 1 || wt * TW < rows) {   // this wave has tokens
                const uint8_t *stage = lds + slot * STAGE;
                const uint8_t *wl = stage + (wn * NW + c) * kQ, *xl = stage + (BN + wt * TW + c) * kQ;
                auto read = [&](const uint8_t *l, int i) {
                    l += 16 * kQ * i;
                    return pair(*(const u32x4 *)(l + at), *(const u32x4 *)(l + (at ^ 64)));
                };
                const float *sc = (const float *)(stage + CODES) + 128 * wave;
                float s[NJ];
                auto scales = [&](int at) {
#pragma unroll
                    for (int j = 0; j < NJ; ++j) {
                        s[j] = sc[16 * j + c] * sc[at];
                        least = min(least, scale_class(s[j]));
                    }
                };
                scales(64);
                // weight rows are read one tile ahead of their products
                i32x8 b[NJ], a = read(wl, 0);
#pragma unroll
                for (int j = 0; j < NJ; ++j) b[j] = read(xl, j);
#pragma unroll
                for (int i = 0; i < NI; ++i) {
                    const i32x8 a2 = read(wl, i + 1 < NI ? i + 1 : i);
                    if (M == Mode::GateUp && i == NI / 2) scales(96);   // on to the up rows
                    f32x4 v[NJ];
#pragma unroll
                    for (int j = 0; j < NJ; ++j) v[j] = mfma128<F32>(a, b[j]);
#pragma unroll
                    for (int j = 0; j < NJ; ++j) acc[i][j] += v[j] * s[j];
                    a = a2;
                }
            }
            slot = slot + 1 == S ? 0 : slot + 1;
        }
        if (__any(least < kOddClass)) {
            // Some were no normal numbers: the wave takes its sums again, straight from
            // memory, a matrix instruction at a time.
#pragma unroll
            for (int i = 0; i < NI; ++i) {
#pragma unroll
                for (int j = 0; j < NJ; ++j) {
                    int lane = threadIdx.x & 63;
                    asm volatile("" : "+v"(lane));   // addresses live for their products only
                    const int g = lane >> 4, c = lane & 15;
                    int n = wn * NW + 16 * i + c, r = min(wt * TW + 16 * j + c, rows - 1);
                    const float *sw = ws;
                    if constexpr (M == Mode::GateUp) {
                        const bool up = i >= NI / 2;
                        n = min(n0 + wn * (NW / 2) + 16 * (i % (NI / 2)) + c, p.N - 1) + (up ? p.N : 0);
                        r = p.order[row0 + r] / p.top_k;
                        if (up && lane < 32) sw += (int64_t)n_tiles * p.KB;
                        if (!up && lane >= 32) sw -= (int64_t)n_tiles * p.KB;
                    } else {
                        n = min(n, p.N - 1 - n0);
                    }
                    const uint8_t *w = wsrc + (int64_t)n * p.K, *x = xsrc + (int64_t)r * p.K;
                    const float *sx = xscale + (int64_t)r * p.KB;
                    f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
                    for (int kb = kb0; kb < kb1; ++kb) {
                        const int64_t at = (int64_t)kQ * kb + 16 * g;
                        u32x4 a[2], b[2];
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const bool in = at + 64 * h < p.K;
                            a[h] = in ? *(const u32x4 *)(w + at + 64 * h) : (u32x4){0u, 0u, 0u, 0u};
                            b[h] = in ? *(const u32x4 *)(x + at + 64 * h) : (u32x4){0u, 0u, 0u, 0u};
                        }
                        v += scaled(mfma128<F32>(pair(a[0], a[1]), pair(b[0], b[1])), sx[kb], sw[kb]);
                    }
                    acc[i][j] = v;
                }
            }
        }

        // the next unit's first steps go to the stages that the last step left free,
        // and this one's results through the last step's
        uint8_t *last = lds + (slot == 0 ? S - 1 : slot - 1) * STAGE;
        const int nb_ = nb, n0_ = n0, row0_ = row0, rows_ = rows, split_ = split;
        unit += gridDim.x;
        const bool again = unit < units;
        if (again) {
            take(unit);
            start();
        }
        finish<M, F32, BN, BT, WN, WT, STAGE>(p, last, acc, to, n_tiles, nb_, n0_, row0_, rows_, splits, split_);
        if (!again) break;
    }
}

// One launch of `kernel` with `bytes` of LDS, of `most` that it may ask for;
// `resident`: of each device, the workgroups that it holds at once, once `most` is set
template <typename K, typename... A>
hipError_t launch_lds(K kernel, std::atomic<int> (&resident)[64], int most, int bytes, int64_t grid, bool loops,
                      int threads, hipStream_t st, A... args) {
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    int at_once = dev < 64 ? resident[dev].load() : 0;
    if (!at_once) {
        int cus = 0, per = 0;
        e = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, most);
        if (e == hipSuccess) e = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev);
        if (e == hipSuccess) e = hipOccupancyMaxActiveBlocksPerMultiprocessor(&per, (const void *)kernel, threads, bytes);
        if (e != hipSuccess) return e;
        at_once = std::max(1, cus * per);
        if (dev < 64) resident[dev].store(at_once);
    }
    if (loops) grid = std::min<int64_t>(grid, at_once);
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(threads), bytes, st, args...);
    return hipSuccess;
}

template <Mode M, bool F32, bool ONCE, int BN, int BT, int WN, int WT, int S>
hipError_t launch_tiled(const ProductArgs &p, int t_tiles, int splits, hipStream_t st) {
    constexpr int bytes = S * ((BN + BT) * kQ + 512 * WN * WT);
    static_assert(bytes <= 160 * 1024);
    static std::atomic<int> resident[64];
    const int n_tiles = cdiv(p.N, M == Mode::GateUp ? BN / 2 : BN);
    return launch_lds(tiled_kernel<M, F32, ONCE, BN, BT, WN, WT, S>, resident, bytes, bytes,
                      (int64_t)n_tiles * t_tiles * splits, true, 64 * WN * WT, st, p, n_tiles, t_tiles, splits);
}

}  // namespace fp8
}  // namespace echo
