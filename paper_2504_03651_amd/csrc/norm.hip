// norm.hip -- norms, gate and residual between two blocks (include/echo_norm.h) for gfx950.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "echo_norm.h"
#include "fp8.hpp"
#include "status.hpp"

namespace echo {
namespace norm {

using fp8::any_f32x4;
using fp8::any_u32x2;
using fp8::any_u32x4;
using fp8::f2bf;
using fp8::f2bf2;
using fp8::f32x4;
using fp8::u32x2;
using fp8::u32x4;

// Codes of up to so many rows take a row by more waves of fewer values each, which has
// the shorter way (8 rows of 2048, two LAYER norms, launches one after the other: 3.9 us,
// by half the waves 5.0; 184 rows 4.3 and 5.4; two RMS norms of 8 rows of 4096 are the
// other way round, 3.7 and 3.4); past them what a wave does once for its values weighs
// more (4,640 rows of 4096: 39 and 32 us).
constexpr int kFewRows = 512;

struct Rows {
    uint8_t *data;   // null: there is none
    int64_t stride;  // elements
    int f32;
};

struct Args {
    Rows block, gate, residual, sum, y;
    float *y_scale;   // null: y is no codes
    const uint8_t *post_w, *post_b, *pre_w, *pre_b;
    int H, post, pre, param_f32;
    float post_eps, pre_eps, residual_scale, block_scale, weight_offset;
    double inv_h;   // 1 / H
    int rows, in_place;
};

// Pairs of norms that have a form of their own, without the branches for all the others
enum class Lean { No, Rms, Layer };

// Rows of whole eights, of any other width, and those shorter than eight
enum class Width { Whole, Odd, Tiny };

// Eight neighbouring values as they lie in memory, at any alignment of an element.
// BF: all tensors and parameters of the call are bf16.  TINY: n of them are there.
template <bool BF, bool TINY>
struct Raw {
    u32x4 a[BF ? 1 : 2];
    __device__ __forceinline__ void load(const uint8_t *p, int f32, int64_t at, int n) {
        if (!BF && f32) {
            const float *q = (const float *)p + at;
            if constexpr (TINY) {
#pragma unroll
                for (int i = 0; i < 8; ++i) a[BF ? 0 : i / 4][i % 4] = i < n ? __float_as_uint(q[i]) : 0u;
            } else {
                a[0] = __builtin_bit_cast(u32x4, *(const any_f32x4 *)q);
                a[BF ? 0 : 1] = __builtin_bit_cast(u32x4, *(const any_f32x4 *)(q + 4));
            }
        } else {
            const uint16_t *q = (const uint16_t *)p + at;
            if constexpr (TINY) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    a[0][i] = (2 * i < n ? q[2 * i] : 0u) | (2 * i + 1 < n ? (uint32_t)q[2 * i + 1] << 16 : 0u);
            } else {
                a[0] = *(const any_u32x4 *)q;
            }
        }
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < (BF ? 1 : 2); ++i) a[i] = (u32x4){0u, 0u, 0u, 0u};
    }
    __device__ __forceinline__ float get(int f32, int i) const {
        const uint32_t half = i & 1 ? a[0][i / 2] & 0xFFFF0000u : a[0][i / 2] << 16;
        if constexpr (BF) return __uint_as_float(half);
        return __uint_as_float(f32 ? a[BF ? 0 : i / 4][i % 4] : half);
    }
};

template <bool BF, bool TINY>
__device__ __forceinline__ void store8(uint8_t *p, int f32, int64_t at, int n, const float (&v)[8]) {
    if (!BF && f32) {
        float *q = (float *)p + at;
        if constexpr (TINY) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n) q[i] = v[i];
        } else {
            *(any_f32x4 *)q = (f32x4){v[0], v[1], v[2], v[3]};
            *(any_f32x4 *)(q + 4) = (f32x4){v[4], v[5], v[6], v[7]};
        }
    } else {
        uint16_t *q = (uint16_t *)p + at;
        if constexpr (TINY) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n) q[i] = (uint16_t)f2bf(v[i]);
        } else {
            *(any_u32x4 *)q = (u32x4){f2bf2(v[0], v[1]), f2bf2(v[2], v[3]), f2bf2(v[4], v[5]), f2bf2(v[6], v[7])};
        }
    }
}

// Sums and maxima over a row's WAVES waves: the lanes of sixteen meet by DPP, those of
// a wave by swapping rows, the waves in LDS, a barrier each, in places that take turns.
template <int CTRL>
__device__ __forceinline__ uint32_t turned(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
}
template <int LANES>
__device__ __forceinline__ void swapped(uint32_t v, uint32_t &x, uint32_t &y) {   // rows of v, and their neighbours'
    if constexpr (LANES == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        x = r[0], y = r[1];
    } else {
        const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        x = r[0], y = r[1];
    }
}
template <int CTRL, typename F>
__device__ __forceinline__ float meet(float v, F join) {
    return join(v, __uint_as_float(turned<CTRL>(__float_as_uint(v))));
}
template <int CTRL, typename F>
__device__ __forceinline__ double meet(double v, F join) {
    return join(v, __hiloint2double((int)turned<CTRL>((uint32_t)__double2hiint(v)), (int)turned<CTRL>((uint32_t)__double2loint(v))));
}
template <int LANES, typename F>
__device__ __forceinline__ float meet_rows(float v, F join) {
    uint32_t x, y;
    swapped<LANES>(__float_as_uint(v), x, y);
    return join(__uint_as_float(x), __uint_as_float(y));
}
template <int LANES, typename F>
__device__ __forceinline__ double meet_rows(double v, F join) {
    uint32_t xl, yl, xh, yh;
    swapped<LANES>((uint32_t)__double2loint(v), xl, yl);
    swapped<LANES>((uint32_t)__double2hiint(v), xh, yh);
    return join(__hiloint2double((int)xh, (int)xl), __hiloint2double((int)yh, (int)yl));
}

template <typename T, int WAVES>
struct Across {
    T (*room)[2 * WAVES];
    int turn;
    template <typename F>
    __device__ __forceinline__ T wave(T v, F join) {
        v = meet<0x128>(v, join);   // row_ror:8, 4, 2, 1
        v = meet<0x124>(v, join);
        v = meet<0x122>(v, join);
        v = meet<0x121>(v, join);
        v = meet_rows<16>(v, join);
        return meet_rows<32>(v, join);
    }
    template <typename F>
    __device__ __forceinline__ T all(T v, F join) {
        v = wave(v, join);
        if constexpr (WAVES > 1) {
            T *part = room[turn];
            turn ^= 1;
            if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
            __syncthreads();
            v = part[0];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) v = join(v, part[w]);
        }
        return v;
    }
    static __device__ __forceinline__ T add(T a, T b) { return a + b; }
    static __device__ __forceinline__ T more(T a, T b) { return a > b ? a : b; }
    __device__ __forceinline__ T sum(T v) { return all(v, add); }
    __device__ __forceinline__ T max(T v) { return all(v, more); }
    // the sum of s and the largest of m, behind one barrier
    __device__ __forceinline__ void both(T &s, T &m) {
        s = wave(s, add);
        m = wave(m, more);
        if constexpr (WAVES > 1) {
            T *part = room[turn];
            turn ^= 1;
            if ((threadIdx.x & 63) == 0) part[2 * (threadIdx.x >> 6)] = s, part[2 * (threadIdx.x >> 6) + 1] = m;
            __syncthreads();
            s = part[0], m = part[1];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) s = s + part[2 * w], m = more(m, part[2 * w + 1]);
        }
    }
};

__device__ __forceinline__ float inverse_root(float x) { return rsqrtf(x); }
// v_rsq_f64 is good to 2^-24 and better; one step of third order leaves 2^-70 of that
__device__ __forceinline__ double inverse_root(double x) {
    const double y = __builtin_amdgcn_rsq(x), e = __builtin_fma(-x * y, y, 1.0);
    const double root = __builtin_fma(y * e, __builtin_fma(e, 0.375, 0.5), y);
    return x < __builtin_inf() ? root : y;   // of an infinity 0, of a NaN one
}

// A row for WAVES waves (1: four rows a workgroup), V times eight values a lane, held
// in registers from the first step to the last: one pass over memory, which bounds rows
// in fp32 (1,003 rows of 2730, layer norms, 38 MB: 9.6 us, 4.0 TB/s, four sums one after
// the other on the way, those of the means in 64 bits).  Rows that end in codes are bound by instructions as well, some
// 24 in fp64 a value: 4,640 rows of 4096 with a gate, 133 MB, take 32.4 us, 4.1 TB/s, the
// vector units busy two thirds of it.  LEAN: two RMS norms with weights, or two LAYER
// norms with weights and biases, and no branches for all else, which cost copies of
// registers between them (4,640 rows of two RMS norms: 38 us without; 3,937 of 6936 with
// the stream in fp32 98, 70 with; 1,003 rows of two layer norms 10.7, 9.6 with).  T: what sums and rows are held in.
// The last eight of a row begin at H - 8, whatever H is a multiple of: what a lane
// before them has too counts for that one alone (`skip`), and comes out the same, to be
// written twice.  In rows of whole eights lanes behind the end hold zeros.  Where V <= 2
// every input is asked for before the first sum.
template <typename T, int WAVES, int V, bool BF, Width W, Lean LEAN>
__global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES, sizeof(T) == 4 && V == 1 && (BF || WAVES < (LEAN == Lean::No ? 6 : 8)) ? 8 : 1) void join_kernel(Args a, uint32_t first) {
    constexpr bool USUAL = LEAN != Lean::No;
    if (USUAL) {
        a.post = a.pre = LEAN == Lean::Rms ? ECHO_NORM_RMS : ECHO_NORM_LAYER;
        a.weight_offset = 0.f;
    }
    constexpr int LANES = 64 * WAVES;
    constexpr bool EARLY = V <= 2, TINY = W == Width::Tiny, WHOLE = W == Width::Whole;
    typedef Raw<BF, TINY> R;
    __shared__ __align__(16) T room[2][2 * WAVES];
    __shared__ __align__(16) double wide_room[2][2 * WAVES];   // of means
    Across<T, WAVES> across{room, 0};
    Across<double, WAVES> wide{wide_room, 0};
    const int lane = threadIdx.x % LANES;
    int64_t row = WAVES == 1 ? 4 * ((int64_t)first + blockIdx.x) + threadIdx.x / 64 : (int64_t)first + blockIdx.x;
    if (WAVES == 1) {
        if (row >= a.rows) return;
        const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)row);   // a wave has one
        row = (int64_t)((uint64_t)row >> 32 << 32 | lo);
    }
    int col[V], skip[V];   // the first column of a unit, its values that are another's
#pragma unroll
    for (int u = 0; u < V; ++u) {
        const int at = 8 * (lane + LANES * u);
        col[u] = TINY ? 0 : min(at, a.H - 8);
        skip[u] = TINY ? (at ? 8 : 0) : min(at - col[u], 8);
    }
    const int n = TINY ? a.H : 8;
    auto mine = [&](int u, int i) { return WHOLE || (i >= skip[u] && (!TINY || i < a.H)); };
    auto behind = [&](int u) { return WHOLE && skip[u] == 8; };
    auto take = [&](const Rows &r, int u) {
        R v;
        v.load(r.data, r.f32, row * r.stride + col[u], n);
        return v;
    };
    auto param = [&](const uint8_t *p, int u) {
        R v;
        v.load(p, a.param_f32, col[u], n);
        return v;
    };
    const bool block = USUAL || a.block.data, gate = block && a.gate.data, residual = USUAL || a.residual.data;
    const bool y = USUAL || a.y.data, post_w = USUAL || a.post_w, pre_w = USUAL || a.pre_w;
    const bool post_b = USUAL ? LEAN == Lean::Layer : a.post_b != nullptr;
    const bool pre_b = USUAL ? LEAN == Lean::Layer : a.pre_b != nullptr;
    R rb[EARLY ? V : 1], rg[EARLY ? V : 1], rr[EARLY ? V : 1], rw[EARLY ? V : 1], rw2[EARLY ? V : 1];
    if constexpr (EARLY) {
#pragma unroll
        for (int u = 0; u < V; ++u)
            if (block) rb[u] = take(a.block, u);
#pragma unroll
        for (int u = 0; u < V; ++u) {
            if (residual) rr[u] = take(a.residual, u);
            if (gate) rg[u] = take(a.gate, u);
            if (post_w) rw[u] = param(a.post_w, u);
            if (pre_w) rw2[u] = param(a.pre_w, u);
        }
    }
    auto apart = [] {   // loads of the next unit wait for this one's registers
        if constexpr (!EARLY) __builtin_amdgcn_sched_barrier(0);
    };

    T x[V][8];
    constexpr bool CODES = sizeof(T) == 8;
    auto any = [](bool v) { return __builtin_amdgcn_ballot_w64(v) != 0; };   // of what all lanes have alike
    // In fp32 a row whose squares leave the range, or a difference from whose mean may, is
    // taken times 2^shift, which brings the larger of its largest value and the root of eps
    // to about 1, and which its norm does not depend on.  Rows with an infinity stay.
    // (The tests for it, whose rare side lies behind the kernel's end, cost two layer norms
    // of 1,003 rows of 2730 0.2 us of 10.5, two RMS norms 0.1 of 5.7.)
    int shift = 0;
    auto resize = [&](float eps) {
        T top = T(0);
#pragma unroll
        for (int u = 0; u < V; ++u)
#pragma unroll
            for (int i = 0; i < 8; ++i) top = fmax(top, !TINY || mine(u, i) ? fabs(x[u][i]) : T(0));
        top = across.max(top);
        constexpr int kNone = -1000;
        const int of_x = top > T(0) ? __builtin_amdgcn_frexp_expf((float)top) : kNone;
        const int of_eps = eps > 0.f ? __builtin_amdgcn_frexp_expf(sqrtf(eps)) + shift : kNone;
        const int e = __builtin_amdgcn_readfirstlane(max(of_x, of_eps));
        if (e == kNone || any(!(top < (T)INFINITY))) return false;
        shift -= e;
#pragma unroll
        for (int u = 0; u < V; ++u)
#pragma unroll
            for (int i = 0; i < 8; ++i) x[u][i] = __builtin_amdgcn_ldexpf((float)x[u][i], -e);
        return true;
    };
    // x less its mean (LAYER).  Sums of two (in rows of whole eights of eight) are taken in
    // T, their sums in 64 bits, which is exact where the values are all alike, and so is the
    // division: the mean of a row of one value is that value.  (In fp32, with the mean
    // corrected by its residual, rows of 100.1 came out as 2.4e-3; 1,003 rows of 2730, two
    // layer norms, took 0.4 us of 10.5 less.)
    auto centre = [&](int kind) {
        if (kind != ECHO_NORM_LAYER) return;
        auto total = [&] {
            double s = 0.0;
#pragma unroll
            for (int u = 0; u < V; ++u) {
                T two[4];
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    two[i] = (mine(u, 2 * i) ? x[u][2 * i] : T(0)) + (mine(u, 2 * i + 1) ? x[u][2 * i + 1] : T(0));
                if (WHOLE) {
                    s += (double)((two[0] + two[1]) + (two[2] + two[3]));
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) s += (double)two[i];
                }
            }
            return wide.sum(s);
        };
        double s = total();
        // below that a difference from the mean stays in range
        if (!CODES && __builtin_expect_with_probability(any(!(fabs(s) < 0x1p100)), 0, .9))
            if (resize(0.f)) s = total();
        double by_h = s * a.inv_h;
        if (CODES) by_h = fma(fma(-by_h, (double)a.H, s), a.inv_h, by_h);   // in fp32 rounding does that
        const T mean = (T)by_h;
#pragma unroll
        for (int u = 0; u < V; ++u)
#pragma unroll
            for (int i = 0; i < 8; ++i) x[u][i] = behind(u) ? T(0) : x[u][i] - mean;
    };
    // Of this lane.  What is another's, or behind the end (there an infinite gate or weight
    // of the last eight leaves NaN), is left out, not multiplied by 0.
    auto squares = [&] {
        T ss = T(0);
#pragma unroll
        for (int u = 0; u < V; ++u) {
            const T before = ss;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const T with = fma(x[u][i], x[u][i], ss);
                ss = mine(u, i) ? with : ss;
            }
            if (behind(u)) ss = before;
        }
        return ss;
    };
    auto mean_square = [&](T ss, float eps) { return fma(ss, (T)a.inv_h, CODES ? (T)eps : (T)__builtin_amdgcn_ldexpf(eps, 2 * shift)); };
    auto inverse = [&](T ss, float eps) { return inverse_root(mean_square(ss, eps)); };
    auto settled = [&](float eps) {
        T ss = across.sum(squares());
        if constexpr (!CODES) {
            const T ms = mean_square(ss, eps);
            if (__builtin_expect_with_probability(any(!(ms >= 0x1p-60f && ms < (T)INFINITY)), 0, .9))
                if (resize(eps)) ss = across.sum(squares());
        }
        return inverse(ss, eps);
    };
    const T offset = (T)a.weight_offset;
    auto weigh = [&](int u, const R &w) {
        if (a.weight_offset == 0.f) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[u][i] *= (T)w.get(a.param_f32, i);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[u][i] *= (T)w.get(a.param_f32, i) + offset;
        }
    };
    if (block) {
#pragma unroll
        for (int u = 0; u < V; ++u) {
            apart();
            R r = EARLY ? rb[EARLY ? u : 0] : take(a.block, u);
            if (behind(u)) r.clear();
#pragma unroll
            for (int i = 0; i < 8; ++i) x[u][i] = (T)r.get(a.block.f32, i);
        }
        T by = (T)a.block_scale;
        if (a.post != ECHO_NORM_NONE) {
            centre(a.post);
            const T inv = settled(a.post_eps);
            if (post_w) {
#pragma unroll
                for (int u = 0; u < V; ++u) {
                    apart();
                    weigh(u, EARLY ? rw[EARLY ? u : 0] : param(a.post_w, u));
                }
            }
            if (post_b) {
#pragma unroll
                for (int u = 0; u < V; ++u) {
                    apart();
                    const R w = param(a.post_b, u);
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[u][i] = behind(u) ? T(0) : fma(x[u][i], inv, (T)w.get(a.param_f32, i));
                }
            } else {
                by *= inv;
            }
        }
#pragma unroll
        for (int u = 0; u < V; ++u)
#pragma unroll
            for (int i = 0; i < 8; ++i) x[u][i] *= by;
        if (gate) {
#pragma unroll
            for (int u = 0; u < V; ++u) {
                apart();
                const R g = EARLY ? rg[EARLY ? u : 0] : take(a.gate, u);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[u][i] *= (T)g.get(a.gate.f32, i);
            }
        }
    }
    if (residual) {
        const T by = (T)a.residual_scale;
#pragma unroll
        for (int u = 0; u < V; ++u) {
            apart();
            R r = EARLY ? rr[EARLY ? u : 0] : take(a.residual, u);
            if (behind(u)) r.clear();
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const T f = (T)r.get(a.residual.f32, i);
                x[u][i] = block ? fma(f, by, x[u][i]) : f * by;
            }
        }
    }
    // In place, a lane's last eight may be another's too: all have read theirs.
    if (WAVES > 1 && a.in_place) __syncthreads();
    if (a.sum.data) {
#pragma unroll
        for (int u = 0; u < V; ++u) {
            apart();
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = (float)x[u][i];
            if (skip[u] < 8) store8<BF, TINY>(a.sum.data, a.sum.f32, row * a.sum.stride + col[u], n, f);
        }
    }
    if (!y) return;
    // The largest of y, where that is codes, is the largest of x times 1 / root, so that it
    // is looked for along with the squares' sum, but under a bias.
    T inv = T(1), top = T(0);
    auto largest = [&] {   // of this lane: infinite where an infinity or a NaN is
        T top = T(0), odds = T(0);
#pragma unroll
        for (int u = 0; u < V; ++u)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (TINY && !mine(u, i)) continue;
                top = fmax(top, fabs(x[u][i]));
                odds = fma(x[u][i], T(0), odds);   // 0, or NaN
            }
        return odds == T(0) ? top : (T)INFINITY;
    };
    const bool normed = a.pre != ECHO_NORM_NONE;
    shift = 0;
    if (normed) centre(a.pre);
    T ss = T(0);
    if (normed && CODES && !pre_b) ss = squares();
    else if (normed) inv = settled(a.pre_eps);
    if (pre_w && normed) {
#pragma unroll
        for (int u = 0; u < V; ++u) {
            apart();
            weigh(u, EARLY ? rw2[EARLY ? u : 0] : param(a.pre_w, u));
        }
    }
    if (pre_b) {   // (none where there is no norm)
#pragma unroll
        for (int u = 0; u < V; ++u) {
            apart();
            const R w = param(a.pre_b, u);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[u][i] = behind(u) ? T(0) : fma(x[u][i], inv, (T)w.get(a.param_f32, i));
        }
        inv = T(1);
    }
    if constexpr (CODES) {
        top = largest();
        if (pre_b) {
            top = across.max(top);
        } else {
            across.both(ss, top);
            if (normed) inv = inverse(ss, a.pre_eps);
            top *= inv;
        }
    }
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int u = 0; u < V; ++u) {
            apart();
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = x[u][i] * inv;
            if (skip[u] < 8) store8<BF, TINY>(a.y.data, a.y.f32, row * a.y.stride + col[u], n, f);
        }
    } else {
        // top / 127, its product with 1 / 127 corrected by the residual
        constexpr double k127 = 1.0 / 127.0;
        const T part = top * k127;
        float s = (float)(top < (T)INFINITY ? fma(fma(-part, T(127), top), k127, part) : top);
        if (s == 0.f) s = 1.f;
        const bool odd = !(s < INFINITY);
        if (odd) s = __uint_as_float(0x7FC00000u);
        if (lane == 0) a.y_scale[row] = s;
        // 1 / s: v_rcp_f64 is good to 2^-24 and better, a step of third order leaves 2^-70
        const T r0 = __builtin_amdgcn_rcp((T)s), e0 = fma(-(T)s, r0, T(1));
        const T by = fma(r0 * e0, e0 + T(1), r0), both = by * inv;
        // a quotient corrected by its residual is exact where it is a tie, as those of sums
        // that no norm has touched may be; scales that are hardly numbers leave some past 127
        const bool plain = a.pre != ECHO_NORM_NONE && s >= 0x1p-100f;
#pragma unroll
        for (int u = 0; u < V; ++u) {
            apart();
            uint32_t q[2] = {0u, 0u};
            if (!odd) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t c[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const T f = x[u][4 * h + i];
                        T v = f * both;
                        if (!plain) {
                            v = fma(fma(-v, (T)s, f * inv), by, v);
                            v = fmin(fmax(v, T(-127)), T(127));
                        }
                        // the nearest integer (ties to even) in the low bits
                        c[i] = (uint32_t)__double2loint(v + 6755399441055744.0);
                    }
                    q[h] = __builtin_amdgcn_perm(c[1], c[0], 0x0C0C0400u) | __builtin_amdgcn_perm(c[3], c[2], 0x04000C0Cu);
                }
            }
            uint8_t *to = a.y.data + row * a.y.stride + col[u];
            if (skip[u] == 8) continue;
            if constexpr (TINY) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < n) to[i] = (uint8_t)(q[i / 4] >> (8 * (i % 4)));
            } else {
                typedef uint32_t pair __attribute__((ext_vector_type(2), aligned(1)));
                *(pair *)to = (pair){q[0], q[1]};
            }
        }
    }
}

// Which of the usual pairs the norms are: both RMS with weights alone, or both LAYER with
// weights and biases
Lean lean(const Args &a) {
    if (!a.post_w || !a.pre_w || a.weight_offset != 0.f || !a.block.data || !a.residual.data || !a.y.data) return Lean::No;
    if (a.post == ECHO_NORM_RMS && a.pre == ECHO_NORM_RMS && !a.post_b && !a.pre_b) return Lean::Rms;
    if (a.post == ECHO_NORM_LAYER && a.pre == ECHO_NORM_LAYER && a.post_b && a.pre_b) return Lean::Layer;
    return Lean::No;
}

template <typename T, int WAVES, int V, bool BF, Width W, Lean LEAN = Lean::No>
hipError_t launch(const Args &a, hipStream_t st) {
    if constexpr (LEAN == Lean::No && W != Width::Tiny) {
        const Lean usual = lean(a);
        if (usual == Lean::Rms) return launch<T, WAVES, V, BF, W, Lean::Rms>(a, st);
        if (usual == Lean::Layer) return launch<T, WAVES, V, BF, W, Lean::Layer>(a, st);
    }
    constexpr int kThreads = WAVES == 1 ? 256 : 64 * WAVES;
    constexpr int64_t kMost = ((int64_t)1 << 31) / kThreads;   // a launch has fewer than 2^32 threads
    const int64_t grid = WAVES == 1 ? ((int64_t)a.rows + 3) / 4 : a.rows;
    for (int64_t first = 0; first < grid; first += kMost) {
        hipLaunchKernelGGL((join_kernel<T, WAVES, V, BF, W, LEAN>), dim3((unsigned)std::min(kMost, grid - first)),
                           dim3(kThreads), 0, st, a, (uint32_t)first);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// Sums in fp32 depend on how a row is spread over lanes, so that this goes by its width
// alone; codes, which do not, take fewer waves of more values each where rows are many
// (4,333 rows of 640: 11.2 us by one wave, by four of which a row fills a third 17.1).
// Sixteen waves a row of up to 8192 were slower than eight (12 rows of 5264 into codes 5.9
// and 5.4 us, 1,136 of 7062 into fp32 21.8 and 21.3).
template <typename T, bool BF, Width W>
hipError_t launch_by_width(const Args &a, hipStream_t st) {
    if (a.H <= 512) return launch<T, 1, 1, BF, W>(a, st);
    if constexpr (sizeof(T) == 8)
        if (a.rows > kFewRows) {
            if (a.H <= 1024) return launch<T, 1, 2, BF, W>(a, st);
            if (a.H <= 2048) return launch<T, 2, 2, BF, W>(a, st);
            if (a.H <= 4096) return launch<T, 4, 2, BF, W>(a, st);
        }
    if (a.H <= 1024) return launch<T, 2, 1, BF, W>(a, st);
    if (a.H <= 2048) return launch<T, 4, 1, BF, W>(a, st);
    if (a.H <= 6 * 512) return launch<T, 6, 1, BF, W>(a, st);
    if (a.H <= 4096) return launch<T, 8, 1, BF, W>(a, st);
    if (a.H <= 8192) return launch<T, 8, 2, BF, W>(a, st);
    if (a.H <= 16384) return launch<T, 8, 4, BF, W>(a, st);
    if constexpr (sizeof(T) == 4) return launch<T, 16, 4, BF, W>(a, st);
    return hipErrorInvalidValue;   // codes: refused above
}

template <typename T, bool BF>
hipError_t launch_join(const Args &a, hipStream_t st) {
    if (a.H < 8) return launch<T, 1, 1, false, Width::Tiny>(a, st);
    return a.H % 8 == 0 ? launch_by_width<T, BF, Width::Whole>(a, st) : launch_by_width<T, BF, Width::Odd>(a, st);
}

// rows of a tensor that a call names, checked; `codes`: int8 ones are allowed
int take(const char *name, const echo_rows_t *from, int H, bool codes, bool one_row, Rows *to) {
    *to = Rows{};
    if (!from || !from->data) return ECHO_OK;
    if (from->dtype != ECHO_BF16 && from->dtype != ECHO_F32 && !(codes && from->dtype == ECHO_I8))
        return fail(ECHO_E_UNSUPPORTED, "dtype %d of %s", from->dtype, name);
    if (from->stride < H && !(one_row && from->stride == 0))
        return fail(ECHO_E_INVALID, "stride %lld of %s < hidden %d", (long long)from->stride, name, H);
    const uintptr_t mask = from->dtype == ECHO_F32 ? 3u : from->dtype == ECHO_BF16 ? 1u : 0u;
    if ((uintptr_t)from->data & mask) return fail(ECHO_E_INVALID, "%s must have its type's alignment", name);
    *to = {(uint8_t *)from->data, from->stride, from->dtype == ECHO_F32};
    return ECHO_OK;
}

}  // namespace norm
}  // namespace echo

using namespace echo;
using namespace echo::norm;

extern "C" {

int echo_norm_join(const echo_norm_t *norm, int32_t num_tokens, const echo_rows_t *block,
                   const echo_rows_t *gate, const echo_rows_t *residual, const echo_rows_t *sum,
                   const echo_rows_t *y, float *y_scale, void *stream) {
    clear_error();
    if (!norm) return fail(ECHO_E_INVALID, "norm is NULL");
    const int H = norm->hidden;
    if (H <= 0) return fail(ECHO_E_INVALID, "hidden %d", H);
    if (H > 32768) return fail(ECHO_E_UNSUPPORTED, "hidden %d above 32768", H);
    for (int kind : {norm->post, norm->pre})
        if (kind < ECHO_NORM_NONE || kind > ECHO_NORM_LAYER) return fail(ECHO_E_UNSUPPORTED, "norm %d", kind);
    if (norm->param_dtype != ECHO_BF16 && norm->param_dtype != ECHO_F32)
        return fail(ECHO_E_UNSUPPORTED, "dtype %d of weights", norm->param_dtype);
    for (float eps : {norm->post_eps, norm->pre_eps})
        if (!(eps >= 0.f) || std::isinf(eps)) return fail(ECHO_E_INVALID, "eps %g", eps);
    for (float s : {norm->residual_scale, norm->block_scale, norm->weight_offset})
        if (!std::isfinite(s)) return fail(ECHO_E_INVALID, "scale or weight_offset %g", s);
    const uintptr_t params = (uintptr_t)norm->post_weight | (uintptr_t)norm->post_bias |
                             (uintptr_t)norm->pre_weight | (uintptr_t)norm->pre_bias;
    if (params & (norm->param_dtype == ECHO_F32 ? 3u : 1u))
        return fail(ECHO_E_INVALID, "weights and biases must have their type's alignment");
    if (num_tokens < 0) return fail(ECHO_E_INVALID, "num_tokens %d", num_tokens);
    if (num_tokens == 0) return ECHO_OK;
    Args a{};
    int rc = take("block", block, H, false, false, &a.block);
    if (!rc) rc = take("gate", gate, H, false, true, &a.gate);
    if (!rc) rc = take("residual", residual, H, false, false, &a.residual);
    if (!rc) rc = take("sum", sum, H, false, false, &a.sum);
    if (!rc) rc = take("y", y, H, true, false, &a.y);
    if (rc) return rc;
    if (!a.block.data && !a.residual.data) return fail(ECHO_E_INVALID, "neither block nor residual");
    if (!a.sum.data && !a.y.data) return fail(ECHO_E_INVALID, "neither sum nor y");
    // in place: the same rows of the same type
    const struct {
        const Rows &out, &in;
        bool same_type;
        const char *what;
    } pairs[] = {{a.sum, a.block, a.sum.f32 == a.block.f32, "sum is block"},
                 {a.sum, a.residual, a.sum.f32 == a.residual.f32, "sum is residual"},
                 {a.y, a.block, y && y->dtype != ECHO_I8 && a.y.f32 == a.block.f32, "y is block"},
                 {a.y, a.residual, y && y->dtype != ECHO_I8 && a.y.f32 == a.residual.f32, "y is residual"},
                 {a.sum, a.y, false, "sum is y"},
                 {a.sum, a.gate, false, "sum is gate"},
                 {a.y, a.gate, false, "y is gate"}};
    for (const auto &q : pairs)
        if (q.out.data && q.out.data == q.in.data && (!q.same_type || q.out.stride != q.in.stride))
            return fail(ECHO_E_INVALID, "%s of another type or stride, or may not be", q.what);
    const bool codes = a.y.data && y->dtype == ECHO_I8;
    if (codes && H > 16384) return fail(ECHO_E_UNSUPPORTED, "hidden %d above 16384 for codes", H);
    if (codes && !y_scale) return fail(ECHO_E_INVALID, "y_scale is NULL");
    if (codes && (uintptr_t)y_scale & 3u) return fail(ECHO_E_INVALID, "y_scale must be 4-byte aligned");
    a.y_scale = codes ? y_scale : nullptr;
    a.post_w = (const uint8_t *)norm->post_weight;
    a.post_b = (const uint8_t *)norm->post_bias;
    a.pre_w = (const uint8_t *)norm->pre_weight;
    a.pre_b = (const uint8_t *)norm->pre_bias;
    a.H = H;
    a.post = norm->post;
    a.pre = norm->pre;
    if (a.post == ECHO_NORM_NONE) a.post_w = a.post_b = nullptr;
    if (a.pre == ECHO_NORM_NONE) a.pre_w = a.pre_b = nullptr;
    a.param_f32 = norm->param_dtype == ECHO_F32;
    a.post_eps = norm->post_eps;
    a.pre_eps = norm->pre_eps;
    a.residual_scale = norm->residual_scale;
    a.block_scale = norm->block_scale;
    a.weight_offset = norm->weight_offset;
    a.rows = num_tokens;
    a.inv_h = 1.0 / H;
    for (const Rows &out : {a.sum, a.y})
        a.in_place |= out.data && (out.data == a.block.data || out.data == a.residual.data);
    bool bf = !a.param_f32;
    for (const Rows &r : {a.block, a.gate, a.residual, a.sum, a.y}) bf &= !r.f32;
    const hipStream_t st = (hipStream_t)stream;
    const hipError_t e = codes ? (bf ? launch_join<double, true>(a, st) : launch_join<double, false>(a, st))
                               : (bf ? launch_join<float, true>(a, st) : launch_join<float, false>(a, st));
    return e == hipSuccess ? ECHO_OK : fail(ECHO_E_HIP, "echo_norm_join: %s", hipGetErrorString(e));
}

}  // extern "C"
