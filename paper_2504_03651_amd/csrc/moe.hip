// moe.hip -- routing to experts and their products (include/echo_moe.h), gfx950.
#include <hip/hip_runtime.h>

#include <float.h>
#include <algorithm>
#include <atomic>
#include <cmath>

#include "echo_moe.h"
#include "fp8.hpp"
#include "fp8_tiled.hpp"
#include "status.hpp"

namespace echo {
namespace fp8 {

constexpr int kMaxExperts = 512, kMaxTopK = 64, kMaxGroups = 64;

// ---------------------------------------------------------------- routing

struct RouteArgs {
    const void *logits;
    int64_t stride;
    const float *bias;
    int T, E, top_k, groups, top_groups, group_top;
    bool renormalize;
    float scale;
    int32_t *ids;
    float *weights;
};

// x before y in falling order of (value, -index)
template <typename V>
__device__ __forceinline__ bool ahead(V xv, int xi, V yv, int yi) {
    return xv > yv || (xv == yv && xi < yi);
}

// fp32 as integers of the same order (no NaN; -0 and 0 made equal first)
__device__ __forceinline__ int ordered(float x) {
    const int b = __float_as_int(x);
    return b ^ ((b >> 31) & 0x7FFFFFFF);
}
__device__ __forceinline__ float unordered(int k) { return __int_as_float(k ^ ((k >> 31) & 0x7FFFFFFF)); }

// max over LANES lanes: rotations in rows of 16, then swaps of rows and halves
template <int LANES>
__device__ __forceinline__ int lanes_max(int v) {
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x128, 0xF, 0xF, false));   // row_ror:8
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x124, 0xF, 0xF, false));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x122, 0xF, 0xF, false));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x121, 0xF, 0xF, false));
    if constexpr (LANES == 16) return v;
    const auto a = __builtin_amdgcn_permlane16_swap((uint32_t)v, (uint32_t)v, false, false);
    v = max((int)a[0], (int)a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap((uint32_t)v, (uint32_t)v, false, false);
    return __builtin_amdgcn_readfirstlane(max((int)b[0], (int)b[1]));
}

// Of each token, LANES lanes of the wave: groups by the sum of their best one or
// two of `value` (of all experts, in LDS): the kept ones as bits group * lanes, in
// `keep`.  LANES / (a power of two of at least that many groups) = `lanes` lanes share
// a group.  exact: what is in LDS decides; otherwise values are within off (1 + |value|)
// of the true ones, and what is returned is whether every kept group is ahead of every
// dropped one all the same.  A group's sum is then as far off as its values, which
// may be far larger than the sum: 2 off (1 + the larger magnitude), with the true
// best two no further from zero than that.
template <int LANES, typename V>
__device__ __forceinline__ bool keep_groups(const RouteArgs &a, const V *value, int lanes, int lane,
                                            bool exact, V off, uint64_t &keep) {
    const int sub = lane & (LANES - 1), from = lane & ~(LANES - 1);
    const int per = a.E / a.groups, g = sub / lanes, in = sub & (lanes - 1);
    V b1 = -INFINITY, b2 = -INFINITY;
    if (g < a.groups)
        for (int j = in; j < per; j += lanes) {
            const V k = value[g * per + j];
            b2 = k > b1 ? b1 : k > b2 ? k : b2;
            b1 = k > b1 ? k : b1;
        }
    for (int o = 1; o < lanes; o <<= 1) {
        const V c1 = __shfl_xor(b1, o), c2 = __shfl_xor(b2, o);
        const V lo = b1 < c1 ? b1 : c1, hi = b2 < c2 ? c2 : b2;
        b1 = b1 < c1 ? c1 : b1;
        b2 = lo < hi ? hi : lo;
    }
    V v = a.group_top == 2 ? b1 + b2 : b1;
    if (sizeof(V) == 8 && v > (V)DBL_MAX) v = (V)DBL_MAX;
    int rank = 0;
    for (int j = 0; j < a.groups; ++j) rank += ahead(__shfl(v, from + j * lanes), j, v, g);
    auto of = [&](bool x) -> uint64_t {   // this token's lanes where x holds of a group
        const uint64_t m = __ballot(in == 0 && g < a.groups && x) >> from;
        return LANES == 64 ? m : m & ((1ull << (LANES & 63)) - 1);
    };
    keep = of(rank < a.top_groups);
    if (exact || a.top_groups == a.groups) return true;
    if constexpr (sizeof(V) == 4) {
        const bool two = a.group_top == 2;
        // no value, or not two of them: exactly -inf
        const bool none = b1 == -INFINITY || (two && b2 == -INFINITY && b1 < INFINITY);
        const V most = two ? fmaxf(fabsf(b1), fabsf(b2)) : fabsf(b1);
        const V e = none ? 0 : off * (two ? 2 : 1) * (1 + most);
        const bool clear = of(!none && !(fabsf(v) + e < INFINITY)) == 0;   // no infinity, no NaN
        const bool mine = in == 0 && g < a.groups, kept = rank < a.top_groups;
        const int low = ordered(mine && kept ? v - e : INFINITY), high = ordered(mine && !kept ? v + e : -INFINITY);
        return ~lanes_max<LANES>(~low) > lanes_max<LANES>(high) && clear;
    }
    return false;
}

template <int LANES>
__device__ __forceinline__ int lanes_of_group(int groups) {
    int l = LANES;
    while (LANES / l < groups) l >>= 1;
    return l;
}

__device__ __forceinline__ float read_logit(const void *logits, bool f32, int64_t at) {
    const float f = f32 ? ((const float *)logits)[at] : bf2f(((const uint16_t *)logits)[at]);
    return f > -INFINITY ? fminf(f, FLT_MAX) + 0.f : -INFINITY;   // NaN too; -0 becomes 0
}

// fp64 as integers of the same order (no NaN; -0 and 0 made equal first), and their
// max over the wave: rotations in rows of 16 lanes, then swaps of rows and halves
__device__ __forceinline__ int64_t ordered64(double x) {
    const int64_t b = __double_as_longlong(x);
    return b ^ ((b >> 63) & INT64_MAX);
}
__device__ __forceinline__ int64_t two_words(uint32_t lo, uint32_t hi) { return (int64_t)((uint64_t)hi << 32 | lo); }
template <int DPP>
__device__ __forceinline__ int64_t max_of_turn(int64_t v) {
    return max(v, two_words(__builtin_amdgcn_update_dpp(0, (uint32_t)v, DPP, 0xF, 0xF, false),
                            __builtin_amdgcn_update_dpp(0, (uint32_t)(v >> 32), DPP, 0xF, 0xF, false)));
}
__device__ __forceinline__ int64_t wave_max64(int64_t v) {
    v = max_of_turn<0x121>(max_of_turn<0x122>(max_of_turn<0x124>(max_of_turn<0x128>(v))));   // row_ror
    const auto a = __builtin_amdgcn_permlane16_swap((uint32_t)v, (uint32_t)v, false, false);
    const auto b = __builtin_amdgcn_permlane16_swap((uint32_t)(v >> 32), (uint32_t)(v >> 32), false, false);
    v = max(two_words(a[0], b[0]), two_words(a[1], b[1]));
    const auto c = __builtin_amdgcn_permlane32_swap((uint32_t)v, (uint32_t)v, false, false);
    const auto d = __builtin_amdgcn_permlane32_swap((uint32_t)(v >> 32), (uint32_t)(v >> 32), false, false);
    return max(two_words(c[0], d[0]), two_words(c[1], d[1]));
}

// The definition, in 64 bits: what route_kernel takes where 32 do not decide.
// id and weight of lane j: of the row's j-th expert.  `row`: E doubles of LDS.
// Few rows come here and each waits for its instructions: loops stay loops.
template <bool F32, bool SIGMOID, int PER>
__device__ __forceinline__ void route_row64(const RouteArgs &a, int64_t t, double *row, int lane,
                                            int &id, float &weight) {
    auto logit = [&](int e) { return (double)read_logit(a.logits, F32, t * a.stride + e); };
    double top = -DBL_MAX, sum = 0.0;   // softmax: the largest logit, and the sum
    if constexpr (!SIGMOID) {
#pragma unroll 1
        for (int e = lane; e < a.E; e += 64) top = fmax(top, logit(e));
        for (int o = 1; o < 64; o <<= 1) top = fmax(top, __shfl_xor(top, o));
#pragma unroll 1
        for (int e = lane; e < a.E; e += 64) {
            const double z = logit(e);
            sum += z == -INFINITY ? 0.0 : exp(z - top);
        }
        for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o);
    }
    auto score = [&](double z) {
        if constexpr (SIGMOID) return z == -INFINITY ? 0.0 : 1.0 / (1.0 + exp(-z));
        else return z == -INFINITY || !(sum > 0.0) ? 0.0 : exp(z - top) / sum;
    };
    // keys, or what groups go by: a sum of two is of scores
    const bool scores = a.bias || (a.groups > 1 && a.group_top == 2);
#pragma unroll 1
    for (int e = lane; e < a.E; e += 64) {
        const double z = logit(e);
        double k = z;
        if (scores && z > -INFINITY) {
            k = score(z);
            if (a.bias) k += (double)a.bias[e];
            k = k > -INFINITY ? fmin(k, DBL_MAX) : -INFINITY;   // a NaN too
        }
        row[e] = k;
    }
    wave_lds();
    uint64_t keep = ~0ull;
    const int per = a.E / a.groups, lanes = lanes_of_group<64>(a.groups);
    if (a.groups > 1) keep_groups<64, double>(a, row, lanes, lane, true, 0.0, keep);
    int64_t key[PER];
    const int64_t none = ordered64(-INFINITY);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int e = lane + 64 * i;
        key[i] = none;
        if (e < a.E && (keep >> (e / per * lanes) & 1)) key[i] = ordered64((a.bias ? row[e] : logit(e)) + 0.0);
    }
    id = -1;
#pragma unroll 1
    for (int j = 0; j < a.top_k; ++j) {
        int64_t m = key[0];
#pragma unroll
        for (int i = 1; i < PER; ++i) m = max(m, key[i]);
        m = wave_max64(m);
        if (m <= none) break;
        bool found = false;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const uint64_t hit = __ballot(key[i] == m);
            if (found || !hit) continue;
            found = true;
            const int l = __builtin_ctzll(hit);
            if (lane == l) key[i] = none;
            if (lane == j) id = l + 64 * i;
        }
    }
    double w = id >= 0 ? score(logit(id)) : 0.0;
    if (a.renormalize) {
        double all = w;
        for (int o = 1; o < 64; o <<= 1) all += __shfl_xor(all, o);
        w = all > 0.0 ? w / all : 0.0;
    }
    weight = (float)(w * (double)a.scale);
}

// LANES lanes of a wave per token; lane l of them has experts l, l + LANES, ...
// Without a bias the keys are the logits, exact in fp32.  With one (or where groups
// go by sums of scores) the keys come in fp32, off by less than off (1 + |key|): for
// a sigmoid s = 1 / (1 + e), e = e^-z comes (|z| + 2) 2^-24 off, which makes s (1 - s)
// (|z| + 2) 2^-24 < 0.75 x 2^-24 of it, the sum and the hardware's reciprocal 3 x
// 2^-24 s, with the rounding of the key below 5 x 2^-24, taken as 8; for a softmax,
// with d = top - z, e^-d comes (d + 6) 2^-24 off (expf within three ulps), the sum the
// mean of that over its terms (d: 3.9 at most, of 512) and a rounding for each
// of a lane's PER additions and each step over the lanes, then two roundings, and e^-d
// d is at most 0.37: below PER + log2(LANES) + 18 times 2^-24, the 18 taken as 24.  Where
// two neighbours among the chosen and the next, or a kept group and a dropped one,
// are not further apart than that the row goes to route_row64.  The chosen experts'
// scores are taken in 64 bits.
// Bound by instructions, and where rows go to route_row64 by its 5.5 us: 16,412
// tokens of 256 experts, 8 chosen of 4 groups of 8 with a bias, take 26 us (30 with a
// wave a token, 60 all in 64 bits).
template <bool F32, bool SIGMOID, int PER, int LANES>
__global__ __launch_bounds__(256) void route_kernel(RouteArgs a) {
    extern __shared__ double route_lds[];
    static_assert(LANES == 16 || LANES == 64);
    constexpr int TOKENS = 64 / LANES;   // of a wave
    const int lane = threadIdx.x & 63, sub = lane & (LANES - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t t0 = ((int64_t)blockIdx.x * 4 + wave) * TOKENS;
    if (t0 >= a.T) return;
    const int64_t t = min(t0 + lane / LANES, (int64_t)a.T - 1);
    constexpr float off = 0x1p-24f * (SIGMOID ? 8 : PER + (LANES == 16 ? 4 : 6) + 24);
    // of a wave: E doubles, or E floats of each token
    double *row = route_lds + wave * a.E * (TOKENS > 1 ? TOKENS / 2 : 1);
    float z[PER];
    int key[PER];
    const int none = ordered(-INFINITY);
    auto logit = [&](int64_t t, int e) { return read_logit(a.logits, F32, t * a.stride + e); };
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int e = sub + LANES * i;
        z[i] = e < a.E ? logit(t, e) : -INFINITY;
        key[i] = ordered(z[i]);
    }
    float top = 0.f;
    if constexpr (!SIGMOID) {
        int m = key[0];
#pragma unroll
        for (int i = 1; i < PER; ++i) m = max(m, key[i]);
        top = unordered(lanes_max<LANES>(m));
    }
    const bool sums = a.groups > 1 && a.group_top == 2 && !a.bias;   // groups by sums of scores
    if (a.bias || sums) {
        float sc[PER];
        if constexpr (SIGMOID) {
#pragma unroll
            for (int i = 0; i < PER; ++i)
                sc[i] = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504f * z[i]));
        } else {
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                sc[i] = z[i] == -INFINITY ? 0.f : expf(z[i] - top);
                sum += sc[i];
            }
            for (int o = 1; o < LANES; o <<= 1) sum += __shfl_xor(sum, o);
            const float r = sum > 0.f ? 1.f / sum : 0.f;
#pragma unroll
            for (int i = 0; i < PER; ++i) sc[i] *= r;
        }
        if (a.bias) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const float k = sc[i] + a.bias[min(sub + LANES * i, a.E - 1)];
                key[i] = z[i] > -INFINITY && k > -INFINITY ? ordered(k) : none;   // not for NaN
            }
        }
        if (a.groups > 1) {
            float *value = (float *)row + lane / LANES * a.E;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int e = sub + LANES * i;
                if (e < a.E) value[e] = sums ? (z[i] > -INFINITY ? sc[i] : -INFINITY) : unordered(key[i]);
            }
        }
    } else if (a.groups > 1) {
        float *value = (float *)row + lane / LANES * a.E;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (sub + LANES * i < a.E) value[sub + LANES * i] = z[i];
    }
    bool sure = true;   // the same in a token's lanes
    if (a.groups > 1) {
        const int lanes = lanes_of_group<LANES>(a.groups);
        wave_lds();
        uint64_t keep;
        sure = keep_groups<LANES, float>(a, (const float *)row + lane / LANES * a.E, lanes, lane,
                                         !a.bias && !sums, off, keep);
        const uint32_t per = a.E / a.groups, inv = ((1u << 20) + per - 1) / per;   // e / per, e < 512
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const uint32_t at = ((sub + LANES * i) * inv >> 20) * lanes;
            if (!(LANES == 16 ? (uint32_t)keep >> at & 1 : (uint32_t)(keep >> at) & 1)) key[i] = none;
        }
    }
    // lane j: the row's j-th expert
    int id = -1;
    float before = INFINITY;
    for (int j = 0; j < a.top_k + (a.bias ? 1 : 0); ++j) {
        int m = key[0];
#pragma unroll
        for (int i = 1; i < PER; ++i) m = max(m, key[i]);
        m = lanes_max<LANES>(m);
        const bool is = m > none;
        if (!__any(is)) break;
        if (a.bias && is) {
            const float v = unordered(m);
            sure = sure && before - v > 2 * off * (1.f + fabsf(v));   // not for infinities
            before = fminf(v, FLT_MAX);
            if (v == INFINITY) sure = false;
        }
        if constexpr (LANES == 64) {
            bool found = false;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const uint64_t hit = __ballot(key[i] == m);
                if (found || !hit) continue;
                found = true;
                const int l = __builtin_ctzll(hit);
                if (lane == l) key[i] = none;
                if (lane == j) id = l + 64 * i;
            }
        } else {
            // the lowest expert with that key: of this lane, then of the token's lanes
            int mine = kMaxExperts;
#pragma unroll
            for (int i = PER - 1; i >= 0; --i) mine = key[i] == m ? sub + LANES * i : mine;
            const int e = -lanes_max<LANES>(-mine);
#pragma unroll
            for (int i = 0; i < PER; ++i) key[i] = e == sub + LANES * i ? none : key[i];
            if (sub == j && is) id = e;
        }
    }
    if (sub >= a.top_k) id = -1;   // the one looked at for its distance
    const float mine = id >= 0 ? logit(t, id) : -INFINITY;
    auto any = [&](bool x) {   // in this token's lanes
        const uint64_t m = __ballot(x) >> (lane & ~(LANES - 1));
        return LANES == 64 ? m != 0 : (m & ((1ull << (LANES & 63)) - 1)) != 0;
    };
    if (!SIGMOID && any(id >= 0 && mine - top < -690.f)) sure = false;   // scores near 64 bits' end
    double s = 0.0;
    if constexpr (SIGMOID) {
        if (id >= 0) s = 1.0 / (1.0 + exp(-(double)mine));
    } else {
        if (id >= 0) s = exp((double)mine - (double)top);
    }
    double sum = 1.0;
    if (a.renormalize) {
        sum = s;
        for (int o = 1; o < LANES; o <<= 1) sum += __shfl_xor(sum, o);
    } else if (!SIGMOID) {
        sum = 0.0;
#pragma unroll
        for (int i = 0; i < PER; ++i) sum += z[i] == -INFINITY ? 0.0 : exp((double)z[i] - (double)top);
        for (int o = 1; o < LANES; o <<= 1) sum += __shfl_xor(sum, o);
    }
    const float weight = (float)((sum > 0.0 ? s / sum : 0.0) * (double)a.scale);
    if (sure && sub < a.top_k && t0 + lane / LANES < a.T) {
        a.ids[t * a.top_k + sub] = id;
        a.weights[t * a.top_k + sub] = weight;
    }
    // the whole wave for each token left
    for (uint64_t left = __ballot(!sure && sub == 0 && t0 + lane / LANES < a.T); left; left &= left - 1) {
        const int64_t at = t0 + __builtin_ctzll(left) / LANES;
        int id64;
        float w64;
        wave_lds();
        route_row64<F32, SIGMOID, (PER * LANES + 63) / 64>(a, at, row, lane, id64, w64);
        if (lane < a.top_k) {
            a.ids[at * a.top_k + lane] = id64;
            a.weights[at * a.top_k + lane] = w64;
        }
    }
}

template <bool F32, bool SIGMOID, int LANES>
void launch_route(const RouteArgs &a, hipStream_t st) {
    constexpr int U = 64 / LANES;
    const dim3 grid((unsigned)cdiv(a.T, 4 * U)), block(256);
    const size_t lds = 4 * (size_t)a.E * std::max(8, 4 * U);
    if (a.E <= 64) hipLaunchKernelGGL((route_kernel<F32, SIGMOID, U, LANES>), grid, block, lds, st, a);
    else if (a.E <= 128) hipLaunchKernelGGL((route_kernel<F32, SIGMOID, 2 * U, LANES>), grid, block, lds, st, a);
    else if (LANES == 16 || a.E <= 256)
        hipLaunchKernelGGL((route_kernel<F32, SIGMOID, 4 * U, LANES>), grid, block, lds, st, a);
    else if constexpr (LANES == 64)
        hipLaunchKernelGGL((route_kernel<F32, SIGMOID, 8, LANES>), grid, block, lds, st, a);
}

// Sixteen lanes a token take half the instructions, but four times as long over one
// token: many tokens of up to 256 experts go that way, where 16 lanes have a place
// for each chosen expert and the next, and one for each group.  Us by a wave a token
// and by 16 lanes, 8 chosen, for 2,000, 4,000, 8,000 and 16,000 tokens:
//    64 experts              4.8 5.3    5.6 5.3    7.7 5.7    11.9 6.9
//   128, 4 groups            6.8 7.9    8.3 8.1    13.2 11.0  19.0 12.7
//   256, 8 groups, a bias    11.4 14.9  15.6 18.0  20.8 20.3  29.6 26.6
//   512                      7.5 11.9   8.9 12.3   14.2 14.9  24.1 31.5
template <bool F32, bool SIGMOID>
void launch_route(RouteArgs a, hipStream_t st) {
    constexpr int kMost = 1 << 25;   // tokens of a launch, which has fewer than 2^32 threads
    for (; a.T > kMost; a.T -= kMost) {
        RouteArgs part = a;
        part.T = kMost;
        launch_route<F32, SIGMOID>(part, st);
        a.logits = (const uint8_t *)a.logits + kMost * a.stride * (F32 ? 4 : 2);
        a.ids += (int64_t)kMost * a.top_k;
        a.weights += (int64_t)kMost * a.top_k;
    }
    if (a.T > 4096 && a.E <= 256 && a.top_k < 16 && a.groups <= 16) launch_route<F32, SIGMOID, 16>(a, st);
    else launch_route<F32, SIGMOID, 64>(a, st);
}

// ------------------------------------------------------------ the experts

// The pairs in order of expert, each expert's cut into tiles of `tile` rows:
// counts, their prefix sums, then every pair to its place.  Up to 64 workgroups
// of 1,024 threads have `chunk` pairs each; more than one find the counts of all
// chunks in `counts` [workgroup][E], from count_pairs_kernel.  The order inside an
// expert is the order of the atomics, which no result hangs on: a pair's row is
// computed alone and ends at the pair's own place.  37,120 pairs of 64 experts: 5 us
// to count and 8 to place (38 in one workgroup).  Bound by latency.
__global__ __launch_bounds__(1024) void count_pairs_kernel(const int32_t *ids, int R, int E, int chunk,
                                                           int *counts) {
    __shared__ int count[kMaxExperts];
    const int tid = threadIdx.x;
    if (tid < kMaxExperts) count[tid] = 0;
    __syncthreads();
    const int end = min(R, (int)(blockIdx.x + 1) * chunk);
    for (int i = blockIdx.x * chunk + tid; i < end; i += 1024) {
        const int e = ids[i];
        if (e >= 0 && e < E) atomicAdd(&count[e], 1);
    }
    __syncthreads();
    if (tid < E) counts[blockIdx.x * E + tid] = count[tid];
}

__global__ __launch_bounds__(1024) void place_pairs_kernel(const int32_t *ids, int R, int E, int chunk,
                                                           const int *counts, int tile, int *num_tiles,
                                                           Tile *tiles, int *order) {
    // of each expert: its pairs, then the next free place; the first place and tile
    __shared__ int count[kMaxExperts], first[kMaxExperts], tfirst[kMaxExperts];
    const int tid = threadIdx.x, me = blockIdx.x;
    const int begin = me * chunk, end = min(R, begin + chunk);
    int before = 0;   // pairs of expert tid in the chunks before this one
    if (tid < kMaxExperts) {
        int n = 0;
        if (counts && tid < E)
            for (int b = 0; b < (int)gridDim.x; ++b) {
                const int c = counts[b * E + tid];
                n += c;
                before += b < me ? c : 0;
            }
        count[tid] = n;
    }
    __syncthreads();
    if (!counts) {
        for (int i = begin + tid; i < end; i += 1024) {
            const int e = ids[i];
            if (e >= 0 && e < E) atomicAdd(&count[e], 1);
        }
        __syncthreads();
    }
    if (tid < 64) {   // prefix sums, eight experts a lane
        constexpr int PER = kMaxExperts / 64;
        int n = 0, t = 0;
        for (int i = 0; i < PER; ++i) {
            const int c = count[PER * tid + i];
            n += c;
            t += (c + tile - 1) / tile;
        }
        int sn = n, st = t;
        for (int o = 1; o < 64; o <<= 1) {
            const int an = __shfl_up(sn, o), at = __shfl_up(st, o);
            if (tid >= o) sn += an, st += at;
        }
        if (tid == 63 && me == 0) *num_tiles = st;
        sn -= n;
        st -= t;
        for (int i = 0; i < PER; ++i) {
            const int c = count[PER * tid + i];
            first[PER * tid + i] = sn;
            tfirst[PER * tid + i] = st;
            sn += c;
            st += (c + tile - 1) / tile;
        }
    }
    __syncthreads();
    if (tid < E) {
        const int n = count[tid], f = first[tid];
        if (me == 0)
            for (int i = 0; i * tile < n; ++i)
                tiles[tfirst[tid] + i] = Tile{tid, f + i * tile, min(tile, n - i * tile), 0};
        count[tid] = f + before;
    }
    __syncthreads();
    for (int i = begin + tid; i < end; i += 1024) {
        const int e = ids[i];
        if (e >= 0 && e < E) order[atomicAdd(&count[e], 1)] = i;
    }
}

// out[t] = residual[t] + sum_j weights[t][j] y[t][j], eight columns a thread; y fp16
// times 2^ye, of 2^shift columns each.  Bound by memory: 37,120 outputs of 2048 in 38
// us, 5.0 TB/s.
__global__ __launch_bounds__(256) void combine_kernel(const uint16_t *y, const int8_t *ye, int shift,
                                                      const int32_t *ids, const float *weights,
                                                      const uint16_t *residual, uint16_t *out,
                                                      int64_t n8, int H, int E, int top_k) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= n8) return;
    const int64_t t = i / (H / 8);
    const int h = 8 * (int)(i - t * (H / 8)), groups = ((H - 1) >> shift) + 1;
    float v[8] = {};
    for (int j = 0; j < top_k; ++j) {
        const int64_t pair = t * top_k + j;
        const int e = ids[pair];
        if (e < 0 || e >= E) continue;
        const float w = weights[pair];
        const int up = ye[pair * groups + (h >> shift)];
        const u32x4 q = *(const u32x4 *)(y + pair * H + h);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const f16x2 two = __builtin_bit_cast(f16x2, (uint32_t)q[r]);
            v[2 * r] += w * __builtin_amdgcn_ldexpf((float)two[0], up);
            v[2 * r + 1] += w * __builtin_amdgcn_ldexpf((float)two[1], up);
        }
    }
    if (residual) {
        const u32x4 q = *(const u32x4 *)(residual + t * H + h);
#pragma unroll
        for (int r = 0; r < 4; ++r) v[2 * r] += bf2f(q[r] & 0xFFFFu), v[2 * r + 1] += bf2f(q[r] >> 16);
    }
    u32x4 o;
#pragma unroll
    for (int r = 0; r < 4; ++r) o[r] = f2bf2(v[2 * r], v[2 * r + 1]);
    *(u32x4 *)(out + t * H + h) = o;
}

}  // namespace fp8
}  // namespace echo

using namespace echo;
using namespace echo::fp8;

namespace {

struct Ws {
    int tile, max_tiles;   // rows of a tile, and the most tiles there can be
    int chunk, chunks;     // pairs that a workgroup places, and workgroups
    size_t num_tiles, counts, tiles, order, hs, hc, y, ye, total;
};

int plan_ws(const echo_experts_t *x, int32_t T, int32_t top_k, Ws *w) {
    if (!x) return fail(ECHO_E_INVALID, "experts is NULL");
    if (x->num_experts < 1 || x->num_experts > kMaxExperts)
        return fail(ECHO_E_UNSUPPORTED, "num_experts %d (1..%d)", x->num_experts, kMaxExperts);
    if (x->hidden <= 0 || x->intermediate <= 0)
        return fail(ECHO_E_INVALID, "hidden %d, intermediate %d", x->hidden, x->intermediate);
    if (x->hidden % 16 || x->intermediate % 16)
        return fail(ECHO_E_UNSUPPORTED, "hidden %d and intermediate %d must be multiples of 16",
                    x->hidden, x->intermediate);
    // offsets inside a tile of rows of `intermediate` codes are 32 bits
    if (x->intermediate > 1 << 23)
        return fail(ECHO_E_UNSUPPORTED, "intermediate %d above %d", x->intermediate, 1 << 23);
    if (T < 0) return fail(ECHO_E_INVALID, "num_tokens %d", T);
    if (top_k < 1 || top_k > kMaxTopK) return fail(ECHO_E_INVALID, "top_k %d (1..%d)", top_k, kMaxTopK);
    const int64_t R = (int64_t)T * top_k;
    if (R > 1 << 24) return fail(ECHO_E_UNSUPPORTED, "%lld pairs of token and expert", (long long)R);
    // offsets of codes inside an expert's matrices and inside x are 32 bits
    if (2 * (int64_t)x->intermediate * x->hidden > UINT32_MAX || (int64_t)T * x->hidden > UINT32_MAX)
        return fail(ECHO_E_UNSUPPORTED, "more than 2^32 codes in an expert's matrix (%d x %d) or in x (%d x %d)",
                    2 * x->intermediate, x->hidden, T, x->hidden);
    const int E = x->num_experts;
    // Tiles of as many pairs as experts get on average.  Us with tiles of 16, 32, 64 and
    // 128 rows, for 64 experts of 2048 x 1024, 128 of 1024 x 512, 16 of 4096 x 4096:
    //     4 pairs  78 78 -  -       52 52 -  -        183 190  -   -
    //     8        99 81 83 -       66 55 58 -        213 189 183  -
    //    16       105 103 88 101    72 68 60 70       221 231 186 218
    //    64       253 166 127 145   158 107 94 104    478 309 238 233
    //    80       295 183 156 150   187 121 105 106   584 375 298 275
    //   128       444 250 197 176   267 168 137 121   882 496 368 287
    // At 12 pairs tiles of 64 would be up to 11% faster than those of 32, but take their
    // gate and up sums from e4m3 products (run_experts).
    w->tile = R > 72 * (int64_t)E ? 128 : R > 12 * (int64_t)E ? 64 : R > 4 * (int64_t)E ? 32 : 16;
    w->max_tiles = (int)(R / w->tile + std::min<int64_t>(E, R));
    if ((int64_t)w->max_tiles * cdiv(x->hidden, 16) > INT32_MAX ||
        (int64_t)w->max_tiles * cdiv(x->intermediate, 16) > INT32_MAX)
        return fail(ECHO_E_UNSUPPORTED, "%lld pairs of token and expert", (long long)R);
    size_t o = 0;
    auto take = [&](size_t n) { const size_t at = o; o += (n + 255) / 256 * 256; return at; };
    w->chunk = std::max(4096, cdiv(R, 64));
    w->chunks = cdiv(R, w->chunk);
    w->num_tiles = take(4);
    w->counts = take(4 * (size_t)E * w->chunks);
    w->tiles = take(sizeof(Tile) * (R / 16 + std::min<int64_t>(E, R)));   // as for the smallest: no fall with T
    w->order = take(4 * R);
    w->hs = take(4 * R * cdiv(x->intermediate, kQ));
    w->hc = take(R * x->intermediate);
    w->y = take(2 * R * x->hidden);
    w->ye = take(R * cdiv(x->hidden, 16));   // of 16 columns or more
    w->total = R ? o : 0;
    return ECHO_OK;
}

int launched(const char *what) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? ECHO_OK : fail(ECHO_E_HIP, "%s: %s", what, hipGetErrorString(e));
}

// The forms of both products: the gate and up rows of 128 columns, and rows of
// the down matrix, by the tile's pairs.  columns: of y under one exponent.
// The gate and up sums decide codes, and one next to a border falls on either side of
// it by an e4m3 step.  Tiles of 16 and 32 pairs, which wait for their weights, take
// these sums from exact products at no cost (8 tokens through 64 experts of 2048 x
// 1024 59.4 and 59.5 us); larger ones, where a step more or less is one of many and
// exact products cost time (300 tokens 115 and 134 us, 4,640 505 and 620), take
// e4m3 products: 1.5e-5 off a sum, and 1.1 to 1.4 times the error of exact sums behind
// (2-norm of the outputs against 64 bits over 40 sizes: 1.5e-3 to 1.7e-3 with exact
// sums, their own rounding; 1.7e-3 to 2.3e-3).
template <int BT, int GN, int GT, int GS, int BN, int DN, int DT, int DS>
hipError_t run_experts(const ProductArgs &gu, ProductArgs dn, int max_tiles, int *columns, hipStream_t st) {
    hipError_t e = launch_tiled<Mode::GateUp, (BT <= 32), (BT <= 64), 256, BT, GN, GT, GS>(gu, max_tiles, 1, st);
    if (e == hipSuccess) e = hipGetLastError();
    if (e != hipSuccess) return e;
    *columns = BN / DN;
    dn.y_groups = cdiv(dn.N, *columns);
    return launch_tiled<Mode::Down, false, (BT <= 64), BN, BT, DN, DT, DS>(dn, max_tiles, 1, st);
}

}  // namespace

extern "C" {

int echo_moe_route(const echo_router_t *r, const void *logits, int32_t logits_dtype,
                   int64_t logits_stride, int32_t num_tokens, const float *bias, int32_t *ids,
                   float *weights, void *stream) {
    clear_error();
    if (!r) return fail(ECHO_E_INVALID, "router is NULL");
    if (r->num_experts < 1 || r->num_experts > kMaxExperts)
        return fail(ECHO_E_UNSUPPORTED, "num_experts %d (1..%d)", r->num_experts, kMaxExperts);
    if (r->score != ECHO_SCORE_SOFTMAX && r->score != ECHO_SCORE_SIGMOID)
        return fail(ECHO_E_UNSUPPORTED, "score %d", r->score);
    if (r->num_groups < 1 || r->num_groups > kMaxGroups || r->num_experts % r->num_groups)
        return fail(ECHO_E_INVALID, "num_groups %d of %d experts (1..%d, of equal size)",
                    r->num_groups, r->num_experts, kMaxGroups);
    const int per = r->num_experts / r->num_groups;
    if (r->top_groups < 1 || r->top_groups > r->num_groups)
        return fail(ECHO_E_INVALID, "top_groups %d of %d", r->top_groups, r->num_groups);
    if (r->group_top < 1 || r->group_top > 2 || (r->num_groups > 1 && r->group_top > per))
        return fail(ECHO_E_INVALID, "group_top %d of %d experts a group", r->group_top, per);
    if (r->top_k < 1 || r->top_k > kMaxTopK || r->top_k > r->top_groups * per)
        return fail(ECHO_E_INVALID, "top_k %d (1..%d, of %d experts)", r->top_k, kMaxTopK,
                    r->top_groups * per);
    if (!std::isfinite(r->scale)) return fail(ECHO_E_INVALID, "scale is not finite");
    if (logits_dtype != ECHO_BF16 && logits_dtype != ECHO_F32)
        return fail(ECHO_E_UNSUPPORTED, "dtype %d of logits", logits_dtype);
    if (num_tokens < 0) return fail(ECHO_E_INVALID, "num_tokens %d", num_tokens);
    if (num_tokens == 0) return ECHO_OK;
    if (!logits || !ids || !weights) return fail(ECHO_E_INVALID, "logits, ids or weights is NULL");
    if (logits_stride < r->num_experts)
        return fail(ECHO_E_INVALID, "logits_stride %lld < num_experts %d", (long long)logits_stride,
                    r->num_experts);
    const bool f32 = logits_dtype == ECHO_F32;
    if ((uintptr_t)logits & (f32 ? 3u : 1u) ||
        ((uintptr_t)ids | (uintptr_t)weights | (uintptr_t)bias) & 3u)
        return fail(ECHO_E_INVALID, "a buffer is not aligned to its type");
    const RouteArgs a{logits, logits_stride, bias, num_tokens, r->num_experts, r->top_k,
                      r->num_groups, r->top_groups, r->group_top, r->renormalize != 0, r->scale,
                      ids, weights};
    const hipStream_t st = (hipStream_t)stream;
    const bool sg = r->score == ECHO_SCORE_SIGMOID;
    if (f32) sg ? launch_route<true, true>(a, st) : launch_route<true, false>(a, st);
    else sg ? launch_route<false, true>(a, st) : launch_route<false, false>(a, st);
    return launched("echo_moe_route");
}

size_t echo_moe_experts_workspace_bytes(const echo_experts_t *experts, int32_t num_tokens,
                                        int32_t top_k) {
    clear_error();
    Ws w;
    return plan_ws(experts, num_tokens, top_k, &w) ? 0 : w.total;
}

int echo_moe_experts(const echo_experts_t *m, const void *x, const float *x_scale,
                     int32_t num_tokens, int32_t top_k, const int32_t *ids, const float *weights,
                     const void *residual, void *out, void *workspace, size_t workspace_bytes,
                     void *stream) {
    clear_error();
    Ws w;
    int rc = plan_ws(m, num_tokens, top_k, &w);
    if (rc) return rc;
    if (!m->w_gate_up || !m->gate_up_scale || !m->w_down || !m->down_scale)
        return fail(ECHO_E_INVALID, "an expert weight or scale is NULL");
    if (((uintptr_t)m->w_gate_up | (uintptr_t)m->w_down) & 15u)
        return fail(ECHO_E_INVALID, "expert weights must be 16-byte aligned");
    if (((uintptr_t)m->gate_up_scale | (uintptr_t)m->down_scale) & 3u)
        return fail(ECHO_E_INVALID, "expert scales are not aligned to their type");
    if (num_tokens == 0) return ECHO_OK;
    if (!x || !x_scale || !ids || !weights || !out)
        return fail(ECHO_E_INVALID, "x, x_scale, ids, weights or out is NULL");
    if (((uintptr_t)x | (uintptr_t)out | (uintptr_t)residual) & 15u)
        return fail(ECHO_E_INVALID, "x, residual and out must be 16-byte aligned");
    if (((uintptr_t)x_scale | (uintptr_t)ids | (uintptr_t)weights) & 3u)
        return fail(ECHO_E_INVALID, "a buffer is not aligned to its type");
    if (!workspace || workspace_bytes < w.total || ((uintptr_t)workspace & 255u))
        return fail(ECHO_E_WORKSPACE, "workspace of %zu bytes (need %zu, 256-byte aligned)",
                    workspace_bytes, w.total);
    const hipStream_t st = (hipStream_t)stream;
    uint8_t *base = (uint8_t *)workspace;
    const int E = m->num_experts, H = m->hidden, I = m->intermediate, R = num_tokens * top_k;
    const int HB = cdiv(H, kQ), IB = cdiv(I, kQ);
    int *counts = w.chunks > 1 ? (int *)(base + w.counts) : nullptr;
    if (counts) {
        hipLaunchKernelGGL(count_pairs_kernel, dim3(w.chunks), dim3(1024), 0, st, ids, R, E, w.chunk, counts);
        if ((rc = launched("counting of pairs"))) return rc;
    }
    hipLaunchKernelGGL(place_pairs_kernel, dim3(w.chunks), dim3(1024), 0, st, ids, R, E, w.chunk, counts,
                       w.tile, (int *)(base + w.num_tiles), (Tile *)(base + w.tiles), (int *)(base + w.order));
    if ((rc = launched("placing of pairs"))) return rc;

    ProductArgs gu{};
    gu.x = (const uint8_t *)x;
    gu.xs = x_scale;
    gu.w = (const uint8_t *)m->w_gate_up;
    gu.ws = m->gate_up_scale;
    gu.w_expert = 2 * (int64_t)I * H;
    gu.ws_expert = 2 * (int64_t)IB * HB;
    gu.T = R;
    gu.N = I;
    gu.K = H;
    gu.KB = HB;
    gu.hc = base + w.hc;
    gu.hs = (float *)(base + w.hs);
    gu.num_tiles = (const int *)(base + w.num_tiles);
    gu.tiles = (const Tile *)(base + w.tiles);
    gu.order = (const int *)(base + w.order);
    gu.top_k = top_k;
    ProductArgs dn = gu;
    dn.x = gu.hc;
    dn.xs = gu.hs;
    dn.w = (const uint8_t *)m->w_down;
    dn.ws = m->down_scale;
    dn.w_expert = (int64_t)H * I;
    dn.ws_expert = (int64_t)HB * IB;
    dn.N = H;
    dn.K = I;
    dn.KB = IB;
    dn.y = base + w.y;
    dn.y_stride = H;
    dn.ye = (int8_t *)(base + w.ye);
    int columns = 0;
    const hipError_t e =
        w.tile == 128  ? run_experts<128, 4, 2, 3, 256, 4, 2, 3>(gu, dn, w.max_tiles, &columns, st)
        : w.tile == 64 ? run_experts<64, 4, 2, 3, 128, 4, 1, 3>(gu, dn, w.max_tiles, &columns, st)
        : w.tile == 32 ? run_experts<32, 4, 1, 2, 128, 4, 1, 3>(gu, dn, w.max_tiles, &columns, st)
                       : run_experts<16, 8, 1, 2, 64, 4, 1, 4>(gu, dn, w.max_tiles, &columns, st);
    if (e != hipSuccess) return fail(ECHO_E_HIP, "experts' products: %s", hipGetErrorString(e));
    if ((rc = launched("experts' products"))) return rc;
    const int64_t n8 = (int64_t)num_tokens * H / 8;   // below 2^29
    hipLaunchKernelGGL(combine_kernel, dim3((unsigned)((n8 + 255) / 256)), dim3(256), 0, st,
                       (const uint16_t *)(base + w.y), dn.ye, __builtin_ctz(columns), ids, weights, (const uint16_t *)residual,
                       (uint16_t *)out, n8, H, E, top_k);
    return launched("weighted sum");
}

}  // extern "C"
