// rope.hip -- rotary positions (include/echo_rope.h) for gfx950.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "echo_rope.h"
#include "fp8.hpp"
#include "status.hpp"

namespace echo {
namespace rope {

using fp8::cdiv;

struct Tensor {
    const uint8_t *in;
    uint8_t *out;
    int64_t in_token, in_head, out_token, out_head;   // elements
    int heads;
};

struct Args {
    Tensor t[2];
    int heads;                  // of both
    const double *freq;
    const int32_t *pos;
    int tokens, D, R;
    int per_head;               // items of a head: R / 2P that turn, then copies
    int step_t, step_h, step_it;   // of the items that a workgroup's threads take at a time
    float magnitude, sign;
};

// cos and sin of p f, times the magnitude.  The turns p f / 2 pi are held in two
// fp64 numbers, so that only the eighth of a turn that is left is rounded to fp32.
__device__ __forceinline__ float2 turn_of(int p, double f, float magnitude, float sign) {
#pragma clang fp contract(off)   // t is the rounded product wherever it is used
    constexpr double kHi = 0.15915494309189535, kLo = -9.839338337591243e-18;   // 1 / 2 pi
    const double a = (double)p * f, ar = __builtin_fma((double)p, f, -a);
    const double t = a * kHi, tr = __builtin_fma(a, kHi, -t) + a * kLo + ar * kHi;
    const double whole = (t - __builtin_rint(t)) + tr;       // about -0.5 to 0.5 turns
    const double quarter = __builtin_rint(4.0 * whole);
    float s, c;
    sincospif((float)(2.0 * whole - 0.5 * quarter), &s, &c);
    const int q = (int)quarter & 3;
    const float x = q & 1 ? s : c, y = q & 1 ? c : s;
    return {(q == 1 || q == 2 ? -x : x) * magnitude, (q >= 2 ? -y : y) * magnitude * sign};
}

// N neighbouring elements, at any alignment of an element
template <bool F32, int N>
struct Some {
    uint32_t b[N];   // as fp32
    __device__ __forceinline__ void load(const uint8_t *at) {
        if constexpr (F32) {
            typedef uint32_t vec __attribute__((ext_vector_type(N), aligned(4)));
            const vec v = *(const vec *)at;
#pragma unroll
            for (int i = 0; i < N; ++i) b[i] = v[i];
        } else {
            typedef uint16_t vec __attribute__((ext_vector_type(N), aligned(2)));
            const vec v = *(const vec *)at;
#pragma unroll
            for (int i = 0; i < N; ++i) b[i] = (uint32_t)v[i] << 16;
        }
    }
    __device__ __forceinline__ void store(uint8_t *at) const {
        if constexpr (F32) {
            typedef uint32_t vec __attribute__((ext_vector_type(N), aligned(4)));
            vec v;
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = b[i];
            *(vec *)at = v;
        } else {
            typedef uint16_t vec __attribute__((ext_vector_type(N), aligned(2)));
            vec v;
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = (uint16_t)(b[i] >> 16);
            *(vec *)at = v;
        }
    }
    __device__ __forceinline__ float get(int i) const { return __uint_as_float(b[i]); }
    __device__ __forceinline__ void set(int i, float v) {
        b[i] = F32 ? __float_as_uint(v) : fp8::f2bf(v) << 16;
    }
};

// A workgroup takes `each` tokens and a part of their heads' items: an item is P pairs,
// or 2 P columns behind the rotary ones.  The tokens' turns are computed once, in LDS, for
// all of their heads.  Bound by memory: 4,640 tokens of 40 heads of 128 in bf16 (95 MB
// read and written) take 19.5 us, 4.9 TB/s, the rate of a copy; 1,531 of 30 heads of 80 in
// fp32, pairs two at a time, 7.9 us, 3.7 TB/s.
template <bool F32, bool INTER, int P>
__global__ __launch_bounds__(256) void rotate_kernel(Args a, int each, int parts) {
    extern __shared__ float2 turns[];   // [each][R / 2]
    constexpr int B = F32 ? 4 : 2;
    const int group = blockIdx.x / parts, part = blockIdx.x - group * parts;
    const int t0 = group * each, tokens = min(each, a.tokens - t0);
    const int half = a.R / 2;
    for (int i = threadIdx.x; i < tokens * half; i += 256) {
        const int t = i / half;
        turns[i] = turn_of(a.pos[t0 + t], a.freq[i - t * half], a.magnitude, a.sign);
    }
    __syncthreads();
    // A thread's items are a fixed number of tokens, heads and items of a head apart:
    // adding those with carries takes the place of two divisions an item (1,531 tokens
    // of 30 heads of 80, fp32: 8.2 us with them, 7.5 without)
    const int turning = half / P;
    int t = 0, h, it;
    {
        const int i = part * 256 + threadIdx.x, hi = i / a.per_head;
        it = i - hi * a.per_head;
        t = hi / a.heads;
        h = hi - t * a.heads;
    }
    while (t < tokens) {
        const bool second = h >= a.t[0].heads;
        const Tensor &x = second ? a.t[1] : a.t[0];
        const int64_t head = second ? h - a.t[0].heads : h;
        const uint8_t *in = x.in + ((int64_t)(t0 + t) * x.in_token + head * x.in_head) * B;
        uint8_t *out = x.out + ((int64_t)(t0 + t) * x.out_token + head * x.out_head) * B;
        if (it < turning) {
            const float2 *w = turns + t * half + P * it;
            const int lo = INTER ? 2 * P * it : P * it, hi = INTER ? lo + P : lo + half;
            Some<F32, P> u, v;
            u.load(in + lo * B);
            v.load(in + hi * B);
            if (INTER) {
                // pairs are neighbours: P of them lie in u and v side by side
                float f[2 * P];
#pragma unroll
                for (int k = 0; k < P; ++k) f[k] = u.get(k), f[P + k] = v.get(k);
#pragma unroll
                for (int k = 0; k < P; ++k) {
                    const float c = w[k].x, s = w[k].y, p = f[2 * k], q = f[2 * k + 1];
                    const float o0 = p * c - q * s, o1 = q * c + p * s;
                    if (2 * k < P) u.set(2 * k, o0);
                    else v.set(2 * k - P, o0);
                    if (2 * k + 1 < P) u.set(2 * k + 1, o1);
                    else v.set(2 * k + 1 - P, o1);
                }
            } else {
#pragma unroll
                for (int k = 0; k < P; ++k) {
                    const float c = w[k].x, s = w[k].y, p = u.get(k), q = v.get(k);
                    u.set(k, p * c - q * s);
                    v.set(k, q * c + p * s);
                }
            }
            u.store(out + lo * B);
            v.store(out + hi * B);
        } else if (in != out) {
            const int col = a.R + 2 * P * (it - turning);
            Some<F32, P> u, v;
            u.load(in + col * B);
            const bool two = P > 1 || col + 1 < a.D;   // an odd head's last column
            if (two) v.load(in + (col + P) * B);
            u.store(out + col * B);
            if (two) v.store(out + (col + P) * B);
        }
        it += a.step_it;
        h += a.step_h;
        t += a.step_t;
        if (it >= a.per_head) it -= a.per_head, ++h;
        if (h >= a.heads) h -= a.heads, ++t;
    }
}

template <bool F32, bool INTER, int P>
hipError_t launch(Args a, hipStream_t st) {
    const int half = a.R / 2;
    a.per_head = half / P + cdiv(a.D - a.R, 2 * P);
    const int items = a.heads * a.per_head;
    // tokens of a workgroup: as many as have turns for its threads, one where there are few
    const int each = std::max(1, std::min({256 / half, a.tokens / 1024, (1 << 24) / items}));
    constexpr int kMost = 1 << 22;   // groups; a launch has fewer than 2^32 threads
    for (int left = a.tokens;;) {
        a.tokens = (int)std::min<int64_t>(left, (int64_t)kMost * each);
        const int groups = cdiv(a.tokens, each);
        const int parts = std::max(1, std::min(cdiv((int64_t)items * each, 256), 1024 / groups));
        const int step = 256 * parts;
        a.step_it = step % a.per_head;
        a.step_h = step / a.per_head % a.heads;
        a.step_t = step / a.per_head / a.heads;
        hipLaunchKernelGGL((rotate_kernel<F32, INTER, P>), dim3((unsigned)(groups * parts)), dim3(256),
                           each * half * sizeof(float2), st, a, each, parts);
        const hipError_t e = hipGetLastError();
        left -= a.tokens;
        if (e != hipSuccess || left == 0) return e;
        a.pos += a.tokens;
        for (Tensor &t : a.t) {
            t.in += a.tokens * t.in_token * (F32 ? 4 : 2);
            t.out += a.tokens * t.out_token * (F32 ? 4 : 2);
        }
    }
}

template <bool F32, bool INTER>
hipError_t launch_by_width(const Args &a, hipStream_t st) {
    auto fits = [&](int P) { return a.R / 2 % P == 0 && (a.D - a.R) % (2 * P) == 0; };
    if (!F32 && fits(8)) return launch<F32, INTER, 8>(a, st);
    if (fits(4)) return launch<F32, INTER, 4>(a, st);
    if (fits(2)) return launch<F32, INTER, 2>(a, st);
    return launch<F32, INTER, 1>(a, st);
}

int check(const echo_rope_t *r) {
    if (!r) return fail(ECHO_E_INVALID, "rope is NULL");
    if (r->head_dim <= 0 || r->head_dim > 1024) return fail(ECHO_E_UNSUPPORTED, "head_dim %d", r->head_dim);
    if (r->rotary_dim < 2 || r->rotary_dim > r->head_dim || r->rotary_dim % 2)
        return fail(ECHO_E_INVALID, "rotary_dim %d of head_dim %d", r->rotary_dim, r->head_dim);
    if (r->layout != ECHO_ROPE_HALF && r->layout != ECHO_ROPE_INTERLEAVED)
        return fail(ECHO_E_UNSUPPORTED, "layout %d", r->layout);
    return ECHO_OK;
}

}  // namespace rope
}  // namespace echo

using namespace echo;
using namespace echo::rope;

extern "C" {

int echo_rope_frequencies(const echo_rope_t *r, double *frequencies, double *magnitude) {
    clear_error();
    const int rc = check(r);
    if (rc) return rc;
    if (!frequencies || !magnitude) return fail(ECHO_E_INVALID, "frequencies or magnitude is NULL");
    const int kind = r->scaling, R = r->rotary_dim;
    if (kind < ECHO_ROPE_NONE || kind > ECHO_ROPE_YARN) return fail(ECHO_E_UNSUPPORTED, "scaling %d", kind);
    const bool turns = kind == ECHO_ROPE_BANDS || kind == ECHO_ROPE_YARN;
    if (!(r->theta > (kind == ECHO_ROPE_YARN ? 1.0 : 0.0)) || std::isinf(r->theta))
        return fail(ECHO_E_INVALID, "theta %g", r->theta);
    if (kind != ECHO_ROPE_NONE && (!(r->factor >= 1.0) || std::isinf(r->factor)))
        return fail(ECHO_E_INVALID, "factor %g", r->factor);
    if (turns && (!(r->low > 0.0) || !(r->high > r->low) || std::isinf(r->high)))
        return fail(ECHO_E_INVALID, "low %g, high %g", r->low, r->high);
    if (turns && r->original_length <= 0) return fail(ECHO_E_INVALID, "original_length %d", r->original_length);
    const double s = kind == ECHO_ROPE_NONE ? 1.0 : r->factor, two_pi = 6.283185307179586;
    const double L = r->original_length;
    double theta = r->theta, lo = 0.0, hi = 0.0;
    if (kind == ECHO_ROPE_NTK && R > 2) theta *= std::pow(s, R / (R - 2.0));
    if (kind == ECHO_ROPE_YARN) {
        auto index = [&](double u) { return R * std::log(L / (two_pi * u)) / (2.0 * std::log(theta)); };
        lo = std::max(std::floor(index(r->high)), 0.0);
        hi = std::min(std::ceil(index(r->low)), R - 1.0);
    }
    for (int i = 0; i < R / 2; ++i) {
        const double f = std::pow(theta, -2.0 * i / R);
        double m = kind == ECHO_ROPE_LINEAR ? 0.0 : 1.0;
        if (kind == ECHO_ROPE_BANDS) m = (L * f / two_pi - r->low) / (r->high - r->low);
        if (kind == ECHO_ROPE_YARN) m = 1.0 - std::min(std::max((i - lo) / std::max(hi - lo, 0.001), 0.0), 1.0);
        m = std::min(std::max(m, 0.0), 1.0);
        frequencies[i] = f / s * (1.0 - m) + f * m;
    }
    *magnitude = kind == ECHO_ROPE_YARN ? 0.1 * std::log(s) + 1.0 : 1.0;
    return ECHO_OK;
}

int echo_rope_rotate(const echo_rope_t *rope, const double *frequencies, double magnitude,
                     const int32_t *positions, int32_t num_tokens, int32_t dtype,
                     const echo_rope_heads_t *tensors, int32_t num_tensors, int32_t inverse,
                     void *stream) {
    clear_error();
    const int rc = check(rope);
    if (rc) return rc;
    if (num_tokens < 0) return fail(ECHO_E_INVALID, "num_tokens %d", num_tokens);
    if (dtype != ECHO_BF16 && dtype != ECHO_F32) return fail(ECHO_E_UNSUPPORTED, "dtype %d", dtype);
    if (num_tensors < 1 || num_tensors > 2 || !tensors) return fail(ECHO_E_INVALID, "%d tensors", num_tensors);
    if (!std::isfinite((float)magnitude)) return fail(ECHO_E_INVALID, "magnitude %g", magnitude);
    if (num_tokens == 0) return ECHO_OK;
    if (!frequencies || !positions) return fail(ECHO_E_INVALID, "frequencies or positions is NULL");
    if ((uintptr_t)frequencies & 7u || (uintptr_t)positions & 3u)
        return fail(ECHO_E_INVALID, "frequencies must be 8-byte and positions 4-byte aligned");
    const uintptr_t mask = dtype == ECHO_F32 ? 3u : 1u;
    Args a{};
    int64_t heads = 0;
    for (int i = 0; i < num_tensors; ++i) {
        const echo_rope_heads_t &t = tensors[i];
        if (t.heads <= 0) return fail(ECHO_E_INVALID, "tensor %d: %d heads", i, t.heads);
        if (!t.in || !t.out) return fail(ECHO_E_INVALID, "tensor %d: in or out is NULL", i);
        if (((uintptr_t)t.in | (uintptr_t)t.out) & mask)
            return fail(ECHO_E_INVALID, "tensor %d must have its type's alignment", i);
        if (t.in == t.out && (t.in_token != t.out_token || t.in_head != t.out_head))
            return fail(ECHO_E_INVALID, "tensor %d: in place with other strides", i);
        // what is written lies token by token, or head by head
        const double D = rope->head_dim, T = num_tokens, H = t.heads;
        const double th = std::fabs((double)t.out_head), tt = std::fabs((double)t.out_token);
        if ((H > 1 && th < D) || (T > 1 && tt < D) ||
            (H > 1 && T > 1 && tt < (H - 1) * th + D && th < (T - 1) * tt + D))
            return fail(ECHO_E_INVALID, "tensor %d: heads of out overlap (strides %lld, %lld)", i,
                        (long long)t.out_token, (long long)t.out_head);
        a.t[i] = {(const uint8_t *)t.in, (uint8_t *)t.out, t.in_token, t.in_head, t.out_token, t.out_head, t.heads};
        heads += t.heads;
    }
    if (heads * rope->head_dim > 1 << 24)
        return fail(ECHO_E_UNSUPPORTED, "%lld heads of %d", (long long)heads, rope->head_dim);
    a.heads = (int)heads;
    a.freq = frequencies;
    a.pos = positions;
    a.tokens = num_tokens;
    a.D = rope->head_dim;
    a.R = rope->rotary_dim;
    a.magnitude = (float)magnitude;
    a.sign = inverse ? -1.f : 1.f;
    const hipStream_t st = (hipStream_t)stream;
    const bool inter = rope->layout == ECHO_ROPE_INTERLEAVED;
    const hipError_t e = dtype == ECHO_F32
        ? (inter ? launch_by_width<true, true>(a, st) : launch_by_width<true, false>(a, st))
        : (inter ? launch_by_width<false, true>(a, st) : launch_by_width<false, false>(a, st));
    return e == hipSuccess ? ECHO_OK : fail(ECHO_E_HIP, "echo_rope_rotate: %s", hipGetErrorString(e));
}

}  // extern "C"
