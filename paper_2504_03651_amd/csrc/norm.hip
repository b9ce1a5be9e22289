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
    int rows;
};

// Eight neighbouring values at any alignment of an element, n of which are there
struct Raw {
    u32x4 a, b;
    __device__ __forceinline__ void load(const uint8_t *p, int f32, int64_t at, int n) {
        if (f32) {
            const float *q = (const float *)p + at;
            if (n >= 8) {
                a = __builtin_bit_cast(u32x4, *(const any_f32x4 *)q);
                b = __builtin_bit_cast(u32x4, *(const any_f32x4 *)(q + 4));
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    a[i] = i < n ? __float_as_uint(q[i]) : 0u;
                    b[i] = i + 4 < n ? __float_as_uint(q[i + 4]) : 0u;
                }
            }
        } else {
            const uint16_t *q = (const uint16_t *)p + at;
            if (n >= 8) {
                a = *(const any_u32x4 *)q;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    a[i] = (2 * i < n ? q[2 * i] : 0u) | (2 * i + 1 < n ? (uint32_t)q[2 * i + 1] << 16 : 0u);
            }
        }
    }
    __device__ __forceinline__ void get(int f32, float (&v)[8]) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t wide = i < 4 ? a[i % 4] : b[i % 4];
            const uint32_t half = i & 1 ? a[i / 2] & 0xFFFF0000u : a[i / 2] << 16;
            v[i] = __uint_as_float(f32 ? wide : half);
        }
    }
};

// n of eight values to a row of bf16 or fp32
__device__ __forceinline__ void store8(uint8_t *p, int f32, int64_t at, int n, const float (&v)[8]) {
    if (f32) {
        float *q = (float *)p + at;
        if (n >= 8) {
            *(any_f32x4 *)q = (f32x4){v[0], v[1], v[2], v[3]};
            *(any_f32x4 *)(q + 4) = (f32x4){v[4], v[5], v[6], v[7]};
        } else {
#pragma unroll
            for (int i = 0; i < 7; ++i)
                if (i < n) q[i] = v[i];
        }
    } else {
        uint16_t *q = (uint16_t *)p + at;
        if (n >= 8) {
            *(any_u32x4 *)q = (u32x4){f2bf2(v[0], v[1]), f2bf2(v[2], v[3]), f2bf2(v[4], v[5]), f2bf2(v[6], v[7])};
        } else {
#pragma unroll
            for (int i = 0; i < 7; ++i)
                if (i < n) q[i] = (uint16_t)f2bf(v[i]);
        }
    }
}

// Sums and maxima over a row's WAVES waves.  `room` alternates between two places, so
// that one barrier a call is enough.
template <typename T, int WAVES>
struct Across {
    T (*room)[WAVES];
    int turn;
    template <typename F>
    __device__ __forceinline__ T all(T v, F join) {
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) v = join(v, __shfl_xor(v, o));
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
    __device__ __forceinline__ T sum(T v) {
        return all(v, [](T a, T b) { return a + b; });
    }
    __device__ __forceinline__ T max(T v) {
        return all(v, [](T a, T b) { return a > b ? a : b; });
    }
};

__device__ __forceinline__ float root(float x) { return sqrtf(x); }
__device__ __forceinline__ double root(double x) { return sqrt(x); }

// x -> its norm: mean and squares by sums over the row, then weight and bias
template <typename T, int V, int LANES, typename S>
__device__ __forceinline__ void normed(const Args &a, int kind, const uint8_t *w, const uint8_t *b, float eps,
                                       int lane, S &across, T (&x)[V][8]) {
    if (kind == ECHO_NORM_NONE) return;
    // (sums are divided by H: a row of one value has exactly that for its mean)
    T mean = T(0);
    if (kind == ECHO_NORM_LAYER) {
        T s = T(0);
#pragma unroll
        for (int u = 0; u < V; ++u)
#pragma unroll
            for (int i = 0; i < 8; ++i) s += x[u][i];   // 0 past the row's end
        mean = across.sum(s) / (T)a.H;
#pragma unroll
        for (int u = 0; u < V; ++u)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                x[u][i] = 8 * (lane + LANES * u) + i < a.H ? x[u][i] - mean : T(0);
    }
    T ss = T(0);
#pragma unroll
    for (int u = 0; u < V; ++u)
#pragma unroll
        for (int i = 0; i < 8; ++i) ss += x[u][i] * x[u][i];
    const T inv = T(1) / root(across.sum(ss) / (T)a.H + (T)eps);
#pragma unroll
    for (int u = 0; u < V; ++u) {
        const int col = 8 * (lane + LANES * u), n = a.H - col;
        if (n <= 0) continue;
        Raw r;
        float f[8];
        if (w) {
            r.load(w, a.param_f32, col, n);
            r.get(a.param_f32, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[u][i] *= inv * ((T)f[i] + (T)a.weight_offset);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[u][i] *= inv;
        }
        if (b) {
            r.load(b, a.param_f32, col, n);
            r.get(a.param_f32, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[u][i] += (T)f[i];
        }
    }
}

// A row for WAVES waves (1: four rows a workgroup), V times eight values a lane, held
// in registers from the first step to the last.  T: what sums and rows are held in.
template <typename T, int WAVES, int V>
__global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES) void join_kernel(Args a, uint32_t first) {
    constexpr int LANES = 64 * WAVES;
    __shared__ T room[2][WAVES];
    Across<T, WAVES> across{room, 0};
    const int lane = threadIdx.x % LANES;
    const int64_t row = WAVES == 1 ? 4 * ((int64_t)first + blockIdx.x) + threadIdx.x / 64 : (int64_t)first + blockIdx.x;
    if (WAVES == 1 && row >= a.rows) return;
    T x[V][8];
    auto column = [&](int u) { return 8 * (lane + LANES * u); };
#pragma unroll
    for (int u = 0; u < V; ++u)
#pragma unroll
        for (int i = 0; i < 8; ++i) x[u][i] = T(0);
    if (a.block.data) {
#pragma unroll
        for (int u = 0; u < V; ++u) {
            const int n = a.H - column(u);
            if (n <= 0) continue;
            Raw r;
            float f[8];
            r.load(a.block.data, a.block.f32, row * a.block.stride + column(u), n);
            r.get(a.block.f32, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[u][i] = (T)f[i];
        }
        normed<T, V, LANES>(a, a.post, a.post_w, a.post_b, a.post_eps, lane, across, x);
    }
#pragma unroll
    for (int u = 0; u < V; ++u) {
        const int col = column(u), n = a.H - col;
        if (n <= 0) continue;
        Raw r;
        float f[8];
        if (a.block.data) {
            if (a.gate.data) {
                r.load(a.gate.data, a.gate.f32, row * a.gate.stride + col, n);
                r.get(a.gate.f32, f);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[u][i] *= (T)f[i];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) x[u][i] *= (T)a.block_scale;
        }
        if (a.residual.data) {
            r.load(a.residual.data, a.residual.f32, row * a.residual.stride + col, n);
            r.get(a.residual.f32, f);
            if (a.block.data) {
#pragma unroll
                for (int i = 0; i < 8; ++i) x[u][i] += (T)a.residual_scale * (T)f[i];
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) x[u][i] = (T)a.residual_scale * (T)f[i];
            }
        }
        // past the row's end all is 0, whatever the gate's and norm's zeros met
#pragma unroll
        for (int i = 0; i < 8; ++i) x[u][i] = i < n ? x[u][i] : T(0);
        if (a.sum.data) {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = (float)x[u][i];
            store8(a.sum.data, a.sum.f32, row * a.sum.stride + col, n, f);
        }
    }
    if (!a.y.data) return;
    normed<T, V, LANES>(a, a.pre, a.pre_w, a.pre_b, a.pre_eps, lane, across, x);
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int u = 0; u < V; ++u) {
            const int n = a.H - column(u);
            if (n > 0) store8(a.y.data, a.y.f32, row * a.y.stride + column(u), n, x[u]);
        }
    } else {
        T top = T(0);
#pragma unroll
        for (int u = 0; u < V; ++u)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const T m = fabs(x[u][i]);
                top = fmax(top, i < a.H - column(u) ? (m != m ? (T)INFINITY : m) : T(0));
            }
        top = across.max(top);
        float s = (float)(top / T(127));
        if (s == 0.f) s = 1.f;
        const bool odd = !(s < INFINITY);
        if (odd) s = __uint_as_float(0x7FC00000u);
        if (lane == 0) a.y_scale[row] = s;
        const T by = T(1) / (T)s;
#pragma unroll
        for (int u = 0; u < V; ++u) {
            const int col = column(u), n = a.H - col;
            if (n <= 0) continue;
            uint32_t q[2] = {0u, 0u};
            if (!odd) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    // the quotient, corrected by its residual: exact where it is a tie
                    T v = x[u][i] * by;
                    v = fma(fma(-v, (T)s, x[u][i]), by, v);
                    v = v > T(127) ? T(127) : v < T(-127) ? T(-127) : v;
                    // the nearest integer (ties to even) in the low bits
                    const uint32_t code = (uint32_t)__double_as_longlong(v + 6755399441055744.0) & 0xFFu;
                    q[i / 4] |= code << (8 * (i % 4));
                }
            }
            uint8_t *to = a.y.data + row * a.y.stride + col;
            if (n >= 8) {
                typedef uint32_t pair __attribute__((ext_vector_type(2), aligned(1)));
                *(pair *)to = (pair){q[0], q[1]};
            } else {
#pragma unroll
                for (int i = 0; i < 7; ++i)
                    if (i < n) to[i] = (uint8_t)(q[i / 4] >> (8 * (i % 4)));
            }
        }
    }
}

template <typename T, int WAVES, int V>
hipError_t launch(const Args &a, hipStream_t st) {
    constexpr int64_t kMost = 1 << 22;   // a launch has fewer than 2^32 threads
    const int64_t grid = WAVES == 1 ? ((int64_t)a.rows + 3) / 4 : a.rows;
    for (int64_t first = 0; first < grid; first += kMost) {
        hipLaunchKernelGGL((join_kernel<T, WAVES, V>), dim3((unsigned)std::min(kMost, grid - first)),
                           dim3(WAVES == 1 ? 256 : 64 * WAVES), 0, st, a, (uint32_t)first);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T>
hipError_t launch_by_width(const Args &a, hipStream_t st) {
    if (a.H <= 512) return launch<T, 1, 1>(a, st);
    if (a.H <= 2048) return launch<T, 4, 1>(a, st);
    if (a.H <= 4096) return launch<T, 4, 2>(a, st);
    if (a.H <= 8192) return launch<T, 8, 2>(a, st);
    if (a.H <= 16384) return launch<T, 8, 4>(a, st);
    return launch<T, 8, 8>(a, st);
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
    a.param_f32 = norm->param_dtype == ECHO_F32;
    a.post_eps = norm->post_eps;
    a.pre_eps = norm->pre_eps;
    a.residual_scale = norm->residual_scale;
    a.block_scale = norm->block_scale;
    a.weight_offset = norm->weight_offset;
    a.rows = num_tokens;
    const hipError_t e = codes ? launch_by_width<double>(a, (hipStream_t)stream)
                               : launch_by_width<float>(a, (hipStream_t)stream);
    return e == hipSuccess ? ECHO_OK : fail(ECHO_E_HIP, "echo_norm_join: %s", hipGetErrorString(e));
}

}  // extern "C"
