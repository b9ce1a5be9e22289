// int8.hip -- quantisation and products in 8-bit integers (include/echo_int8.h) for gfx950.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>

#include "echo_int8.h"
#include "int8_cut.hpp"
#include "int8_stream.hpp"
#include "rows.hpp"
#include "status.hpp"

namespace echo {
namespace int8 {

// ----------------------------------------------------------- quantisation

// Codes are those of correctly rounded quotients.  With r = RN(1 / s) a product by r,
// corrected by its exact residual (Markstein), gives the same code for every bf16 value
// and every scale fp32(b / 127) of a bf16 b; for fp32 values the residual is taken twice,
// after which the quotient itself is the correctly rounded one.  Both need a scale in
// [2^-100, 2^100]; others divide.  The quotient of a row's largest value is below 127.5
// by far more than its rounding, so nothing needs clamping then.  Bound by memory: 66.5
// million bf16 values (4,640 rows of 14336) take 38.6 us, 5.2 TB/s; 8 fp32 rows of 4096 3.0.

// Codes of four quotients, in a word: adding 1.5 * 2^23 leaves the nearest integer (ties
// to even) in the low bits.
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
    constexpr float kInt = 12582912.f;
    const uint32_t lo = __builtin_amdgcn_perm(__float_as_uint(b + kInt), __float_as_uint(a + kInt), 0x0C0C0400u);
    const uint32_t hi = __builtin_amdgcn_perm(__float_as_uint(d + kInt), __float_as_uint(c + kInt), 0x04000C0Cu);
    return lo | hi;
}

template <bool F32>
__device__ __forceinline__ float quotient(float x, float s, float r, bool plain) {
    if (!plain) return __builtin_amdgcn_fmed3f(x / s, -127.f, 127.f);
    float q = x * r;
    if (F32) q = __builtin_fmaf(__builtin_fmaf(-q, s, x), r, q);
    return __builtin_fmaf(__builtin_fmaf(-q, s, x), r, q);
}

// bits of the largest magnitude of the lanes of a wave
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
    for (int o = 32; o > 0; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o));
    return v;
}

// A row for WAVES waves, 256 / (64 WAVES) rows a workgroup; V times eight values a lane,
// held in registers between the search for the largest and the codes, so that a row is
// read once.  HELD false: rows
// longer than that are read twice.
template <bool F32, int WAVES, int V, bool HELD>
__global__ __launch_bounds__(256) void quantize_kernel(const void *x, int64_t stride, int rows, int cols,
                                                       uint8_t *codes, float *scales, uint32_t first) {
    constexpr int LANES = 64 * WAVES, ROWS = 4 / WAVES;
    __shared__ uint32_t part[4];
    const int lane = threadIdx.x % LANES;
    const int64_t row = ((int64_t)first + blockIdx.x) * ROWS + threadIdx.x / LANES;
    if (WAVES == 1 && row >= rows) return;
    const int64_t at = row * stride;
    Eight<F32> v[V];
    uint32_t t = 0;
    for (int base = 0;; base += 8 * LANES * V) {
#pragma unroll
        for (int u = 0; u < V; ++u) {
            const int col = base + 8 * (lane + LANES * u);
            if (col < cols) v[u].load(x, at + col);   // cols a multiple of 16
            else v[u].zero();
        }
#pragma unroll
        for (int u = 0; u < V; ++u) t = max(t, v[u].top());
        if (HELD || base + 8 * LANES * V >= cols) break;
    }
    t = wave_max(t);
    if (WAVES > 1) {
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = t;
        __syncthreads();
        t = max(max(part[0], part[1]), max(part[2], part[3]));
    }
    const bool odd = t >= 0x7F800000u;   // an infinity or a NaN
    float s = __uint_as_float(t) / 127.f;
    if (s == 0.f) s = 1.f;
    if (odd) s = __uint_as_float(0x7FC00000u);
    if (lane == 0) scales[row] = s;
    const bool plain = s >= 0x1p-100f && s <= 0x1p100f;
    const float r = 1.f / s;
    for (int base = 0; base < cols; base += 8 * LANES * V) {
#pragma unroll
        for (int u = 0; u < V; ++u) {
            const int col = base + 8 * (lane + LANES * u);
            if (col >= cols) continue;
            if (!HELD) v[u].load(x, at + col);
            u32x2 q = {0u, 0u};
            if (!odd) {
                float f[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] = quotient<F32>(v[u].get(i), s, r, plain);
                q = (u32x2){codes4(f[0], f[1], f[2], f[3]), codes4(f[4], f[5], f[6], f[7])};
            }
            *(u32x2 *)(codes + row * cols + col) = q;
        }
        if (HELD) break;
    }
}

template <bool F32, int WAVES, int V, bool HELD>
hipError_t launch_quantize(const void *x, int64_t stride, int rows, int cols, uint8_t *codes, float *scales,
                           hipStream_t st) {
    constexpr int64_t kMost = 1 << 23;   // a launch has fewer than 2^32 threads
    const int64_t grid = cdiv(rows, 4 / WAVES);
    for (int64_t first = 0; first < grid; first += kMost) {
        hipLaunchKernelGGL((quantize_kernel<F32, WAVES, V, HELD>), dim3((unsigned)std::min(kMost, grid - first)),
                           dim3(256), 0, st, x, stride, rows, cols, codes, scales, (uint32_t)first);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <bool F32>
hipError_t quantize(const void *x, int64_t stride, int rows, int cols, uint8_t *codes, float *scales, hipStream_t st) {
    if (cols <= 512) return launch_quantize<F32, 1, 1, true>(x, stride, rows, cols, codes, scales, st);
    if (cols <= 1024) return launch_quantize<F32, 1, 2, true>(x, stride, rows, cols, codes, scales, st);
    if (cols <= 2048) return launch_quantize<F32, 4, 1, true>(x, stride, rows, cols, codes, scales, st);
    if (cols <= 4096) return launch_quantize<F32, 4, 2, true>(x, stride, rows, cols, codes, scales, st);
    if (cols <= 8192) return launch_quantize<F32, 4, 4, true>(x, stride, rows, cols, codes, scales, st);
    if (cols <= 16384) return launch_quantize<F32, 4, 8, true>(x, stride, rows, cols, codes, scales, st);
    return launch_quantize<F32, 4, 4, false>(x, stride, rows, cols, codes, scales, st);
}

// -------------------------------------------------------------- products

// y from the sums of all ranges of K, E columns a thread
template <bool F32>
__global__ __launch_bounds__(256) void add_parts_kernel(Product p, int ranges) {
    const int q = p.part_pitch / 4;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= (int64_t)p.T * q) return;
    const int64_t t = i / q;
    const int n = 4 * (int)(i - t * q);
    Columns<4> cols;
    cols.load(p, n);
    const Scale xs = split(p.xs[t]);
    const int32_t *from = p.part + t * p.part_pitch + n;
    i32x4 s = {0, 0, 0, 0};
    for (int r = 0; r < ranges; r += 4) {   // four at a time are under way
        i32x4 more[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            more[k] = *(const i32x4 *)(from + min(r + k, ranges - 1) * (int64_t)p.T * p.part_pitch);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (r + k < ranges) s += more[k];
    }
    const int sum[4] = {s[0], s[1], s[2], s[3]};
    float v[4];
    cols.apply(p, sum, xs, v);
    put_sum<F32, 4>(p, t, n, v);
}

// stages of a wave's ring, for NT = 1 and 2: at most 160 KiB for eight waves
constexpr int rows_depth(int NT, int XR) { return std::min(6, 160 * 1024 / (kStreamWaves * stream_stage(NT, XR))); }

template <bool F32, int NT>
hipError_t launch_rows(const Product &p, hipStream_t st) {
    switch (rows_tokens(p.T)) {   // up to 32 tokens every weight is read once
        case 8: return launch_stream<F32, true, NT, 8, rows_depth(NT, 8)>(p, st);
        case 16: return launch_stream<F32, true, NT, 16, rows_depth(NT, 16)>(p, st);
        default:
            return p.T <= 32 ? launch_stream<F32, true, NT, 32, rows_depth(NT, 32)>(p, st)
                             : launch_stream<F32, false, NT, 32, rows_depth(NT, 32)>(p, st);
    }
}

template <bool F32, int BN, int BT, int WN, int WT, int S>
hipError_t launch_tiles(const Product &p, int ranges, hipStream_t st) {
    if constexpr (BT <= 64)
        if (p.T <= BT) return launch_tiled<F32, true, BN, BT, WN, WT, S>(p, ranges, st);
    return launch_tiled<F32, false, BN, BT, WN, WT, S>(p, ranges, st);
}

template <bool F32>
hipError_t launch_gemm(const Product &p, Cut c, hipStream_t st) {
    hipError_t e = hipSuccess;
    switch (c.form) {
        case kRows16: return launch_rows<F32, 1>(p, st);
        case kRows32: return launch_rows<F32, 2>(p, st);
        case k64x32: e = launch_tiles<F32, 64, 32, 4, 1, 6>(p, c.ranges, st); break;
        case k64x64: e = launch_tiles<F32, 64, 64, 4, 1, 4>(p, c.ranges, st); break;
        case k128x64: e = launch_tiles<F32, 128, 64, 4, 1, 3>(p, c.ranges, st); break;
        case k128x96: e = launch_tiles<F32, 128, 96, 4, 2, 4>(p, c.ranges, st); break;
        case k128x128: e = launch_tiles<F32, 128, 128, 4, 2, 4>(p, c.ranges, st); break;
        case k128x160:   // one tile of tokens: a wave's sixteen weight rows against all of them
                         // (137 x 4096 x 14336 in six ranges: 20.7 us, by 4 x 2 waves 21.1)
            e = p.T <= 160 ? launch_tiles<F32, 128, 160, 8, 1, 4>(p, c.ranges, st)
                           : launch_tiles<F32, 128, 160, 4, 2, 4>(p, c.ranges, st);
            break;
        case k256x128: e = launch_tiles<F32, 256, 128, 4, 2, 3>(p, c.ranges, st); break;
        default:   // fp32 results of these tiles would spill registers: not chosen
            if constexpr (F32) e = hipErrorInvalidValue;
            else if (c.form == k128x128two) e = launch_tiles<F32, 128, 128, 2, 2, 2>(p, c.ranges, st);
            else e = launch_tiles<F32, 256, 192, 4, 2, 2>(p, c.ranges, st);
    }
    if (e != hipSuccess || c.ranges == 1 || (e = hipGetLastError()) != hipSuccess) return e;
    const int64_t n = (int64_t)p.T * (p.part_pitch / 4);
    hipLaunchKernelGGL(add_parts_kernel<F32>, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, p, c.ranges);
    return hipSuccess;
}

}  // namespace int8
}  // namespace echo

using namespace echo;
using namespace echo::int8;

namespace {

int launched(const char *what) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? ECHO_OK : fail(ECHO_E_HIP, "%s: %s", what, hipGetErrorString(e));
}

int check_sizes(int32_t T, int32_t N, int32_t K) {
    if (T < 0) return fail(ECHO_E_INVALID, "num_tokens %d", T);
    if (N <= 0 || K <= 0) return fail(ECHO_E_INVALID, "out_features %d, in_features %d", N, K);
    if (K % 16) return fail(ECHO_E_UNSUPPORTED, "in_features %d is not a multiple of 16", K);
    // sums of K products of -128 and -128 stay below 2^31
    if (K > 131056) return fail(ECHO_E_UNSUPPORTED, "in_features %d above 131056", K);
    if ((int64_t)cdiv(N, 16) * cdiv(T, 16) > INT32_MAX / 2 || N > 1 << 30 || T > 1 << 30)
        return fail(ECHO_E_UNSUPPORTED, "product of %d x %d too large", T, N);
    return ECHO_OK;
}

}  // namespace

extern "C" {

int echo_int8_quantize(const void *x, int32_t x_dtype, int64_t x_stride, int32_t rows,
                       int32_t cols, int8_t *codes, float *scales, void *stream) {
    clear_error();
    if (x_dtype != ECHO_BF16 && x_dtype != ECHO_F32)
        return fail(ECHO_E_UNSUPPORTED, "dtype %d of x", x_dtype);
    if (rows < 0 || cols <= 0) return fail(ECHO_E_INVALID, "rows %d, cols %d", rows, cols);
    if (cols % 16) return fail(ECHO_E_UNSUPPORTED, "cols %d is not a multiple of 16", cols);
    if (cols > 1 << 30) return fail(ECHO_E_UNSUPPORTED, "cols %d above 2^30", cols);
    if (rows == 0) return ECHO_OK;
    const int size = x_dtype == ECHO_F32 ? 4 : 2;
    if (!x || !codes || !scales) return fail(ECHO_E_INVALID, "x, codes or scales is NULL");
    if (x_stride < cols || x_stride % (16 / size))
        return fail(ECHO_E_INVALID, "x_stride %lld: at least cols %d, rows at 16-byte steps",
                    (long long)x_stride, cols);
    if (((uintptr_t)x | (uintptr_t)codes) & 15u)
        return fail(ECHO_E_INVALID, "x and codes must be 16-byte aligned");
    if ((uintptr_t)scales & 3u) return fail(ECHO_E_INVALID, "scales must be 4-byte aligned");
    const hipStream_t st = (hipStream_t)stream;
    const hipError_t e = size == 4 ? quantize<true>(x, x_stride, rows, cols, (uint8_t *)codes, scales, st)
                                   : quantize<false>(x, x_stride, rows, cols, (uint8_t *)codes, scales, st);
    return e == hipSuccess ? ECHO_OK : fail(ECHO_E_HIP, "echo_int8_quantize: %s", hipGetErrorString(e));
}

size_t echo_int8_gemm_workspace_bytes(int32_t num_tokens, int32_t out_features,
                                      int32_t in_features) {
    clear_error();
    if (check_sizes(num_tokens, out_features, in_features) || num_tokens == 0) return 0;
    return most_parts_bytes(num_tokens, out_features, in_features);
}

int echo_int8_gemm(const int8_t *x, const float *x_scale, const int8_t *w, const float *w_scale,
                   int32_t num_tokens, int32_t out_features, int32_t in_features,
                   const float *bias, const void *residual, void *y, int32_t y_dtype,
                   int64_t y_stride, void *workspace, size_t workspace_bytes, void *stream) {
    clear_error();
    const int rc = check_sizes(num_tokens, out_features, in_features);
    if (rc) return rc;
    if (y_dtype != ECHO_BF16 && y_dtype != ECHO_F32)
        return fail(ECHO_E_UNSUPPORTED, "dtype %d of y", y_dtype);
    if (num_tokens == 0) return ECHO_OK;
    if (!x || !x_scale || !w || !w_scale || !y)
        return fail(ECHO_E_INVALID, "x, w, their scales or y is NULL");
    if (y_stride < out_features)
        return fail(ECHO_E_INVALID, "y_stride %lld < out_features %d", (long long)y_stride,
                    out_features);
    if (((uintptr_t)x | (uintptr_t)w) & 15u)
        return fail(ECHO_E_INVALID, "x and w must be 16-byte aligned");
    const uintptr_t ya = (uintptr_t)y | (uintptr_t)residual;
    if (((uintptr_t)x_scale | (uintptr_t)w_scale | (uintptr_t)bias) & 3u || ya & (y_dtype == ECHO_F32 ? 3u : 1u))
        return fail(ECHO_E_INVALID, "scales, bias, y and residual must have their types' alignment");
    const Cut cut = cut_of(num_tokens, out_features, in_features, y_dtype == ECHO_F32);
    const size_t need = most_parts_bytes(num_tokens, out_features, in_features);
    if (need && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 255u)))
        return fail(ECHO_E_WORKSPACE, "workspace of %zu bytes (need %zu, 256-byte aligned)",
                    workspace_bytes, need);
    Product p{};
    p.x = (const uint8_t *)x;
    p.xs = x_scale;
    p.w = (const uint8_t *)w;
    p.ws = w_scale;
    p.bias = bias;
    p.T = num_tokens;
    p.N = out_features;
    p.K = in_features;
    p.KB = cdiv(in_features, kStep);
    p.residual = residual;
    p.y = y;
    p.y_stride = y_stride;
    p.part = (int32_t *)workspace;
    p.part_pitch = pitch_of(out_features);
    const hipError_t e = y_dtype == ECHO_F32 ? launch_gemm<true>(p, cut, (hipStream_t)stream)
                                             : launch_gemm<false>(p, cut, (hipStream_t)stream);
    if (e != hipSuccess) return fail(ECHO_E_HIP, "echo_int8_gemm: %s", hipGetErrorString(e));
    return launched("echo_int8_gemm");
}

}  // extern "C"
