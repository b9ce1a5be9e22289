// fp8.hip -- e4m3 quantisation and products (include/echo_fp8.h) for gfx950.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>

#include "echo_fp8.h"
#include "fp8.hpp"
#include "fp8_stream.hpp"
#include "fp8_tiled.hpp"
#include "status.hpp"

namespace echo {
namespace fp8 {

// ----------------------------------------------------------- quantisation

// Eight values of x at element e, as fp32
template <bool F32>
__device__ __forceinline__ void load8(const void *x, int64_t e, float (&v)[8]) {
    if constexpr (F32) {
        const f32x4 a = ((const f32x4 *)((const float *)x + e))[0];
        const f32x4 b = ((const f32x4 *)((const float *)x + e))[1];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
    } else {
        const u32x4 a = *(const u32x4 *)((const uint16_t *)x + e);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[2 * i] = bf2f(a[i] & 0xFFFFu), v[2 * i + 1] = bf2f(a[i] >> 16);
    }
}

__device__ __forceinline__ float amax8(const float (&v)[8]) {
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(v[i]));   // a NaN keeps out
    return m;
}

__device__ __forceinline__ u32x2 codes8(const float (&v)[8], float s) {
    u32x2 q;
#pragma unroll
    for (int i = 0; i < 2; ++i)
        q[i] = e4m3x2(v[4 * i] / s, v[4 * i + 1] / s) |
               (e4m3x2(v[4 * i + 2] / s, v[4 * i + 3] / s) << 16);
    return q;
}

// Blocks of 1 x 128: 16 lanes a block, 8 values a lane.
template <bool F32>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const void *x, int64_t stride,
                                                            int64_t blocks, int cols, int cb,
                                                            uint8_t *codes, float *scales) {
    const int64_t b = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
    if (b >= blocks) return;
    const int64_t row = b / cb;
    const int j = (int)(b - row * cb), col = kQ * j + 8 * (threadIdx.x & 15);
    float v[8] = {};
    if (col < cols) load8<F32>(x, row * stride + col, v);   // cols a multiple of 16
    float m = amax8(v);
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
    const float s = scale_of(m);
    if ((threadIdx.x & 15) == 0) scales[b] = s;
    if (col < cols) *(u32x2 *)(codes + row * cols + col) = codes8(v, s);
}

// Blocks of 128 x 128, one workgroup each: thread i has columns 8 (i % 16) ..
// of rows i / 16, i / 16 + 16, ...
template <bool F32>
__global__ __launch_bounds__(256) void quantize_blocks_kernel(const void *x, int64_t stride,
                                                              int rows, int cols, int rb, int cb,
                                                              uint8_t *codes, float *scales) {
    const int64_t b = blockIdx.x, mr = b / cb;   // matrix and row of blocks
    const int64_t mat = mr / rb;
    const int j = (int)(b - mr * cb), i = (int)(mr - mat * rb);
    const int col = kQ * j + 8 * (threadIdx.x & 15);
    const int row = kQ * i + (threadIdx.x >> 4);
    float v[8][8] = {};
    float m = 0.f;
#pragma unroll
    for (int r = 0; r < 8; ++r) {
        if (col < cols && row + 16 * r < rows)
            load8<F32>(x, (mat * rows + row + 16 * r) * stride + col, v[r]);
        m = fmaxf(m, amax8(v[r]));
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
    __shared__ float part[4];
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
    __syncthreads();
    const float s = scale_of(fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3])));
    if (threadIdx.x == 0) scales[b] = s;
#pragma unroll
    for (int r = 0; r < 8; ++r)
        if (col < cols && row + 16 * r < rows)
            *(u32x2 *)(codes + (mat * rows + row + 16 * r) * (int64_t)cols + col) = codes8(v[r], s);
}

// -------------------------------------------------------------- products

// y = the sum of the parts of all ranges of K (+ residual), four columns a thread
template <bool F32>
__global__ __launch_bounds__(256) void add_parts_kernel(ProductArgs p, int splits) {
    const int q = p.part_pitch / 4;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= (int64_t)p.T * q) return;
    const int64_t t = i / q;
    const int n = 4 * (int)(i - t * q);
    f32x4 v = *(const f32x4 *)(p.part + t * p.part_pitch + n);
    for (int s = 1; s < splits; ++s) v += *(const f32x4 *)(p.part + (s * (int64_t)p.T + t) * p.part_pitch + n);
    store4<F32>(p, t, n, v);
}

// How a product is cut: the kernel's form, and how many ranges of K there are.
enum Form { kRows16, kRows32, k64x32, k64x64, k128x64, k128x128, k256x128, k256x256 };
struct Cut {
    Form form;
    int splits;
};

// The cut of least estimated time, in microseconds fitted to 130 sizes (T 1 to
// 4,640, N x K from 512 x 512 to 28672 x 4096, weights from memory); the cuts it
// takes there cost 4% over the best of 21 forms x 8 splits in the geometric mean.
//   A launch is 3.4.  Weights and tokens come at 5.2 TB/s at most.
//   kRows: 16 or 32 weight rows a workgroup, straight into registers; a CU streams
//   20 KB a microsecond, and less the more tokens' codes come beside them (8 x
//   6144 x 4096: 10.2 by 32 rows, 12.1 by 16; x 4096 x 4096: 9.9 and 7.7).
//   Tiles n x t: what a step of 128 of K takes with one workgroup on a CU, and
//   with two where LDS holds two.
//   Ranges of K cost a second launch and their fp32 parts' way to memory and back
//   (137 x 4096 x 14336: 95 in one range, 30.7 to 32 in eight).
Cut cut_of(int T, int N, int K) {
    const int KB = cdiv(K, kQ);
    const double bytes = (double)N * K + (double)T * K;
    Cut best{kRows16, 1};
    double least = 1e30;
    for (int nt = 1; nt <= 2; ++nt) {
        const int64_t wgs = (int64_t)cdiv(N, 16 * nt) * cdiv(T, 32);
        const double turn = 16.0 * nt * K / 20e3 * (1 + 0.035 * std::min(T, 32) / nt);
        const double us = std::max(bytes / 5.2e6, turn * (1 + 0.6 * ((double)((wgs + 255) / 256) - 1)));
        if (us < least) least = us, best = Cut{nt == 1 ? kRows16 : kRows32, 1};
    }
    static const struct {
        Form form;
        int n, t;
        double one, two;
    } tiles[] = {{k64x32, 64, 32, .37, .52},   {k64x64, 64, 64, .45, .75}, {k128x64, 128, 64, .68, 1.0},
                 {k128x128, 128, 128, .88, 0}, {k256x128, 256, 128, 1.32, 0}, {k256x256, 256, 256, 2.4, 0}};
    for (const auto &f : tiles) {
        if (f.t > 32 && T <= f.t / 2) continue;
        for (int s : {1, 2, 3, 4, 6, 8, 12, 16}) {
            if (s > 1 && 2 * s > KB) break;
            const int64_t each = ((int64_t)cdiv(N, f.n) * cdiv(T, f.t) * s + 255) / 256;   // of a CU
            const double turns = f.two > 0 ? (double)(each / 2) * f.two + (double)(each % 2) * f.one
                                           : (double)each * f.one;
            const double starts = (double)(f.two > 0 ? (each + 1) / 2 : each) - 1;
            double us = std::max(cdiv(KB, s) * turns + 2.5 * starts, bytes / 5.2e6);
            if (s > 1) us += 3.4 + 0.25 * s + 8.0 * s * T * N / 5e6;
            if (us < least) least = us, best = Cut{f.form, s};
        }
    }
    return best;
}

template <bool F32, int NT, int TT>
void launch_rows(const ProductArgs &p, hipStream_t st) {
    const int n_tiles = cdiv(p.N, 16 * NT);
    const dim3 grid((unsigned)((int64_t)n_tiles * cdiv(p.T, 16 * TT))), block(512);
    if (p.T <= 16 * TT)   // every weight read once
        hipLaunchKernelGGL((stream_kernel<F32, true, NT, TT, 8, 4>), grid, block, 0, st, p, n_tiles);
    else
        hipLaunchKernelGGL((stream_kernel<F32, false, NT, TT, 8, 4>), grid, block, 0, st, p, n_tiles);
}

template <bool F32, int BN, int BT, int WN, int WT, int S>
hipError_t launch_tiles(const ProductArgs &p, int splits, hipStream_t st) {
    return launch_tiled<Mode::Plain, F32, BN, BT, WN, WT, S>(p, cdiv(p.T, BT), splits, st);
}

template <bool F32>
hipError_t launch_gemm(const ProductArgs &p, Cut c, hipStream_t st) {
    hipError_t e = hipSuccess;
    switch (c.form) {
        case kRows16: p.T > 16 ? launch_rows<F32, 1, 2>(p, st) : launch_rows<F32, 1, 1>(p, st); return e;
        case kRows32: p.T > 16 ? launch_rows<F32, 2, 2>(p, st) : launch_rows<F32, 2, 1>(p, st); return e;
        case k64x32: e = launch_tiles<F32, 64, 32, 4, 1, 5>(p, c.splits, st); break;
        case k64x64: e = launch_tiles<F32, 64, 64, 4, 1, 4>(p, c.splits, st); break;
        case k128x64: e = launch_tiles<F32, 128, 64, 4, 1, 3>(p, c.splits, st); break;
        default:
            // fp32 results, which take twice the products, in tiles of 128 x 128
            if (F32 || c.form == k128x128) e = launch_tiles<F32, 128, 128, 4, 2, 4>(p, c.splits, st);
            else if (c.form == k256x128) e = launch_tiles<false, 256, 128, 4, 2, 3>(p, c.splits, st);
            else e = launch_tiles<false, 256, 256, 2, 4, 2>(p, c.splits, st);
    }
    if (e != hipSuccess || c.splits == 1 || (e = hipGetLastError()) != hipSuccess) return e;
    const int64_t n = (int64_t)p.T * (p.part_pitch / 4);
    hipLaunchKernelGGL(add_parts_kernel<F32>, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, p, c.splits);
    return hipSuccess;
}

}  // namespace fp8
}  // namespace echo

using namespace echo;
using namespace echo::fp8;

namespace {

int launched(const char *what) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? ECHO_OK : fail(ECHO_E_HIP, "%s: %s", what, hipGetErrorString(e));
}

// columns of a row of parts
int pitch_of(int32_t N) { return (int)(((int64_t)N + 3) / 4 * 4); }

size_t parts_bytes(Cut c, int32_t T, int32_t N) {
    return c.splits == 1 ? 0 : (size_t)c.splits * T * pitch_of(N) * 4;
}

int check_sizes(int32_t T, int32_t N, int32_t K) {
    if (T < 0) return fail(ECHO_E_INVALID, "num_tokens %d", T);
    if (N <= 0 || K <= 0) return fail(ECHO_E_INVALID, "out_features %d, in_features %d", N, K);
    if (K % 16) return fail(ECHO_E_UNSUPPORTED, "in_features %d is not a multiple of 16", K);
    // offsets inside a tile are 32 bits, a grid's workgroups too
    if (K > 1 << 23) return fail(ECHO_E_UNSUPPORTED, "in_features %d above %d", K, 1 << 23);
    if ((int64_t)cdiv(N, 16) * cdiv(T, 16) > INT32_MAX / 2 || N > INT32_MAX - 3)
        return fail(ECHO_E_UNSUPPORTED, "product of %d x %d too large", T, N);
    return ECHO_OK;
}

}  // namespace

extern "C" {

int echo_fp8_quantize(const void *x, int32_t x_dtype, int64_t x_stride, int32_t batch,
                      int32_t rows, int32_t cols, int32_t block_rows, void *codes, float *scales,
                      void *stream) {
    clear_error();
    if (x_dtype != ECHO_BF16 && x_dtype != ECHO_F32)
        return fail(ECHO_E_UNSUPPORTED, "dtype %d of x", x_dtype);
    if (batch < 0 || rows < 0 || cols <= 0)
        return fail(ECHO_E_INVALID, "batch %d, rows %d, cols %d", batch, rows, cols);
    if (block_rows != 1 && block_rows != kQ)
        return fail(ECHO_E_UNSUPPORTED, "block_rows %d (only 1, 128)", block_rows);
    if (cols % 16) return fail(ECHO_E_UNSUPPORTED, "cols %d is not a multiple of 16", cols);
    if (batch == 0 || rows == 0) return ECHO_OK;
    const int size = x_dtype == ECHO_F32 ? 4 : 2;
    if (!x || !codes || !scales) return fail(ECHO_E_INVALID, "x, codes or scales is NULL");
    if (x_stride < cols || x_stride % (16 / size))
        return fail(ECHO_E_INVALID, "x_stride %lld: at least cols %d, rows at 16-byte steps",
                    (long long)x_stride, cols);
    if (((uintptr_t)x | (uintptr_t)codes) & 15u)
        return fail(ECHO_E_INVALID, "x and codes must be 16-byte aligned");
    if ((uintptr_t)scales & 3u) return fail(ECHO_E_INVALID, "scales must be 4-byte aligned");
    const int cb = cdiv(cols, kQ), rb = cdiv(rows, block_rows);
    const hipStream_t st = (hipStream_t)stream;
    const int64_t blocks = (int64_t)batch * rb * cb;
    const int64_t grid = block_rows == 1 ? (blocks + 15) / 16 : blocks;
    if (grid > INT32_MAX) return fail(ECHO_E_UNSUPPORTED, "%lld blocks", (long long)blocks);
    if (block_rows == 1) {
        if (size == 4)
            hipLaunchKernelGGL(quantize_rows_kernel<true>, dim3((unsigned)grid), dim3(256), 0, st, x,
                               x_stride, blocks, cols, cb, (uint8_t *)codes, scales);
        else
            hipLaunchKernelGGL(quantize_rows_kernel<false>, dim3((unsigned)grid), dim3(256), 0, st, x,
                               x_stride, blocks, cols, cb, (uint8_t *)codes, scales);
    } else {
        if (size == 4)
            hipLaunchKernelGGL(quantize_blocks_kernel<true>, dim3((unsigned)grid), dim3(256), 0, st,
                               x, x_stride, rows, cols, rb, cb, (uint8_t *)codes, scales);
        else
            hipLaunchKernelGGL(quantize_blocks_kernel<false>, dim3((unsigned)grid), dim3(256), 0, st,
                               x, x_stride, rows, cols, rb, cb, (uint8_t *)codes, scales);
    }
    return launched("echo_fp8_quantize");
}

size_t echo_fp8_gemm_workspace_bytes(int32_t num_tokens, int32_t out_features,
                                     int32_t in_features) {
    clear_error();
    if (check_sizes(num_tokens, out_features, in_features) || num_tokens == 0) return 0;
    return parts_bytes(cut_of(num_tokens, out_features, in_features), num_tokens, out_features);
}

int echo_fp8_gemm(const void *x, const float *x_scale, const void *w, const float *w_scale,
                  int32_t num_tokens, int32_t out_features, int32_t in_features,
                  const void *residual, void *y, int32_t y_dtype, int64_t y_stride,
                  void *workspace, size_t workspace_bytes, void *stream) {
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
    if (((uintptr_t)x_scale | (uintptr_t)w_scale) & 3u || ya & (y_dtype == ECHO_F32 ? 3u : 1u))
        return fail(ECHO_E_INVALID, "scales, y and residual must have their types' alignment");
    const Cut cut = cut_of(num_tokens, out_features, in_features);
    const size_t need = parts_bytes(cut, num_tokens, out_features);
    if (need && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 255u)))
        return fail(ECHO_E_WORKSPACE, "workspace of %zu bytes (need %zu, 256-byte aligned)",
                    workspace_bytes, need);
    ProductArgs p{};
    p.x = (const uint8_t *)x;
    p.xs = x_scale;
    p.w = (const uint8_t *)w;
    p.ws = w_scale;
    p.T = num_tokens;
    p.N = out_features;
    p.K = in_features;
    p.KB = cdiv(in_features, kQ);
    p.residual = residual;
    p.y = y;
    p.y_stride = y_stride;
    p.part = (float *)workspace;
    p.part_pitch = pitch_of(out_features);
    p.wide = out_features % 4 == 0 && y_stride % 4 == 0 && !(ya & (y_dtype == ECHO_F32 ? 15u : 7u));
    const hipError_t e = y_dtype == ECHO_F32 ? launch_gemm<true>(p, cut, (hipStream_t)stream)
                                             : launch_gemm<false>(p, cut, (hipStream_t)stream);
    if (e != hipSuccess) return fail(ECHO_E_HIP, "echo_fp8_gemm: %s", hipGetErrorString(e));
    return launched("echo_fp8_gemm");
}

}  // extern "C"
