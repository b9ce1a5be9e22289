// fp8.hip -- e4m3 quantisation and products (include/echo_fp8.h) for gfx950.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>

#include "echo_fp8.h"
#include "fp8.hpp"
#include "fp8_stream.hpp"
#include "status.hpp"

namespace echo {
namespace fp8 {

// ----------------------------------------------------------- quantisation

// Codes are those of correctly rounded quotients.  For a bf16 value and a scale in
// [2^-100, 2^100] one multiplication by r = RN(1 / s) and one corrected by its exact
// residual (Markstein) give the same code for every value there is and every
// scale fp32(b / 448) of a bf16 b; fp32 values are divided.  A block's largest
// magnitude is found among the bits, where a NaN is larger than all else: blocks
// with a NaN or a scale outside that range take the general form, and no quotient
// of the others is past 448 by more than a rounding, so nothing needs clamping.  66.5 million
// bf16 activations take 36 us, 5.6 TB/s (by division, clamped and with 64-bit
// indices 54), a matrix of 117 million in blocks of 128 x 128 68 (101); fp32 ones 62
// and 104 us, 5.4 and 5.6 TB/s.

// Eight values as they lie in memory
template <bool F32>
struct Eight {
    u32x4 a[F32 ? 2 : 1];
    __device__ __forceinline__ void load(const void *x, int64_t e) {
        const u32x4 *q = (const u32x4 *)((const uint8_t *)x + e * (F32 ? 4 : 2));
#pragma unroll
        for (int i = 0; i < (F32 ? 2 : 1); ++i) a[i] = q[i];
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < (F32 ? 2 : 1); ++i) a[i] = (u32x4){0u, 0u, 0u, 0u};
    }
    __device__ __forceinline__ float get(int i) const {
        if constexpr (F32) return __uint_as_float(a[i / 4][i % 4]);
        return __uint_as_float(i & 1 ? a[0][i / 2] & 0xFFFF0000u : a[0][i / 2] << 16);
    }
    // bits of the largest magnitude, as fp32: above infinity's with a NaN
    __device__ __forceinline__ uint32_t top() const {
        if constexpr (F32) {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) m = max(m, a[i / 4][i % 4] & 0x7FFFFFFFu);
            return m;
        }
        typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
        u16x2 m = {0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i)
            m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, a[0][i] & 0x7FFF7FFFu));
        return (uint32_t)max(m[0], m[1]) << 16;
    }
    // the largest magnitude of those that are no NaN
    __device__ __forceinline__ float amax() const {
        float m = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(get(i)));
        return m;
    }
    __device__ __forceinline__ u32x2 codes(float s, float r, bool plain) const {
        u32x2 q;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float x = get(4 * h + i);
                if (F32 || !plain) {
                    v[i] = x / s;
                } else {
                    const float q0 = x * r;
                    v[i] = __builtin_copysignf(__builtin_fmaf(__builtin_fmaf(-q0, s, x), r, q0), x);
                }
            }
            if (plain) {
                int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
                w = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], w, true);
                q[h] = (uint32_t)w;
            } else {
                q[h] = e4m3x2(v[0], v[1]) | (e4m3x2(v[2], v[3]) << 16);
            }
        }
        return q;
    }
};

// max over the 16 lanes of a row of the wave
__device__ __forceinline__ uint32_t max16(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xF, 0xF, false));   // row_ror:8
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x124, 0xF, 0xF, false));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x122, 0xF, 0xF, false));
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x121, 0xF, 0xF, false));
}

// whether a block's scale s, of the top bits t, takes the plain form (a subnormal
// scale is rounded too coarsely for quotients to end at 448)
__device__ __forceinline__ bool plain_block(uint32_t t, float s) {
    return t < 0x7F800000u && s >= 0x1p-100f && s <= 0x1p100f;
}

// Blocks of 1 x 128: 16 lanes a block, 8 values a lane, two blocks at a time; a
// workgroup has 32 blocks of one row.  first: of the launch's workgroups, in all.
template <bool F32>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const void *x, int64_t stride, int cols,
                                                            int cb, int parts, uint8_t *codes,
                                                            float *scales, uint32_t first) {
    const uint32_t b = first + blockIdx.x;
    const int64_t row = b / parts;
    const int j0 = 32 * (int)(b - row * parts) + (threadIdx.x >> 4);
    const int lane8 = 8 * (threadIdx.x & 15);
    Eight<F32> v[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int col = kQ * (j0 + 16 * u) + lane8;
        if (col < cols) v[u].load(x, row * stride + col);   // cols a multiple of 16
        else v[u].zero();
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int j = j0 + 16 * u, col = kQ * j + lane8;
        const uint32_t t = max16(v[u].top());
        float s = scale_of(__uint_as_float(t));
        const bool plain = plain_block(t, s);
        u32x2 q;
        if (__all(plain)) {
            q = v[u].codes(s, 1.0f / s, true);
        } else {
            if (t > 0x7F800000u) s = scale_of(__uint_as_float(max16(__float_as_uint(v[u].amax()))));
            q = v[u].codes(s, 0.f, false);
        }
        if (j < cb && lane8 == 0) scales[row * cb + j] = s;
        if (col < cols) *(u32x2 *)(codes + row * cols + col) = q;
    }
}

// Blocks of 128 x 128, one workgroup each: thread i has columns 8 (i % 16) ..
// of rows i / 16, i / 16 + 16, ...
template <bool F32>
__global__ __launch_bounds__(256) void quantize_blocks_kernel(const void *x, int64_t stride,
                                                              int rows, int cols, int rb, int cb,
                                                              uint8_t *codes, float *scales, uint32_t first) {
    const int64_t b = first + blockIdx.x, mr = b / cb;   // matrix and row of blocks
    const int64_t mat = mr / rb;
    const int j = (int)(b - mr * cb), i = (int)(mr - mat * rb);
    const int col = kQ * j + 8 * (threadIdx.x & 15);
    const int row = kQ * i + (threadIdx.x >> 4);
    __shared__ uint32_t part[16];
    auto all_max = [&](uint32_t t) {   // of the workgroup
        t = max16(t);
        __syncthreads();
        if ((threadIdx.x & 15) == 0) part[threadIdx.x >> 4] = t;
        __syncthreads();
        return max16(part[threadIdx.x & 15]);
    };
    Eight<F32> v[8];
    uint32_t t = 0;
#pragma unroll
    for (int r = 0; r < 8; ++r) {
        if (col < cols && row + 16 * r < rows) v[r].load(x, (mat * rows + row + 16 * r) * stride + col);
        else v[r].zero();
    }
#pragma unroll
    for (int r = 0; r < 8; ++r) t = max(t, v[r].top());
    t = all_max(t);
    float s = scale_of(__uint_as_float(t));
    const bool plain = plain_block(t, s);
    if (t > 0x7F800000u) {
        float m = 0.f;
#pragma unroll
        for (int r = 0; r < 8; ++r) m = fmaxf(m, v[r].amax());
        s = scale_of(__uint_as_float(all_max(__float_as_uint(m))));
    }
    const float inv = 1.0f / s;
    if (threadIdx.x == 0) scales[b] = s;
    auto store = [&](int r, u32x2 q) {
        if (col < cols && row + 16 * r < rows)
            *(u32x2 *)(codes + (mat * rows + row + 16 * r) * (int64_t)cols + col) = q;
    };
    if (plain) {
#pragma unroll
        for (int r = 0; r < 8; ++r) store(r, v[r].codes(s, inv, true));
    } else {
#pragma unroll
        for (int r = 0; r < 8; ++r) store(r, v[r].codes(s, inv, false));
    }
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

// stages of a wave's ring, for NT = 1 and 2
constexpr int rows_depth(int NT, int XR) {
    return XR == 8 ? (NT == 1 ? 5 : 3) : XR == 16 ? (NT == 1 ? 4 : 3) : NT == 1 ? 3 : 2;
}
constexpr int rows_tokens(int T) { return T <= 8 ? 8 : T <= 16 ? 16 : 32; }
bool rows_fit(int NT, int T, int K) {
    const int XR = rows_tokens(T);
    return stream_bytes(NT, XR, rows_depth(NT, XR), cdiv(cdiv(K, kQ), kStreamWaves)) * kStreamWaves <= 160 * 1024;
}

// How a product is cut: the kernel's form, and how many ranges of K there are.
enum Form { kRows16, kRows32, k64x32, k64x64, k128x64, k128x128, k256x128, k256x256 };
struct Cut {
    Form form;
    int splits;
};

// Tiles n x t: what a step of 128 of K takes with one workgroup on a CU, and with two
// where LDS holds two
constexpr struct {
    Form form;
    int n, t;
    double one, two;
} kTileForms[] = {{k64x32, 64, 32, .37, .52},   {k64x64, 64, 64, .45, .75}, {k128x64, 128, 64, .68, 1.0},
                  {k128x128, 128, 128, .88, 0}, {k256x128, 256, 128, 1.32, 0}, {k256x256, 256, 256, 2.4, 0}};
constexpr int kRanges[] = {1, 2, 3, 4, 6, 8, 12, 16};

// Products of more tiles, or whose parts would take more, are not cut into ranges of K
// (of 2 million sizes of K up to 19,200 none would be), so that there is a bound on
// the parts of every product of up to T tokens.
constexpr int kRangeTiles = 2048;
constexpr size_t kPartBytes = 256u << 20;

// columns of a row of parts
int pitch_of(int N) { return (int)(((int64_t)N + 3) / 4 * 4); }
size_t parts_bytes(int splits, int T, int N) { return splits == 1 ? 0 : (size_t)splits * T * pitch_of(N) * 4; }

// The most bytes of parts of up to T tokens.  A form's tiles in s ranges are at most
// kRangeTiles: with m = kRangeTiles / its tiles of N, s times its tiles of tokens is at
// most m, and s times the tokens at most m t.
size_t most_parts_bytes(int T, int N, int K) {
    int s_most = 1;
    for (int s : kRanges)
        if (2 * s <= cdiv(K, kQ)) s_most = s;
    int64_t rows = 0;   // s times the tokens
    for (const auto &f : kTileForms) {
        const int m = kRangeTiles / cdiv(N, f.n);
        if (m > 1 && s_most > 1) rows = std::max(rows, std::min((int64_t)std::min(s_most, m) * T, (int64_t)m * f.t));
    }
    return std::min<size_t>((size_t)rows * pitch_of(N) * 4, kPartBytes);
}

// The cut of least estimated time, in microseconds fitted to bf16 results of 130 sizes
// (T 1 to 4,640, N x K from 512 x 512 to 28672 x 4096, weights from memory).  Over 144
// sizes of today's kernels it is 1.6% (geometric mean) above the best cut of each,
// 29% at most (80 to 96 x 4096 x 4096, where rows would be best), over 60 with fp32
// results 2.8% and 34%.
//   Weights and tokens come at 5.2 TB/s at most.
//   kRows: 16 or 32 weight rows a workgroup, every wave on its own; one workgroup a
//   CU, which takes in 50 KB a microsecond, tokens among them (8 x 6144 x 4096: 8.5
//   by 32 rows, 11.1 by 16; 8 x 4096 x 4096: 8.1 and 7.4).
//   Ranges of K cost a second launch and their fp32 parts' way to memory and back
//   (137 x 4096 x 14336: 125 in one range, 33 in eight, 41 in sixteen).
Cut cut_of(int T, int N, int K) {
    const int KB = cdiv(K, kQ);
    const double bytes = (double)N * K + (double)T * K;
    Cut best{kRows16, 1};
    double least = 1e30;
    for (int nt = 1; nt <= 2; ++nt) {
        if (!rows_fit(nt, T, K)) continue;
        const int x = rows_tokens(T);
        const int64_t turns = ((int64_t)cdiv(N, 16 * nt) * cdiv(T, x > 16 ? 32 : 16) + 255) / 256;
        if (turns >= 1 << 15) continue;   // a launch has fewer than 2^32 threads
        const double us = std::max(bytes / 5.2e6, (double)turns * (16 * nt + x) * K / 50e3) + 0.6 +
                          1.5 * (double)(turns - 1);
        if (us < least) least = us, best = Cut{nt == 1 ? kRows16 : kRows32, 1};
    }
    for (const auto &f : kTileForms) {
        if (f.t > 32 && T <= f.t / 2) continue;
        for (int s : kRanges) {
            const int64_t all = (int64_t)cdiv(N, f.n) * cdiv(T, f.t) * s;
            if (s > 1 && (2 * s > KB || all > kRangeTiles || parts_bytes(s, T, N) > kPartBytes)) break;
            const int64_t each = (all + 255) / 256;   // of a CU
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

template <bool F32, int NT>
hipError_t launch_rows(const ProductArgs &p, hipStream_t st) {
    switch (rows_tokens(p.T)) {   // up to 32 tokens every weight is read once
        case 8: return launch_stream<F32, true, NT, 8, rows_depth(NT, 8)>(p, st);
        case 16: return launch_stream<F32, true, NT, 16, rows_depth(NT, 16)>(p, st);
        default:
            return p.T <= 32 ? launch_stream<F32, true, NT, 32, rows_depth(NT, 32)>(p, st)
                             : launch_stream<F32, false, NT, 32, rows_depth(NT, 32)>(p, st);
    }
}

template <bool F32, int BN, int BT, int WN, int WT, int S>
hipError_t launch_tiles(const ProductArgs &p, int splits, hipStream_t st) {
    if constexpr (BT <= 64)
        if (p.T <= BT) return launch_tiled<Mode::Plain, F32, true, BN, BT, WN, WT, S>(p, 1, splits, st);
    return launch_tiled<Mode::Plain, F32, false, BN, BT, WN, WT, S>(p, cdiv(p.T, BT), splits, st);
}

template <bool F32>
hipError_t launch_gemm(const ProductArgs &p, Cut c, hipStream_t st) {
    hipError_t e = hipSuccess;
    switch (c.form) {
        case kRows16: return launch_rows<F32, 1>(p, st);
        case kRows32: return launch_rows<F32, 2>(p, st);
        case k64x32: e = launch_tiles<F32, 64, 32, 4, 1, 5>(p, c.splits, st); break;
        case k64x64: e = launch_tiles<F32, 64, 64, 4, 1, 4>(p, c.splits, st); break;
        default:
            // fp32 results, which widen every operand that a wave reads, in waves of
            // 64 x 64, two workgroups a CU (4,640 x 4096 x 4096: 178 us, in tiles of 128 x
            // 64 with waves of 32 x 64 214; 1,024 x 6144 x 4096 69 and 66)
            if (c.form == k128x64) e = launch_tiles<F32, 128, 64, 4, 1, 3>(p, c.splits, st);
            else if (F32) e = launch_tiles<true, 128, 128, 2, 2, 2>(p, c.splits, st);
            else if (c.form == k128x128) e = launch_tiles<false, 128, 128, 4, 2, 4>(p, c.splits, st);
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

int check_sizes(int32_t T, int32_t N, int32_t K) {
    if (T < 0) return fail(ECHO_E_INVALID, "num_tokens %d", T);
    if (N <= 0 || K <= 0) return fail(ECHO_E_INVALID, "out_features %d, in_features %d", N, K);
    if (K % 16) return fail(ECHO_E_UNSUPPORTED, "in_features %d is not a multiple of 16", K);
    // offsets inside a tile are 32 bits, a grid's workgroups too
    if (K > 1 << 23) return fail(ECHO_E_UNSUPPORTED, "in_features %d above %d", K, 1 << 23);
    if ((int64_t)cdiv(N, 16) * cdiv(T, 16) > INT32_MAX / 2 || N > 1 << 30 || T > 1 << 30)
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
    const int parts = cdiv(cb, 32);   // workgroups of a row
    const int64_t grid = block_rows == 1 ? (int64_t)batch * rows * parts : blocks;
    if (grid > INT32_MAX) return fail(ECHO_E_UNSUPPORTED, "%lld blocks", (long long)blocks);
    // a launch has fewer than 2^32 threads
    constexpr int64_t kMost = 1 << 23;
    for (int64_t first = 0; first < grid; first += kMost) {
        const dim3 groups((unsigned)std::min(kMost, grid - first)), threads(256);
        if (block_rows == 1) {
            if (size == 4)
                hipLaunchKernelGGL(quantize_rows_kernel<true>, groups, threads, 0, st, x, x_stride, cols, cb,
                                   parts, (uint8_t *)codes, scales, (uint32_t)first);
            else
                hipLaunchKernelGGL(quantize_rows_kernel<false>, groups, threads, 0, st, x, x_stride, cols, cb,
                                   parts, (uint8_t *)codes, scales, (uint32_t)first);
        } else {
            if (size == 4)
                hipLaunchKernelGGL(quantize_blocks_kernel<true>, groups, threads, 0, st, x, x_stride, rows,
                                   cols, rb, cb, (uint8_t *)codes, scales, (uint32_t)first);
            else
                hipLaunchKernelGGL(quantize_blocks_kernel<false>, groups, threads, 0, st, x, x_stride, rows,
                                   cols, rb, cb, (uint8_t *)codes, scales, (uint32_t)first);
        }
        const int rc = launched("echo_fp8_quantize");
        if (rc) return rc;
    }
    return ECHO_OK;
}

size_t echo_fp8_gemm_workspace_bytes(int32_t num_tokens, int32_t out_features,
                                     int32_t in_features) {
    clear_error();
    if (check_sizes(num_tokens, out_features, in_features) || num_tokens == 0) return 0;
    return most_parts_bytes(num_tokens, out_features, in_features);
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
    const size_t need = most_parts_bytes(num_tokens, out_features, in_features);
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
    const hipError_t e = y_dtype == ECHO_F32 ? launch_gemm<true>(p, cut, (hipStream_t)stream)
                                             : launch_gemm<false>(p, cut, (hipStream_t)stream);
    if (e != hipSuccess) return fail(ECHO_E_HIP, "echo_fp8_gemm: %s", hipGetErrorString(e));
    return launched("echo_fp8_gemm");
}

}  // extern "C"
