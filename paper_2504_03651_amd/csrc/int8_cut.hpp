// int8_cut.hpp -- how a product in 8-bit integers is cut: the kernel's form and the ranges
// of K (host code only).
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <algorithm>

namespace echo {
namespace int8 {

constexpr int kStep = 128;   // bytes of a row that a step of a product takes

inline int cuts(int64_t n, int64_t each) { return (int)((n + each - 1) / each); }

constexpr int rows_tokens(int T) { return T <= 8 ? 8 : T <= 16 ? 16 : 32; }

// How a product is cut: the kernel's form, and how many ranges of K there are.
enum Form { kRows16, kRows32, k64x32, k64x64, k128x64, k128x96, k128x128, k128x128two, k128x160, k256x128, k256x192 };
struct Cut {
    Form form;
    int ranges;
};

// Tiles n x t, in microseconds: what a step of 128 of K takes with one workgroup on a CU,
// and with two where LDS holds two; the launch; going on to another tile
constexpr struct {
    Form form;
    int n, t;
    double one, two, launch, on;
} kTileForms[] = {{k64x32, 64, 32, .25, .42, 3.1, 2.},       {k64x64, 64, 64, .27, .41, 3.8, 2.},
                  {k128x64, 128, 64, .54, .75, 3.75, 2.},    {k128x96, 128, 96, .53, 0, 3.7, 2.},
                  {k128x128, 128, 128, .59, 0, 3.75, 2.},    {k128x128two, 128, 128, .70, .85, 3.55, 1.7},
                  {k128x160, 128, 160, .72, 0, 3.5, 2.},     {k256x128, 256, 128, .77, 0, 3.7, 2.},
                  {k256x192, 256, 192, 1.15, 0, 4., 3.4}};
// (sums of ranges in tiles of 256 x 192 would spill registers)
constexpr bool in_ranges(Form f) { return f != k256x192; }
constexpr int kRanges[] = {1, 2, 3, 4, 6, 8, 12, 16};

// Products of more tiles, or whose parts would take more, are not cut into ranges of K,
// so that there is a bound on the parts of every product of up to T tokens.
constexpr int kRangeTiles = 2048;
constexpr size_t kPartBytes = 256u << 20;

// columns of a row of parts
inline int pitch_of(int N) { return (int)(((int64_t)N + 3) / 4 * 4); }
inline size_t parts_bytes(int ranges, int T, int N) { return ranges == 1 ? 0 : (size_t)ranges * T * pitch_of(N) * 4; }

// The most bytes of parts of up to T tokens.  A form's tiles in s ranges are at most
// kRangeTiles: with m = kRangeTiles / its tiles of N, s times its tiles of tokens is at
// most m, and s times the tokens at most m t.
inline size_t most_parts_bytes(int T, int N, int K) {
    int s_most = 1;
    for (int s : kRanges)
        if (2 * s <= cuts(K, kStep)) s_most = s;
    int64_t rows = 0;   // s times the tokens
    for (const auto &f : kTileForms) {
        const int m = kRangeTiles / cuts(N, f.n);
        if (m > 1 && s_most > 1 && in_ranges(f.form)) rows = std::max(rows, std::min((int64_t)std::min(s_most, m) * T, (int64_t)m * f.t));
    }
    return std::min<size_t>((size_t)rows * pitch_of(N) * 4, kPartBytes);
}

// The cut of least estimated time, in microseconds fitted to bf16 results of 430 sizes (T 1
// to 4,640, N 64 to 28,672, K 128 to 14,336, weights from memory).  In the 395 of them whose
// cut was timed it is 1.2% (geometric mean) above the best cut of each, 38% at most (46 x 128
// x 10912: 8.6 us, by 16 weight rows 6.5, whose price is too high where there are few of
// them; then 24%, 20 x 17342 x 8256, 48 us, in four ranges of K 38); over 130 sizes with fp32
// results 1.2% and 35% (54 x 5152 x 8080).
//   Weights and tokens come at 5.0 TB/s at most.
//   kRows: 16 or 32 weight rows a workgroup, every wave on its own; one workgroup a
//   CU, which takes in 70 KB a microsecond, tokens among them (8 x 6144 x 4096, launches
//   one after the other: 7.2 by 32 rows, 9.1 by 16; 64 x 32 tiles take over where a CU has
//   more than one: 8 x 10911 x 3056 13.0, by 32 rows 14.3).
//   k128x128two: four waves of 64 x 64, two workgroups a CU, so that one's results leave
//   beside the other's products (1,847 x 26626 x 512 53 us, in tiles of 256 x 192 73, of
//   128 x 128 by eight waves, four stages and one workgroup a CU, which ranges of K and
//   few tiles take, 71).
//   Ranges of K cost a second launch and their sums' way to memory and back.
inline Cut cut_of(int T, int N, int K, bool f32) {
    const int KB = cuts(K, kStep);
    const double bytes = (double)N * K + (double)T * K;
    Cut best{kRows16, 1};
    double least = 1e30;
    for (int nt = 1; nt <= 2; ++nt) {
        const int x = rows_tokens(T);
        const int64_t turns = ((int64_t)cuts(N, 16 * nt) * cuts(T, x > 16 ? 32 : 16) + 255) / 256;
        if (turns >= 1 << 14) continue;   // a launch has fewer than 2^32 threads
        const double us = std::max(bytes / 5.0e6, (double)turns * (16 * nt + x) * K / 70e3) + 2.6 +
                          1.5 * (double)(turns - 1);
        if (us < least) least = us, best = Cut{nt == 1 ? kRows16 : kRows32, 1};
    }
    for (const auto &f : kTileForms) {
        if ((f.t > 32 && T <= f.t / 3) || (f32 && (f.form == k128x128two || f.form == k256x192))) continue;
        for (int s : kRanges) {
            const int64_t all = (int64_t)cuts(N, f.n) * cuts(T, f.t) * s;
            if (s > 1 && (!in_ranges(f.form) || 2 * s > KB || all > kRangeTiles || parts_bytes(s, T, N) > kPartBytes)) break;
            const int64_t each = (all + 255) / 256;   // of a CU
            const double one = f.form == k128x160 && T <= 160 ? .62 : f.one;   // waves of 16 x 160
            const double turns = f.two > 0 ? (double)(each / 2) * f.two + (double)(each % 2) * one
                                           : (double)each * one;
            const double on = f.on * (double)((f.two > 0 ? (each + 1) / 2 : each) - 1);
            double us = std::max(cuts(KB, s) * turns + on, bytes / 5.0e6) + f.launch;
            if (s > 1) us += 2.6 + 0.19 * s + 8.0 * s * T * N / 5.0e6;
            if (us < least) least = us, best = Cut{f.form, s};
        }
    }
    return best;
}

}  // namespace int8
}  // namespace echo
