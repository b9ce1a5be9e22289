// How the library cuts products in 8-bit integers: for each line "T N K f32" of the input
// the kernel's form, the ranges of K, the form's variant (kernels that are compiled apart)
// and the bytes of the ranges' sums, and the workspace for up to T tokens.
#include <cstdio>

#include "int8_cut.hpp"

using namespace echo::int8;

static int variant(Cut c, int T) {
    if (c.form == kRows16 || c.form == kRows32) return T > 32 ? 33 : rows_tokens(T);
    if (c.form == k128x160) return T <= 160;
    for (const auto &f : kTileForms)
        if (f.form == c.form) return f.t <= 64 && T <= f.t;
    return -1;
}

int main() {
    static const char *names[] = {"rows16", "rows32", "64x32", "64x64", "128x64", "128x96", "128x128", "128x128two", "128x160", "256x128", "256x192"};
    int T, N, K, f32;
    while (std::scanf("%d %d %d %d", &T, &N, &K, &f32) == 4) {
        const Cut c = cut_of(T, N, K, f32);
        std::printf("%s %d %d %zu %zu\n", names[c.form], c.ranges, variant(c, T), parts_bytes(c.ranges, T, N), most_parts_bytes(T, N, K));
    }
}
