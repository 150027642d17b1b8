// CPU-only checker of the norms' layouts (norm_layout.h): for widths, strides and numbers of rows over the whole range, every lane's pieces lie in
// the row and cover it once, and the kernels' offsets are those in 64 bits.  Compiled with g++ -fsanitize=address,undefined and
// run by the CPU test suite, one part for each argument.
#include <stdio.h>
#include <string.h>

#include <vector>

#include "norm_layout.h"

using namespace gas;

static int failures = 0, checked = 0;
#define CHECK(cond, ...)                                   \
    do {                                                   \
        if (!(cond)) {                                     \
            if (++failures <= 20) {                        \
                fprintf(stderr, "FAIL %s:%d: ", __FILE__, __LINE__); \
                fprintf(stderr, __VA_ARGS__);              \
                fprintf(stderr, "\n");                     \
            }                                              \
            return;                                        \
        }                                                  \
    } while (0)

template <int E, bool MASK, int P>
static void lanes(const Layout& l, int F, int64_t n, int64_t ld, bool offsets, const char* what) {
    constexpr int EB = 16 / E;
    const bool tiny = MASK && l.g == 1;
    std::vector<int> times(F, 0);
    for (int index = 0; index < l.g * l.w; ++index)
        for (int i = 0; i < P; ++i) {
            const Piece p = piece_of<E, MASK, P>(index + i * l.g * l.w, i, F);
            CHECK(tiny || (p.c >= 0 && p.c + E <= F), "%s: F=%d ld=%lld, %d lanes: lane %d loads the elements from %d on", what, F, (long long)ld, l.g, index, p.c);
            CHECK(!tiny || p.c + p.skip >= 0, "%s: F=%d: a narrow row's elements from %d on", what, F, p.c + p.skip);
            if (p.on)
                for (int e = p.skip; e < E; ++e) {
                    CHECK(p.c + e >= 0 && p.c + e < F, "%s: F=%d, lane %d has element %d", what, F, index, p.c + e);
                    ++times[p.c + e];
                }
            if (offsets)
                for (int team = 0; team < 64 / l.g && team < n; ++team) {
                    const int64_t want = (team * ld + p.c) * EB, got = tiny ? tiny_offset<EB>(team, ld, p.c) : (int64_t)piece_offset<EB>(team, ld, p.c);
                    CHECK(got == want, "%s: F=%d ld=%lld, %d lanes, row %d, element %d: %lld bytes, not %lld", what, F, (long long)ld, l.g, team, p.c,
                          (long long)got, (long long)want);
                }
        }
    for (int f = 0; f < F; ++f) CHECK(times[f] == 1, "%s: F=%d: element %d is in %d lanes", what, F, f, times[f]);
    ++checked;
}
template <int E>
static void lanes_of(const Layout& l, int F, int64_t n, int64_t ld, bool offsets, const char* what) {
    const bool mask = F % E != 0;
    if (l.p == 1) mask ? lanes<E, true, 1>(l, F, n, ld, offsets, what) : lanes<E, false, 1>(l, F, n, ld, offsets, what);
    else if (l.p == 2) mask ? lanes<E, true, 2>(l, F, n, ld, offsets, what) : lanes<E, false, 2>(l, F, n, ld, offsets, what);
    else mask ? lanes<E, true, 3>(l, F, n, ld, offsets, what) : lanes<E, false, 3>(l, F, n, ld, offsets, what);
}

static void rows(const Layout& l, int F, int64_t n, const char* what) {
    const int64_t a_turn = l.w == 1 ? 4 * (64 / l.g) : 1;
    CHECK(l.turns >= 1 && l.blocks * l.turns * a_turn >= n && (l.blocks - 1) * l.turns * a_turn < n, "%s: F=%d, %lld rows: %lld workgroups of %d turns", what, F,
          (long long)n, (long long)l.blocks, l.turns);
    CHECK(l.blocks * (l.w == 1 ? 256 : l.w * 64) <= 0xFFFFFFFFLL, "%s: F=%d, %lld rows: %lld workgroups, more threads than a launch has", what, F, (long long)n,
          (long long)l.blocks);
    CHECK(l.most_blocks <= kMostSums, "%s: F=%d, %lld rows: sums of %lld workgroups", what, F, (long long)n, (long long)l.most_blocks);
    CHECK(l.blocks <= l.most_blocks || strcmp(what, "backward") != 0, "%s: F=%d, %lld rows: %lld workgroups, room for %lld", what, F, (long long)n,
          (long long)l.blocks, (long long)l.most_blocks);
}

int main(int argc, char** argv) {
    const bool offsets = argc > 1 && strcmp(argv[1], "offsets") == 0;
    std::vector<int> widths;
    for (int F = 1; F <= 70; ++F) widths.push_back(F);
    for (int F : {100, 127, 128, 129, 255, 256, 257, 500, 505, 511, 512, 513, 520, 600, 767, 768, 769, 1000, 1024, 1025, 1433, 1536, 1537, 2000, 2048, 2049, 3071, 3073, 4095, 4096,
                  4097, 6145, 8191, 8192, 8193, 16390})
        widths.push_back(F);
    std::vector<int64_t> strides;                 // beyond the row's width: near powers of two, and at tenths of an octave in between
    for (int b = 0; b < 40; ++b)
        for (int k = 0; k < 10; ++k) strides.push_back((int64_t)(((uint64_t)1 << b) * (1.0 + 0.1 * k)));
    for (int b = 10; b < 40; ++b)
        for (int d : {-9, -1, 1, 8}) strides.push_back(((int64_t)1 << b) + d);
    for (int64_t x : {17'043'521, 17'043'522, 34'087'042, 34'087'043, 34'636'832, 34'636'833}) strides.push_back(x);
    for (int bf = 0; bf < 2; ++bf)
        for (int bwd = 0; bwd < 2; ++bwd) {
            const char* what = bwd ? "backward" : "forward";
            for (int F : widths)
                for (int64_t n : {(int64_t)1, (int64_t)2, (int64_t)63, (int64_t)700, (int64_t)100'000, (int64_t)3'125'002}) {
                    for (int64_t more : strides) {
                        const Layout l = layout_of(n, F, bf, bwd, F + more);
                        if (l.w) rows(l, F, n, what);
                        if (l.w && n <= 63) bf ? lanes_of<8>(l, F, n, F + more, offsets, what) : lanes_of<4>(l, F, n, F + more, offsets, what);
                    }
                }
        }
    if (argc > 1 && strcmp(argv[1], "rows") == 0)
        for (int bf = 0; bf < 2; ++bf)
            for (int bwd = 0; bwd < 2; ++bwd)
                for (int F : widths)
                    for (int b = 0; b < 38; ++b)                  // up to 2^38 rows
                        for (int k = 0; k < 8; ++k) {
                            const int64_t n = ((int64_t)1 << b) + (k < 4 ? k : ((int64_t)1 << b) * (k - 3) / 5);
                            for (int64_t ld : {(int64_t)F, (int64_t)1 << 30}) {
                                if (n > ((int64_t)1 << 58) / ld) continue;                 // no such matrix
                                const Layout l = layout_of(n, F, bf, bwd, ld);
                                if (l.w) rows(l, F, n, bwd ? "backward" : "forward");
                            }
                        }
    printf("%d layouts, %d failures\n", checked, failures);
    return failures != 0;
}
