// Host-side check of the ranges that a context is split into
// (attend_split.hpp): for lengths from nothing to the largest, and any number of
// ranges asked for, they follow one another from the first token to the last
// without gaps, begin at multiples of 64, and are no more than asked for.
// Prints "<splits> splits, <failures> failures" and exits 1 on any failure.
#include <cstdio>

#include "attend_split.hpp"

using namespace tf;

static int fails = 0;

static void check(long long ctx, int most) {
    const Split s = split_context((int)ctx, most);
    long long at = 0;
    bool ok = s.chunk >= 64 && s.chunk % 64 == 0 && s.count >= 1 && s.count <= (most > 1 ? most : 1);
    for (int r = 0; ok && r < s.count; ++r) {
        const long long lo = s.begin(r), hi = s.end(r, (int)ctx);
        ok = lo == at && hi <= ctx && (hi > lo || ctx == 0) && (r + 1 == s.count ? hi == ctx : hi == lo + s.chunk);
        at = hi;
    }
    if (s.count > 1 && 2 * s.chunk <= kSplitLeast) ok = false;
    if (!ok && fails++ < 20) std::printf("FAIL context %lld in at most %d: chunk %d, count %d\n", ctx, most, s.chunk, s.count);
}

int main() {
    const long long largest = 0x7fffff00ll;
    long long n = 0;
    for (int most = 1; most <= kMostSplits; ++most) {
        for (long long ctx = 0; ctx < 3000; ++ctx, ++n) check(ctx, most);
        for (long long back = 0; back < (1ll << 27); back = back < 600 ? back + 1 : back * 2 + 1, ++n) check(largest - back, most);
        for (long long ctx = 1; ctx < largest; ctx = ctx * 3 / 2 + 7, ++n) check(ctx, most);
    }
    std::printf("%lld splits, %d failures\n", n, fails);
    return fails != 0;
}
