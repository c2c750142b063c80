/* The test of shared memory against every byte of small tensors, and on large ones whose answer is known. */
#include <cstdio>
#include <random>
#include <set>

#include "seq_overlap.h"

using xls::Span;
using xls::overlap;

static long long failures;
#define CHECK(c) do { if (!(c)) { ++failures; fprintf(stderr, "line %d: %s\n", __LINE__, #c); } } while (0)

static bool by_bytes(const Span &a, const Span &b)
{
    std::set<int64_t> bytes;
    for (int64_t i = 0; i < a.batch; ++i)
        for (int64_t j = 0; j < a.length; ++j)
            for (int64_t k = 0; k < a.width; ++k) bytes.insert(a.at + i * a.batch_step + j * a.token_step + k);
    for (int64_t i = 0; i < b.batch; ++i)
        for (int64_t j = 0; j < b.length; ++j)
            for (int64_t k = 0; k < b.width; ++k)
                if (bytes.count(b.at + i * b.batch_step + j * b.token_step + k)) return true;
    return false;
}

static bool twice(const Span &s)
{
    std::set<int64_t> bytes;
    for (int64_t i = 0; i < s.batch; ++i)
        for (int64_t j = 0; j < s.length; ++j)
            for (int64_t k = 0; k < s.width; ++k)
                if (!bytes.insert(s.at + i * s.batch_step + j * s.token_step + k).second) return true;
    return false;
}

int main()
{
    std::mt19937_64 rng(1);
    auto draw = [&](int n) { return (int64_t)(rng() % n); };
    long long met = 0;
    for (int i = 0; i < 400000; ++i) {
        Span s[2];
        for (Span &p : s) p = {1000 + draw(60), draw(5), draw(5), draw(24), draw(12), draw(6)};
        if (draw(3) == 0) s[1].batch_step = s[0].batch_step, s[1].token_step = s[0].token_step;
        const bool want = by_bytes(s[0], s[1]);
        met += want;
        CHECK(xls::overlaps_itself(s[0]) == twice(s[0]));
        if (overlap(s[0], s[1]) != want || overlap(s[1], s[0]) != want) {
            ++failures;
            for (const Span &p : s) fprintf(stderr, "%lld: %lld x %lld rows of %lld, steps %lld %lld\n", (long long)p.at, (long long)p.batch, (long long)p.length, (long long)p.width, (long long)p.batch_step, (long long)p.token_step);
            if (failures > 5) return 1;
        }
    }
    CHECK(met > 40000 && met < 360000);
    /* two halves of a wide tensor; the same half; a half one number further; another sequence; tokens outermost */
    const int64_t C = 4096, L = 12321, B = 64, base = 1ll << 40;
    const Span left = {base, B, L, 2 * C * L, 2 * C, C}, right = {base + C, B, L, 2 * C * L, 2 * C, C};
    CHECK(!overlap(left, right) && overlap(left, left) && left == left && !(left == right));
    CHECK(overlap(left, Span{base + 4, B, L, 2 * C * L, 2 * C, C}) && overlap(right, Span{base + C - 1, B, L, 2 * C * L, 2 * C, C}));
    CHECK(overlap(left, Span{base + 2 * C * L * 3, B, L, 2 * C * L, 2 * C, C}) && !overlap(left, Span{base + 2 * C * L * B, B, L, 2 * C * L, 2 * C, C}));
    CHECK(!overlaps_itself(left) && overlaps_itself(Span{base, B, L, 2 * C * (L - 1), 2 * C, C}) && !overlaps_itself(Span{base, B, L, C, 2 * C * B, C}) && overlaps_itself(Span{base, B, L, 0, C, C}));
    const Span outermost = {base, B, L, 2 * C, 2 * C * B, C};
    CHECK(!overlap(outermost, Span{base + C, B, L, 2 * C, 2 * C * B, C}) && overlap(outermost, Span{base + C - 1, B, L, 2 * C, 2 * C * B, C}));
    /* memory without gaps against rows with gaps */
    CHECK(overlap(left, Span{base + 2 * C * 7 + C - 1, 1, 1, 0, 0, 2}) && !overlap(left, Span{base + 2 * C * 7 + C, 1, 1, 0, 0, C}) && overlap(left, Span{base + 77 * C, 1, 100, 0, C, C}));
    printf("%lld of 400000 meet, %lld failures\n", met, failures);
    return failures != 0;
}
