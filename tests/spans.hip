// Host check of meet(): rows of two arrays share bytes exactly where the bytes written down one by one do.
#include <cstdio>
#include <random>
#include <vector>
#include "../paper_2012_09849_amd/csrc/spans.hpp"

using namespace hts;

int main()
{
    std::mt19937 r(1);
    auto pick = [&](int lo, int hi) { return (int64_t)std::uniform_int_distribution<int>(lo, hi)(r); };
    int met = 0, apart = 0;
    for (int k = 0; k < 400000; ++k) {
        Span a{pick(1, 120), pick(0, 24), pick(1, 6), pick(1, 16)}, b{pick(1, 120), pick(0, 24), pick(1, 6), pick(1, 16)};
        if (k % 3 == 0) b.ld = a.ld;
        std::vector<char> bytes(600, 0);
        for (int64_t i = 0; i < a.rows; ++i) for (int64_t j = 0; j < a.bytes; ++j) bytes[a.p + i * a.ld + j] = 1;
        bool want = false;
        for (int64_t i = 0; i < b.rows; ++i) for (int64_t j = 0; j < b.bytes; ++j) want |= bytes[b.p + i * b.ld + j] != 0;
        if (meet(a, b) != want || meet(b, a) != want) {
            printf("a %lld + i %lld, %lld rows of %lld; b %lld + i %lld, %lld rows of %lld: %d\n", (long long)a.p, (long long)a.ld, (long long)a.rows, (long long)a.bytes, (long long)b.p, (long long)b.ld, (long long)b.rows,
                   (long long)b.bytes, (int)want);
            return 1;
        }
        ++(want ? met : apart);
    }
    // far apart in memory, large, interleaved
    const Span wide{1ll << 40, 4096, 1 << 24, 2048}, between{(1ll << 40) + 2048, 4096, 1 << 24, 2048}, into{(1ll << 40) + 2047, 4096, 1 << 24, 2048}, none{0, 0, 0, 8};
    if (meet(wide, between) || !meet(wide, into) || meet(wide, none) || meet(none, wide) || !same(wide, wide)) return 2;
    printf("%s\n", met > 50000 && apart > 50000 ? "ok" : "too few of a kind");
    return 0;
}
