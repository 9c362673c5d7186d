// Host check of meet() of steps of sequences: two arrays share bytes exactly where the bytes written down one by one do.
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
    struct Given { int64_t p, st, sn, T, N, cols; };
    for (int k = 0; k < 400000; ++k) {
        const int size = k & 1 ? 2 : 4;
        auto any = [&]() { return k % 5 == 0 ? Given{pick(1, 200), 0, 0, 1, 1, pick(1, 60)} : Given{pick(1, 120), pick(0, 40), pick(0, 30), pick(1, 5), pick(1, 5), pick(1, 8)}; };
        Given a = any(), b = any();
        if (k % 3 == 0) { b.st = a.st; b.sn = a.sn; }
        std::vector<char> bytes(4096, 0);
        auto each = [&](const Given &g, auto f) {
            for (int64_t t = 0; t < g.T; ++t) for (int64_t n = 0; n < g.N; ++n) for (int64_t j = 0; j < g.cols * size; ++j) f(g.p + (t * g.st + n * g.sn) * size + j);
        };
        each(a, [&](int64_t i) { bytes[i] = 1; });
        bool want = false;
        each(b, [&](int64_t i) { want |= bytes[i] != 0; });
        const Area x = area((const void *)a.p, a.st, a.sn, a.T, a.N, a.cols, size), y = area((const void *)b.p, b.st, b.sn, b.T, b.N, b.cols, size);
        if (meet(x, y) != want || meet(y, x) != want) {
            for (const Given &g : {a, b}) printf("%lld: %lld steps, %lld apart, of %lld sequences, %lld apart, %lld entries\n", (long long)g.p, (long long)g.T, (long long)g.st, (long long)g.N, (long long)g.sn, (long long)g.cols);
            printf("entries of %d bytes: %d\n", size, (int)want);
            return 1;
        }
        ++(want ? met : apart);
    }
    // large, interleaved, at distances whose products leave 64 bits
    const void *base = (const void *)(1ll << 40), *beside = (const void *)((1ll << 40) + 2 * 512), *into = (const void *)((1ll << 40) + 2 * 511);
    const Area wide = area(base, 1 << 20, 1024, 1 << 30, 1 << 10, 512, 2), between = area(beside, 1 << 20, 1024, 1 << 30, 1 << 10, 512, 2), on = area(into, 1 << 20, 1024, 1 << 30, 1 << 10, 512, 2);
    const Area far = area(base, 1 << 20, 1ll << 40, 1 << 4, 1 << 24, 512, 4), near = area(beside, 1 << 20, 1ll << 40, 1 << 4, 1 << 24, 256, 2);
    if (meet(wide, between) || !meet(wide, on) || meet(wide, Area{}) || meet(area(nullptr, 8, 4), wide) || !meet(wide, wide) || !meet(far, near) || !meet(near, far)) return 2;
    printf("%s\n", met > 50000 && apart > 50000 ? "ok" : "too few of a kind");
    return 0;
}
