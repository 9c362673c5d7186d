// Host check of the matrix product's backward call: everything that the slices of dw's and db's reduction write and read lies within the call's workspace, and
// the rows' sums (db) lie behind those of C.
#include <hip/hip_runtime.h>
#include <cstdio>
#include "../paper_2012_09849_amd/csrc/linear_plan.hpp"

using namespace hts;

int main()
{
    long long calls = 0, sliced = 0;
    const int64_t rows[] = {1, 80, 512, 513, 1024, 1025, 3000, 8192, 20000}, outputs[] = {1, 7, 8, 64, 100, 128, 512, 2048};
    for (int size : {2, 4})
        for (int act : {HTS_ACT_NONE, HTS_ACT_SILU})
            for (int64_t M : rows)
                for (int64_t N : outputs)
                    for (int64_t K : {1, 2, 3, 4, 5, 6, 7, 8, 9, 33, 128, 517})
                        for (int dw = 0; dw < 2; ++dw) {
                            const LinearLayout at = linear_layout(size, act, M, N, K);
                            const Slices s = weight_slices(size, act, M, N, K, dw);
                            ++calls;
                            if (s.count == 1) continue;
                            ++sliced;
                            const int64_t last = at.part + 4 * s.count * s.stride;             // where the last slice ends
                            if (last > at.total || s.rows + N > s.stride || (dw && s.rows < N * K) || (int64_t)s.count * s.klen < M) {
                                printf("size %d act %d M %lld N %lld K %lld dw %d: %d slices end at byte %lld of %lld\n", size, act, (long long)M, (long long)N, (long long)K, dw, s.count,
                                       (long long)last, (long long)at.total);
                                return 1;
                            }
                        }
    printf("%lld calls, %lld sliced\n", calls, sliced);
    return 0;
}
