// Built for the host with AddressSanitizer and UndefinedBehaviorSanitizer: the rows of a diagonal that the bias's gradient adds up, against the
// definition, for lengths of any kind, and every word that they stand for read from a buffer of exactly the matrix's size.
#include <limits.h>
#include <stdio.h>
#include <stdlib.h>

#include "../../paper_2402_02320_amd/csrc/generation.hpp"

using namespace spin;

static volatile u32 sink;

int main()
{
    const int sizes[][2] = {{1, 1}, {4, 4}, {3, 9}, {11, 2}};
    for (const auto &size : sizes) {
        const int Q = size[0], K = size[1];
        u32 *x = (u32 *)calloc((size_t)Q * K, sizeof(u32));
        const int lengths[] = {INT_MIN, INT_MIN + 1, INT_MIN + K, -K - 1, -1, 0, 1, K - 1, K, K + 1, INT_MAX - K, INT_MAX};
        for (int length : lengths)
            for (int causal = 0; causal < 2; ++causal)
                for (int first : {-K - Q, -1, 0, 2, K + Q})
                    for (int q0 = 0; q0 < Q; q0 += 2)
                        // a workgroup's last diagonals are past the matrix by up to its number of threads
                        for (int away = -(Q - 1); away < K + 128; ++away) {
                            const int q1 = q0 + 2 < Q ? q0 + 2 : Q;
                            const DiagonalRows r = rows_of_diagonal(away, q0, q1, K, length, causal != 0, first);
                            for (int q = r.from; q < r.to && q < Q + 64; ++q) sink += x[(long)q * K + q + away];
                            for (int q = q0; q < q1; ++q) {
                                const long k = (long)q + away;
                                const bool there = k >= 0 && k < K && k < length && (!causal || k <= (long)q + first);
                                if (there != (q >= r.from && q < r.to)) {
                                    printf("Q %d K %d length %d causal %d first %d away %d q %d\n", Q, K, length, causal, first, away, q);
                                    return 1;
                                }
                            }
                        }
        free(x);
    }
    printf("diagonal run ok\n");
    return 0;
}
