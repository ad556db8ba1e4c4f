// Built for the host with AddressSanitizer and UndefinedBehaviorSanitizer: how many tokens of a sequence are in a chunk, and what the entry points of linear attention and
// layer norm refuse and hand to the launchers, which are written down here instead of launching anything.
#include <limits.h>
#include <stdio.h>
#include <stdlib.h>

#include "../../paper_2402_02320_amd/csrc/linear.hpp"

using namespace spin;

#define CHECK(x)                                                      \
    do {                                                              \
        if (!(x)) { printf("line %d: %s\n", __LINE__, #x); exit(1); } \
    } while (0)

static int launched;
static u64 inverse_seen;
namespace spin {
#define NOTED(T)                                                                                                                  \
    template <> spin_status launch_linattn_scores<T>(const ScoresArgs<T> &, hipStream_t) { return ++launched, SPIN_OK; }          \
    template <> spin_status launch_linattn_states<T>(const StatesArgs<T> &, hipStream_t) { return ++launched, SPIN_OK; }          \
    template <> spin_status launch_linattn_outputs<T>(const OutputsArgs<T> &, hipStream_t) { return ++launched, SPIN_OK; }        \
    template <> spin_status launch_linattn_step<T>(const StepArgs<T> &, hipStream_t) { return ++launched, SPIN_OK; }              \
    template <> spin_status launch_layernorm<T>(const NormArgs<T> &a, hipStream_t) { return inverse_seen = a.inv, ++launched, SPIN_OK; } \
    template <> spin_status launch_layernorm_grad<T>(const NormGradArgs<T> &a, hipStream_t) { return inverse_seen = a.inv, ++launched, SPIN_OK; }
NOTED(u64)
NOTED(u32)
size_t layernorm_grad_workspace(int, int, int, int) { return 256; }
}  // namespace spin

int main()
{
    const int odd[] = {INT_MIN, INT_MIN + 1, -7, -1, 0, 1, 31, 32, 33, 299, 300, 301, INT_MAX};
    for (int chunk = 32; chunk <= 128; chunk *= 2)
        for (int tokens : {1, 32, 300, 1 << 24})
            for (int length : odd) {
                const ChunkView c{1, 1, 1, tokens, chunk, (tokens + chunk - 1) / chunk, 1, 0, nullptr};
                long sum = 0;
                for (int k = 0; k < c.chunks; ++k) {
                    const int L = tokens_in(c, length, k);
                    CHECK(L >= 0 && L <= chunk && (long)k * chunk + L <= tokens);
                    sum += L;
                }
                CHECK(sum == (length < 0 ? 0 : length < tokens ? length : tokens));
            }
    // every number of the descriptors at its extremes: an answer, and no arithmetic that overflows
    u64 *const p = (u64 *)0x10000;
    const spin_masked m{p, p};
    const spin_tuple t{p, p, p};
    for (int field = 0; field < 7; ++field)
        for (int v : odd) {
            spin_linattn s{2, 2, 3, 100, 64, 9, 6, p, nullptr};
            int *const at[] = {&s.n, &s.batch, &s.heads, &s.tokens, &s.chunk, &s.f, &s.g};
            *at[field] = v;
            for (int d : {8, 40, 256, -8, 0, INT_MAX, INT_MIN}) {
                const int before = launched;
                const spin_status st[] = {spin_linattn_scores(&s, d, &m, &m, p, &t, p, nullptr),
                                          spin_linattn_states(&s, d, 40, 0, &m, &m, p, &t, nullptr, p, p, p, (size_t)1 << 50, nullptr),
                                          spin_linattn_outputs(&s, 40, d, 1, 1, &m, &m, &m, &m, p, &t, p, nullptr),
                                          spin_linattn_step(&s, d, 40, p, &m, &m, &m, p, p, &t, p, &t, p, p, nullptr)};
                int ok = 0;
                for (spin_status one : st) ok += one == SPIN_OK;
                CHECK(launched - before == ok);
                CHECK((spin_linattn_states_workspace_bytes(&s, d, 40) != 0) == (st[1] == SPIN_OK));
            }
        }
    u32 *const q = (u32 *)0x10000;
    for (int field = 0; field < 5; ++field)
        for (int v : odd) {
            spin_norm s{2, 7, 33, 9, 15};
            int *const at[] = {&s.n, &s.rows, &s.dim, &s.f, &s.shift};
            *at[field] = v;
            const int before = launched;
            const spin_status st = spin32_layernorm(&s, 2, 1, 1, 1, q, &m, q, q, q, q, &t, q, &t, q, q, nullptr, nullptr, nullptr);
            CHECK(st == spin32_layernorm_grad(&s, &m, &m, q, &m, q, q, &t, q, &t, q, q, q, q, q, q, 256, nullptr));
            CHECK(launched - before == (st == SPIN_OK ? 2 : 0));
            CHECK((spin32_layernorm_grad_workspace_bytes(&s) != 0) == (st == SPIN_OK));
            if (st == SPIN_OK) CHECK(inverse_seen == (((u64)1 << s.shift) + s.dim / 2) / s.dim);
        }
    spin_norm wide{8, 1, 1, 60, 61};
    CHECK(spin_layernorm(&wide, 16, 1, 1, 1, p, &m, p, p, p, p, &t, p, &t, p, p, p, p, nullptr) == SPIN_OK && inverse_seen == (u64)1 << 61);
    printf("run ok\n");
    return 0;
}
