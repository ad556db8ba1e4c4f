// Built for the host with AddressSanitizer and UndefinedBehaviorSanitizer: what the attention's entry points hand to the launchers, which are written
// down here instead of launching anything.
#include <stdio.h>
#include <stdlib.h>

#include "../../paper_2402_02320_amd/csrc/generation.hpp"

using namespace spin;

static const int32_t *depth_seen;
static int launched;

namespace spin {
template <class T> static spin_status note(const AttentionArgs<T> &a)
{
    depth_seen = a.depth;
    ++launched;
    return SPIN_OK;
}
template <> spin_status launch_cache_scores<u64>(const AttentionArgs<u64> &a, hipStream_t) { return note(a); }
template <> spin_status launch_cache_scores<u32>(const AttentionArgs<u32> &a, hipStream_t) { return note(a); }
template <> spin_status launch_cache_values<u64>(const AttentionArgs<u64> &a, hipStream_t) { return note(a); }
template <> spin_status launch_cache_values<u32>(const AttentionArgs<u32> &a, hipStream_t) { return note(a); }
size_t cache_values_workspace(int, int, int, int, int, int, int, int) { return 256; }
#define NOT_CALLED(T)                                                                                                                        \
    template <> spin_status launch_cache_append<T>(const AppendArgs<T> &, hipStream_t) { abort(); }                                          \
    template <> spin_status launch_cache_copy<T>(const CacheView &, int, int, const int32_t *, const int32_t *, T *, T *, hipStream_t) { abort(); } \
    template <>                                                                                                                              \
    spin_status launch_cache_compact<T>(const CacheView &, int, int, int, const int32_t *, const int32_t *, const int32_t *, T *, T *, hipStream_t) \
    {                                                                                                                                        \
        abort();                                                                                                                             \
    }                                                                                                                                        \
    template <> spin_status launch_relbias_trunc<T>(const PairArgs<T> &, hipStream_t) { abort(); }                                           \
    template <> spin_status launch_relbias_grad<T>(const PairArgs<T> &, hipStream_t) { abort(); }
NOT_CALLED(u64)
NOT_CALLED(u32)
}  // namespace spin

#define CHECK(x)                                                      \
    do {                                                              \
        if (!(x)) { printf("line %d: %s\n", __LINE__, #x); exit(1); } \
    } while (0)

int main()
{
    uint64_t word[2] __attribute__((aligned(16))) = {0, 0};
    int32_t index[2] = {0, 0};
    const int32_t *const odd = (const int32_t *)((const char *)index + 1);
    spin_cache c = {2, 4, 2, 16, 64, word, word, 1, 1, index};
    const spin_relbias bias = {32, 0, index, word};
    uint32_t *const w32 = (uint32_t *)word;
    // Distances are of the bias alone: without one, `depth` is nothing that a kernel may follow.
    for (const int32_t *depth : {(const int32_t *)nullptr, (const int32_t *)index, odd}) {
        depth_seen = index + 1;
        CHECK(spin_cache_scores(&c, 2, 1, 1, 0, index, nullptr, word, word, word, nullptr, nullptr, nullptr, 0, nullptr, depth, word, nullptr) == SPIN_OK);
        CHECK(depth_seen == nullptr);
        depth_seen = index + 1;
        CHECK(spin32_cache_scores(&c, 2, 1, 1, 0, index, nullptr, w32, w32, w32, nullptr, nullptr, nullptr, 0, nullptr, depth, w32, nullptr) == SPIN_OK);
        CHECK(depth_seen == nullptr);
    }
    CHECK(spin_cache_scores(&c, 2, 1, 1, 0, index, nullptr, word, word, word, nullptr, nullptr, nullptr, 0, &bias, index, word, nullptr) == SPIN_OK);
    CHECK(depth_seen == index);
    const int before = launched;
    CHECK(spin_cache_scores(&c, 2, 1, 1, 0, index, nullptr, word, word, word, nullptr, nullptr, nullptr, 0, &bias, odd, word, nullptr) == SPIN_EINVAL);
    CHECK(launched == before);
    printf("dispatch run ok\n");
    return 0;
}
