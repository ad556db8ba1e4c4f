// Built for the host with AddressSanitizer and UndefinedBehaviorSanitizer: what the kernels of the paged cache go by (which page a position
// is on, where a row is, what a drafted token sees, the bucket of a distance), over tables and lists on exactly sized heap buffers that
// hold anything; and the entry points' argument checks with what they must refuse.
#include <limits.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include "../../paper_2402_02320_amd/csrc/generation.hpp"

using namespace spin;

#define CHECK(x)                                                      \
    do {                                                              \
        if (!(x)) { printf("line %d: %s\n", __LINE__, #x); exit(1); } \
    } while (0)

static int32_t *list(int n)
{
    return (int32_t *)malloc(n * sizeof(int32_t));
}

int main()
{
    const int32_t odd[] = {0, 1, -1, 4, 5, INT_MAX, INT_MIN, 2};
    for (int shift = 4; shift <= 12; shift += 4) {
        const int batch = 2, table_pages = 4, pages = 5, heads = 3, dim = 24, n = 2;
        int32_t *table = list(batch * table_pages);
        memcpy(table, odd, sizeof odd);
        const CacheView c{pages, heads, dim, table_pages, shift, table};
        const long size = (((long)(n + 1) * pages * heads) << shift) * dim, end = (long)table_pages << shift;
        const long at[] = {LONG_MIN, INT_MIN, -1, 0, 1, (1l << shift) - 1, 1l << shift, end - 1, end, end + 1, INT_MAX, LONG_MAX};
        for (long pos : at)
            for (int b = 0; b < batch; ++b) {
                const int page = page_of(c, b, pos);
                if (pos < 0 || pos >= end) { CHECK(page == -1); continue; }
                const int32_t want = odd[b * table_pages + (pos >> shift)];
                CHECK(page == (want >= 0 && want < pages ? want : -1));
                if (page < 0) continue;
                for (int slot = 0; slot <= n; ++slot)
                    for (int g = 0; g < heads; ++g) CHECK(row_at(c, slot, page, g, pos) + dim <= (size_t)size && row_at(c, slot, page, g, pos) % dim == 0);
            }
        CHECK(row_at(c, n, pages - 1, heads - 1, end - 1) + dim == (size_t)size);
        free(table);
    }
    {                                                     // offsets past 32 bits
        const CacheView c{1 << 20, 8, 128, 1 << 20, 6, nullptr};
        CHECK(row_at(c, 3, (1 << 20) - 1, 7, ((long)INT_MAX + 1) * 64 + 63) == ((((3ul << 20) + (1 << 20) - 1) * 8 + 7) * 64 + 63) * 128);
    }
    for (int nodes = 1; nodes <= 64; nodes += 21) {
        u64 *tree = (u64 *)malloc(nodes * sizeof(u64));
        for (int m = 0; m < nodes; ++m) tree[m] = 0xAAAAAAAAAAAAAAAAull >> (m % 2);
        const int32_t contexts[] = {0, 7, INT_MAX, INT_MIN, -1};
        const int positions[] = {0, 1, 6, 7, 8, 70, INT_MAX};
        for (int chain = 0; chain < 2; ++chain) {
            const DraftView d{nodes, 100, nullptr, chain ? nullptr : tree};
            for (int m = 0; m < nodes; ++m) {
                const u64 row = tree_row(d, 0, m);
                for (int32_t context : contexts)
                    for (int pos : positions) {
                        const long j = (long)pos - context;
                        const bool want = context >= 0 && (j < 0 || (j < nodes && (chain ? j <= m : (j + m) % 2 == 1)));
                        CHECK(sees(row, nodes, context, pos) == want);
                    }
            }
        }
        free(tree);
    }
    for (int reach = 0; reach <= 3; ++reach) {
        int32_t *of = list(2 * reach + 1);
        for (int k = 0; k <= 2 * reach; ++k) of[k] = odd[k];
        const BiasView v{5, reach, of, nullptr};
        const int distances[] = {INT_MIN, -4, -3, -1, 0, 1, 2, 3, 4, INT_MAX};
        for (int d : distances) {
            const int k = (d < -reach ? -reach : d > reach ? reach : d) + reach;
            CHECK(bucket_at(v, d) == (odd[k] >= 0 && odd[k] < 5 ? odd[k] : -1));
        }
        free(of);
    }
    // every refusal comes before a pointer is followed
    uint64_t word[2] __attribute__((aligned(16))) = {0, 0};
    int32_t index = 0;
    spin_cache c = {2, 4, 2, 16, 64, word, word, 1, 1, &index};
    const spin_relbias bias = {32, 16, &index, word};
    const int sizes[] = {INT_MIN, -1, 0, INT_MAX};
    for (int bad : sizes) {
        int *const fields[] = {&c.n, &c.pages, &c.heads, &c.page_tokens, &c.dim, &c.batch, &c.table_pages};
        for (int *f : fields) {
            if (f == &c.table_pages && bad == INT_MAX) continue;              // no more than a long table
            if ((f == &c.pages) && bad == INT_MAX) c.heads = 60000;           // within a pool's words otherwise
            const int keep = *f;
            *f = bad;
            CHECK(spin_cache_append(&c, 1, &index, nullptr, word, word, word, word, nullptr) != SPIN_OK);
            CHECK(spin_cache_compact(&c, 1, &index, &index, &index, nullptr) != SPIN_OK);
            CHECK(spin_cache_scores(&c, 2, 1, 1, 0, &index, nullptr, word, word, word, nullptr, nullptr, nullptr, 0, nullptr, nullptr, word, nullptr) != SPIN_OK);
            CHECK(spin_cache_values_workspace_bytes(&c, 2, 1, 1) == 0 && spin32_cache_values_workspace_bytes(&c, 2, 1, 1) == 0);
            *f = keep;
            c.heads = 2;
        }
        CHECK(spin_cache_append(&c, bad, &index, nullptr, word, word, word, word, nullptr) != SPIN_OK);
        CHECK(spin_cache_copy(&c, bad, &index, &index, nullptr) != SPIN_OK);
        CHECK(spin_cache_compact(&c, bad, &index, &index, &index, nullptr) != SPIN_OK);
        CHECK(spin_cache_values(&c, bad, 1, 1, 0, &index, nullptr, word, word, word, nullptr, nullptr, nullptr, word, word, 1, nullptr) != SPIN_OK);
        CHECK(spin_relbias_trunc(bad, 1, 1, 1, 1, 0, 0, nullptr, 0, word, nullptr, nullptr, nullptr, 0, &bias, word, nullptr) != SPIN_OK);
        CHECK(spin_relbias_trunc(1, bad, 1, 1, 1, 0, 0, nullptr, 0, word, nullptr, nullptr, nullptr, 0, &bias, word, nullptr) != SPIN_OK);
        CHECK(spin_relbias_grad(1, 1, bad, 1, 1, 0, 0, nullptr, word, &bias, word, nullptr) != SPIN_OK);
        CHECK(spin_relbias_grad(1, 1, 1, bad, 1, 0, 0, nullptr, word, &bias, word, nullptr) != SPIN_OK);
        CHECK(spin32_relbias_grad(1, 1, 1, 1, bad, 0, 0, nullptr, (uint32_t *)word, &bias, (uint32_t *)word, nullptr) != SPIN_OK);
        if (bad == INT_MIN || bad == INT_MAX) CHECK(spin_relbias_grad(1, 1, 1, 1, 1, bad, 0, nullptr, word, &bias, word, nullptr) != SPIN_OK);
    }
    printf("generation run ok\n");
    return 0;
}
