/* Host-side paths of the paged cache's calls that run without a GPU, for a build whose host code is instrumented with AddressSanitizer and
 * UndefinedBehaviorSanitizer (tests/test_host_cache.py): argument checks, and the plans of a call and its workspace, which are made before
 * a missing handle is refused.  Sizes go from nothing to the largest that their types hold. */
#include <stdio.h>
#include <string.h>

#include "../../include/dessert.h"

#define COUNT(a) (sizeof(a) / sizeof *(a))

int main(void) {
    /* addresses that no refused call touches */
    int8_t *const codes = (int8_t *)4096;
    float *const f = (float *)8192;
    uint32_t *const u = (uint32_t *)12288, *const w = (uint32_t *)(1ull << 40);
    void *const ws = (void *)16384;
    const uint32_t sizes[] = {0, 1, 5, 16, 64, 100, 300, 4096, 70000, 1u << 24, (1u << 24) + 1, 0x7FFFFF00u, 0x7FFFFF01u, ~0u};
    const uint32_t pages[] = {16, 64, 256, 24}, dims[] = {32, 128, 256, 40}, heads[] = {1, 8, 65535, 0};
    const size_t given[] = {0, 256, ~(size_t)0};
    unsigned long refused = 0, calls = 0;

    for (size_t a = 0; a < COUNT(sizes); ++a)
        for (size_t b = 0; b < COUNT(sizes); ++b)
            for (size_t c = 0; c < COUNT(sizes); ++c)
                for (size_t p = 0; p < COUNT(pages); ++p)
                    for (size_t g = 0; g < COUNT(given); ++g) {
                        const dessert_cache_t cache = {codes, codes, f, f, codes, sizes[b] ? sizes[b] : 1, heads[(a + b) % 4], pages[p], dims[(a + c) % 4]};
                        const dessert_cache_batch_t batch = {u, u, u, sizes[a], sizes[b], sizes[c], sizes[c] < 3000 ? sizes[c] : sizes[a], sizes[b]};
                        const uint32_t q_heads = cache.n_heads * (g ? 4 : 1);
                        const uint64_t stride = (uint64_t)q_heads * cache.dim;
                        void *const work = given[g] ? ws : NULL;
                        refused += dessert_cache_append(NULL, &cache, &batch, f, stride, f, stride, DESSERT_F32) == DESSERT_EINVAL;
                        refused += dessert_cache_attention(NULL, &cache, &batch, f, DESSERT_BF16, stride, q_heads, 1.f, sizes[a], g ? u : NULL, g ? sizes[b] : 0,
                                                           work, given[g], f, f) == DESSERT_EINVAL;
                        refused += dessert_cache_attention(NULL, &cache, &batch, f, DESSERT_F16, stride, q_heads, 1.f, sizes[a], NULL, 0, work, given[g], f, f) ==
                                   DESSERT_EINVAL;
                        refused += dessert_cache_select(NULL, &cache, &batch, codes, f, q_heads, sizes[a], 1, 2, work, given[g], u) == DESSERT_EINVAL;
                        refused += dessert_cache_advance(NULL, &cache, 1, u, u, sizes[b], u, sizes[a], g ? u : NULL, u, g ? sizes[c] : sizes[a], work, given[g], w, w,
                                                         u) == DESSERT_EINVAL;
                        refused += dessert_cache_compact(NULL, &cache, 1, u, u, sizes[b], u, sizes[a], work, given[g], u, u) == DESSERT_EINVAL;
                        refused += dessert_cache_attention_workspace_bytes(NULL, &cache, &batch, q_heads, 0) == 0;
                        refused += dessert_cache_select_workspace_bytes(NULL, &cache, &batch) == 0;
                        refused += dessert_cache_advance_workspace_bytes(NULL, sizes[a], sizes[b]) == 0;
                        refused += dessert_cache_compact_workspace_bytes(NULL, sizes[a]) == 0;
                        calls += 10;
                    }
    refused += dessert_cache_append(NULL, NULL, NULL, NULL, 0, NULL, 0, DESSERT_F16) == DESSERT_EINVAL;
    refused += dessert_cache_advance(NULL, NULL, 0, NULL, NULL, 0, NULL, 0, NULL, NULL, 0, NULL, 0, NULL, NULL, NULL) == DESSERT_EINVAL;
    calls += 2;
    if (refused != calls) {
        printf("FAILED: %lu of %lu refused\n", refused, calls);
        return 1;
    }
    printf("paged cache host sanitizer run: ok\n");
    return 0;
}
