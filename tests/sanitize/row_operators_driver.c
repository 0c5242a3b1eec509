/* Host-side paths of the row operators that run without a GPU, for a build whose host code is instrumented with
 * AddressSanitizer and UndefinedBehaviorSanitizer (tests/test_host_row_sanitized.py): argument checks, and the plans of a call and its
 * workspace, which are made before a missing handle is refused.  Sizes go from nothing to the largest that the header allows. */
#include <stdio.h>
#include <string.h>

#include "../../include/dessert.h"

static int failures = 0;
#define EXPECT(cond)                                                        \
    do {                                                                    \
        if (!(cond)) {                                                      \
            printf("FAILED line %d: %s  (last error: %s)\n", __LINE__, #cond, dessert_last_error()); \
            ++failures;                                                     \
        }                                                                   \
    } while (0)
#define COUNT(a) (sizeof(a) / sizeof *(a))

int main(void) {
    /* addresses that no refused call touches */
    int8_t *const codes = (int8_t *)4096;
    float *const f = (float *)8192;
    uint32_t *const u = (uint32_t *)12288;
    void *const ws = (void *)16384;
    const uint64_t rows[] = {0, 1, 16, 17, 64, 300, 1023, 1024, 4096, 1u << 20, (1ull << 31) - 1, 1ull << 31, 1ull << 40, ~0ull};
    const uint32_t cols[] = {0, 1, 16, 77, 2049, 4096, 8193, 65536, 131071, 131072, 1u << 20, 1u << 30, (1u << 30) + 1, ~0u};
    const uint32_t tops[] = {0, 1, 64, 65, ~0u};
    const size_t given[] = {0, 256, (size_t)1 << 50};
    unsigned long refused = 0, calls = 0;

    for (size_t i = 0; i < COUNT(rows); ++i)
        for (size_t j = 0; j < COUNT(cols); ++j) {
            const uint64_t stride = cols[j] < (1u << 31) ? cols[j] : (1u << 31) - 1;
            for (int scaling = -1; scaling <= 2; ++scaling)
                for (uint32_t dtype = 0; dtype <= 4; ++dtype) {
                    refused += dessert_quantize_rows(NULL, f, dtype, rows[i], cols[j], stride, scaling, codes, f) == DESSERT_EINVAL;
                    ++calls;
                }
            for (size_t w = 0; w < COUNT(given); ++w) {
                for (size_t n = 0; n < COUNT(rows); ++n) {
                    refused += dessert_scaled_matmul(NULL, codes, stride, f, rows[i], codes, stride, f, w ? f : NULL, rows[n], cols[j], DESSERT_F16, f,
                                                     rows[n], given[w] ? ws : NULL, given[w]) == DESSERT_EINVAL;
                    ++calls;
                }
                for (size_t t = 0; t < COUNT(tops); ++t) {
                    refused += dessert_token_logprobs(NULL, f, DESSERT_BF16, rows[i], cols[j], stride, u, tops[t], given[w] ? ws : NULL, given[w], f, f, u, f) ==
                               DESSERT_EINVAL;
                    ++calls;
                    for (size_t k = 0; k < COUNT(cols); ++k) {
                        const uint64_t apart = cols[k] < (1u << 31) ? cols[k] : (1u << 31) - 1;
                        for (unsigned odd = 0; odd < 2; ++odd) {   /* rows at whole 16 bytes, or anywhere: the two ways of the head form */
                            refused += dessert_head_logprobs(NULL, codes + odd, apart, f, rows[i], codes, apart, f, cols[j], cols[k], u, tops[t],
                                                             given[w] ? ws : NULL, given[w], f, f, u, f) == DESSERT_EINVAL;
                            ++calls;
                        }
                    }
                }
            }
        }
    EXPECT(refused == calls);

    /* calls that are right but for the handle come as far as that, with the workspace that they need and not with less */
    EXPECT(dessert_scaled_matmul(NULL, codes, 8192, f, 64, codes, 8192, f, NULL, 4096, 8192, DESSERT_BF16, f, 4096, ws, 8u << 20) == DESSERT_EINVAL &&
           strstr(dessert_last_error(), "index is NULL"));
    EXPECT(dessert_scaled_matmul(NULL, codes, 8192, f, 64, codes, 8192, f, NULL, 4096, 8192, DESSERT_BF16, f, 4096, ws, (8u << 20) - 1) == DESSERT_EINVAL &&
           strstr(dessert_last_error(), "workspace too small: 8388607 bytes given, 8388608 needed"));
    EXPECT(dessert_head_logprobs(NULL, codes, 2048, f, 4096, codes, 2048, f, 32000, 2048, u, 5, ws, (size_t)1 << 30, f, f, u, f) == DESSERT_EINVAL &&
           strstr(dessert_last_error(), "index is NULL"));
    EXPECT(dessert_head_logprobs(NULL, codes, 2048, f, 4096, codes, 2048, f, 32000, 2048, u, 5, ws, 1u << 20, f, f, u, f) == DESSERT_EINVAL &&
           strstr(dessert_last_error(), "workspace too small"));
    EXPECT(dessert_scaled_matmul_workspace_bytes(NULL, 64, 4096, 8192) == 0);
    EXPECT(dessert_token_logprobs_workspace_bytes(NULL, 8, 50257, 5) == 0);
    EXPECT(dessert_head_logprobs_workspace_bytes(NULL, 8, 50257, 64, 5) == 0);
    EXPECT(strlen(dessert_last_error()) < 512);

    if (failures) return 1;
    printf("row operators host sanitizer run: ok, %lu calls\n", calls);
    return 0;
}
