// The plans of the row operators (csrc/row_plans.hpp, csrc/launch_slices.hpp) under the sanitizers, without the handle that the workspace calls
// need: the parts of a plan lie one behind the other in its bytes and fit their launches, from one row to the largest number.
#include <cstdio>
#include <initializer_list>

#include "launch_slices.hpp"
#include "row_plans.hpp"

using namespace dessert;

static int failures = 0;
static void expect(bool ok, const char* what, uint64_t rows, uint64_t vocab, uint32_t k, uint32_t n_top) {
    if (!ok) {
        std::printf("FAILED %s: %llu rows, %llu entries, %u columns, %u alternatives\n", what, (unsigned long long)rows, (unsigned long long)vocab, k, n_top);
        ++failures;
    }
}

int main() {
    const uint64_t most = (1ull << 31) - 1;
    for (uint64_t rows : {(uint64_t)1, (uint64_t)16, (uint64_t)255, (uint64_t)300, (uint64_t)1023, (uint64_t)1024, (uint64_t)4097, (uint64_t)1 << 20, most})
        for (uint32_t vocab : {1u, 127u, 2049u, 20000u, 32000u, 131072u, 1u << 24, 1u << 30})
            for (uint32_t k : {1u, 16u, 776u, 4099u, 8192u, 131071u})
                for (uint32_t n_top : {0u, 1u, 5u, 64u}) {
                    const LogprobPlan p = logprob_plan(rows, vocab, n_top);
                    expect((uint64_t)p.splits * p.segment >= vocab && (uint64_t)(p.splits - 1) * p.segment < vocab, "segments", rows, vocab, k, n_top);
                    expect(p.splits == 1 || (rows < 1024 && p.bytes >= rows * p.splits * (12 + 8ull * n_top)), "parts of rows", rows, vocab, k, n_top);
                    const HeadPlan h = head_plan(rows, vocab, k, n_top);
                    expect(h.rows >= 1 && h.rows <= rows && h.stride >= vocab, "turn", rows, vocab, k, n_top);
                    expect(h.logits_bytes >= h.rows * h.stride * 4 && h.pass_bytes >= h.pass.bytes && h.bytes >= h.logits_bytes + h.pass_bytes, "turn's workspace",
                           rows, vocab, k, n_top);
                    expect(h.logits_bytes <= HEAD_TURN_BYTES || h.rows <= 256, "turn's size", rows, vocab, k, n_top);
                    const GroupPlan g = group_plan(rows, vocab, k, n_top);
                    if (g.rows) {
                        expect(g.rows <= rows && (uint64_t)g.groups * HEAD_GROUP >= vocab, "groups", rows, vocab, k, n_top);
                        const size_t at[] = {g.sums, g.counts, g.lists, g.picked, g.totals, g.logits, g.bytes};
                        const size_t need[] = {(size_t)g.rows * g.groups * 16, (size_t)g.groups * 4, n_top ? (size_t)g.rows * g.groups * 4 : 0,
                                               (size_t)g.rows * n_top * 4, (size_t)g.rows * 8, (size_t)g.rows * n_top * HEAD_GROUP * 4};
                        for (int i = 0; i < 6; ++i)
                            expect(at[i] % 256 == 0 && at[i] + need[i] <= at[i + 1], "groups' workspace", rows, vocab, k, n_top);
                        expect(g.rows * n_top < 1ull << 32, "32-bit places", rows, vocab, k, n_top);
                        expect((uint64_t)g.groups + g.rows * n_top / 32 < 1ull << 24, "a launch over the lists", rows, vocab, k, n_top);
                        expect(g.rows < 1ull << 24, "a launch over the rows", rows, vocab, k, n_top);
                    }
                    expect(head_workspace_upto(rows, vocab, k, n_top) >= std::max(h.bytes, g.bytes), "workspace", rows, vocab, k, n_top);
                    expect(h.rows < 1ull << 24, "a launch over the turn", rows, vocab, k, n_top);
                    expect(scaled_matmul_workspace_upto(rows, vocab, k) >= scaled_matmul_workspace(rows, vocab, k), "parts", rows, vocab, k, n_top);
                }
    uint64_t at = 0;
    in_launches(most, 1, 1024, [&](uint64_t first, uint64_t n, uint32_t workgroups) {
        expect(first == at && n == workgroups, "slices", first, n, workgroups, 0);
        at += n;
    });
    expect(at == most, "slices", at, 0, 0, 0);
    if (failures) return 1;
    std::printf("row plans sanitizer run: ok\n");
    return 0;
}
