// The plans of the paged cache's operators over sizes up to the largest: workspaces hold what the plans lay into them, and what a call gives for a size
// serves every smaller one.
#include <cstdio>

#include "cache_plans.hpp"

using namespace dessert;

static int failures = 0;
#define EXPECT(cond)                                             \
    do {                                                         \
        if (!(cond)) {                                           \
            if (failures < 20) std::printf("FAILED line %d: %s\n", __LINE__, #cond); \
            ++failures;                                          \
        }                                                        \
    } while (0)

int main() {
    const uint64_t seqs[] = {1, 2, 7, 16, 31, 64, 255, 256, 257, 511, 4000, 100000}, tokens[] = {1, 2, 5, 16, 33, 64, 65, 127, 600, 2048, 100000};
    const uint32_t heads[] = {1, 2, 8, 12, 40}, groups[] = {1, 3, 4, 16, 64, 65};
    const uint64_t lengths[] = {0, 1, 64, 256, 257, 500, 1024, 1025, 5000, 131072, CACHE_MOST};
    for (uint32_t dim = 32; dim <= 256; dim += 32)
        for (uint64_t s : seqs)
            for (uint64_t t : tokens)
                for (uint32_t h : heads)
                    for (uint32_t g : groups)
                        for (uint64_t l : lengths)
                            for (int lists = 0; lists < 2; ++lists) {
                                if ((lists ? s * t : s) * h > 0xFFFFFFFFull / 256) continue;      // refused
                                const AttendPlan p = attend_plan(s, t, h, g, dim, l, lists);
                                const uint64_t chunks = l ? divided_up(l, ATTEND_CHUNK) : 1, rows = lists ? g : t * g;
                                EXPECT(p.parts >= 1 && p.parts <= ATTEND_MOST_GROUPS && (uint64_t)p.parts * p.part_chunks >= chunks);
                                EXPECT((uint64_t)(p.parts - 1) * p.part_chunks < chunks);
                                EXPECT((uint64_t)p.tiles * p.rows >= rows);
                                EXPECT(p.groups == (lists ? s * t : s) * h * p.tiles);
                                EXPECT(p.parts == 1 || (p.bytes % 256 == 0 && p.sums == p.groups * p.parts * p.rows * dim * 4 &&
                                                        p.sums + p.groups * p.parts * p.rows * 8 <= p.bytes));
                                EXPECT(p.parts > 1 || p.bytes == 0);
                                // what larger calls are told
                                EXPECT(p.bytes <= attend_workspace_upto(t, g, dim, l, lists));
                                EXPECT(p.bytes <= attend_workspace_upto(t * 2, g, dim, l + 1000, lists));
                                EXPECT(p.bytes <= attend_workspace_upto(t + 1, g, dim, l * 2, lists));
                            }
    for (uint64_t pages = 1; pages <= CACHE_MOST; pages = pages * 3 + 1)
        for (uint64_t n = 0; n <= CACHE_MOST; n = n * 5 + 1) {
            const AdvancePlan p = advance_plan(pages, n);
            EXPECT(p.writers == 0 && p.lowest >= p.writers + 4 * pages && p.stays >= p.lowest + 4 * pages);
            EXPECT(p.free_pages >= p.stays + 4 * pages && p.copies >= p.free_pages + 4 * pages && p.bytes >= p.copies + 8 * n);
            EXPECT(p.bytes <= advance_plan(pages + 7, n + 3).bytes);
            const CompactPlan c = compact_plan(pages);
            EXPECT(c.moved >= 64 && c.holes >= c.moved + 4 * pages && c.bytes >= c.holes + 4 * pages && c.bytes <= compact_plan(pages + 1).bytes);
        }
    for (uint64_t t = 1; t <= CACHE_MOST; t = t * 7 + 1)
        for (uint64_t h = 1; h <= 65535; h = h * 3 + 1)
            for (uint64_t w = 1; w <= CACHE_MOST / 16; w = w * 5 + 1) {
                const size_t n = select_workspace(t, h, w);
                EXPECT(n == ~(size_t)0 || (n % 256 == 0 && n / 4 / w / h >= t));
                EXPECT(n <= select_workspace(t + 1, h, w) && n <= select_workspace(t, h, w + 1));
            }
    for (uint32_t page = 16; page <= 256; page *= 2)
        for (uint64_t t = 1; t < 3000; ++t)
            for (uint64_t first = 0; first < page; first += 5) EXPECT((first + t - 1) / page + 1 <= append_places(t, page));
    if (failures) return 1;
    std::printf("cache plans sanitizer run: ok\n");
    return 0;
}
