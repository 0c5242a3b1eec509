// Sizes, limits and work divisions of the paged cache's operators (host code, no HIP).
#pragma once
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

#include "launch_slices.hpp"

namespace dessert {

constexpr uint32_t CACHE_MIN_PAGE = 16, CACHE_MAX_PAGE = 256, CACHE_MAX_DIM = 256;
constexpr uint32_t CACHE_MOST = 0x7FFFFF00u;   // tokens of a batch, positions, pages: sums with a step's tokens stay in 31 bits

// Pages that a sequence's new tokens touch, at most.
inline uint64_t append_places(uint64_t max_tokens, uint32_t page_tokens) { return (max_tokens + page_tokens - 2) / page_tokens + 1; }

// ---- attention ------------------------------------------------------------------------------------------------------------
// A step of the keys' axis.
constexpr uint32_t ATTEND_CHUNK = 64;
// Rows (query heads of one key head and the new tokens they belong to) of a workgroup, for few rows and for many.
constexpr uint32_t ATTEND_FEW = 16, ATTEND_MANY = 128;
// Up to so many rows of a unit the form for few takes, 16 at a time.  (16 sequences up to 8192, 8 heads of dim 128, us with the one for many / for few:
// 32 rows 98 / 78, 48 rows 111 / 101, 64 rows 113 / 110; 32 sequences up to 1000 of dim 64: 32 rows 28 / 15, 64 rows 36 / 20.)
constexpr uint32_t ATTEND_FEW_ROWS = 64;
// Workgroups that a call is split into along the keys where it has fewer: as many as the chip holds at once (its registers decide), so that
// none begins when others end.
// (One token, 8 heads of 4 query heads, 268 MB of codes, in us: 59 / 63 / 70 with 1024 / 768 / 512 workgroups at dim 32, 68 / 58 / 58 at 64,
// 66 / - / 59 at 128, - / 84 / 74 / 70 with 384 for the second and 256 for the fourth at 256.)
constexpr uint32_t ATTEND_MOST_GROUPS = 1024;
inline uint32_t attend_target(bool few, uint32_t dim) { return !few ? 512 : dim <= 32 ? 1024 : dim <= 64 ? 768 : dim <= 160 ? 512 : 256; }

struct AttendPlan {
    bool few;              // the form for few rows
    uint32_t waves;        // of a workgroup
    uint32_t rows;         // of a workgroup
    uint32_t tiles;        // workgroups along the rows of a unit
    uint32_t units;        // sequences, or with lists of pages the most tokens
    uint32_t parts;        // of the keys' axis at most
    uint32_t part_chunks;  // steps of a part
    uint64_t groups;       // units * heads * tiles
    size_t sums, bytes;    // workspace: partial outputs, from `sums` on partial maxima and sums
};

inline uint64_t divided_up(uint64_t a, uint64_t b) { return (a + b - 1) / b; }

inline size_t attend_bytes(uint64_t slots, uint32_t dim, size_t* sums) {
    const size_t out = slots * dim * sizeof(float);
    if (sums) *sums = out;
    return (out + slots * 2 * sizeof(float) + 255) / 256 * 256;
}

// length: about the most keys that the rows of a unit look at (with lists: n_select pages of them)
inline AttendPlan attend_plan(uint64_t seqs, uint64_t max_tokens, uint32_t heads, uint32_t group, uint32_t dim, uint64_t length, bool lists) {
    AttendPlan p{};
    const uint64_t rows = lists ? group : max_tokens * group;
    p.few = lists || rows <= ATTEND_FEW_ROWS;
    p.rows = p.few ? ATTEND_FEW : ATTEND_MANY;
    // (3584 tokens of 32 heads over up to 8192, in us with 128 / 256 rows to a workgroup: 293 / 351 at dim 32, 332 / 382 at 64, 435 / 421 at 96,
    // 484 / 474 at 128, 813 / 564 at 160, 1004 / 684 at 192, 1204 / 2405 at 256: there the registers of half as many waves are too few)
    if (!p.few && dim >= 128 && dim <= 192 && seqs * heads * divided_up(rows, 2 * ATTEND_MANY) >= 256) p.rows = 2 * ATTEND_MANY;
    p.tiles = (uint32_t)std::max<uint64_t>(1, divided_up(rows, p.rows));
    p.units = (uint32_t)(lists ? seqs * max_tokens : seqs);
    p.groups = (uint64_t)p.units * heads * p.tiles;
    const uint64_t chunks = std::max<uint64_t>(1, divided_up(length, ATTEND_CHUNK));
    const uint64_t target = p.few ? attend_target(true, dim) : attend_target(false, dim) * ATTEND_MANY / p.rows;
    p.waves = p.few ? 4 : p.rows / 32;
    // a part has work for the four waves of a workgroup (one step each) or, of many rows, for a few steps
    uint64_t parts = std::min(std::max<uint64_t>(1, target / std::max<uint64_t>(1, p.groups)), divided_up(chunks, 4));
    // up to 16 steps are done by one workgroup of eight waves rather than split and joined (16 sequences up to 1000 of dim 128: 14.8 us, split 16.1; up
    // to 700 12.3 and 15.2; of wider heads its waves have too few registers)
    if (p.few && parts > 1 && chunks <= 16 && dim <= 160) {
        p.waves = 8;
        parts = 1;
    }
    p.part_chunks = (uint32_t)divided_up(chunks, std::max<uint64_t>(1, parts));
    p.parts = (uint32_t)divided_up(chunks, p.part_chunks);
    if (p.parts > 1) p.bytes = attend_bytes(p.groups * p.parts * p.rows, dim, &p.sums);
    return p;
}

// The launches of a plan's workgroups: launch(first, workgroups) (groups * parts are fewer than 2^32).
template <typename F>
void attend_launches(const AttendPlan& p, F launch) {
    in_launches(p.groups * p.parts, 1, 64 * p.waves, [&](uint64_t first, uint64_t, uint32_t workgroups) { launch((uint32_t)first, workgroups); });
}

// What serves every call of these sizes or smaller ones: a call that is split has at most its form's target of workgroups.
inline size_t attend_workspace_upto(uint64_t max_tokens, uint32_t group, uint32_t dim, uint64_t length, bool lists) {
    if (divided_up(length, ATTEND_CHUNK) <= 4) return 0;
    const uint64_t few = (uint64_t)attend_target(true, dim) * ATTEND_FEW, many = (uint64_t)attend_target(false, dim) * ATTEND_MANY;
    return attend_bytes(lists || max_tokens * group <= ATTEND_FEW_ROWS ? few : std::max(few, many), dim, nullptr);
}

// Scores of the pages of a batch's tokens; all ones for more than any memory holds.
inline size_t select_workspace(uint64_t tokens, uint64_t heads, uint64_t table_pages) {
    if (tokens * heads >= 1ull << 40 || (tokens * heads) >> 20 >= (1ull << 28) / table_pages) return ~(size_t)0;
    return (tokens * heads * table_pages * 4 + 255) / 256 * 256;
}

// ---- pages ------------------------------------------------------------------------------------------------------------------
struct AdvancePlan {
    size_t writers, lowest, stays, free_pages, copies, bytes;
};
inline AdvancePlan advance_plan(uint64_t pages, uint64_t seqs) {
    AdvancePlan p{};
    size_t at = 0;
    auto take = [&](size_t n) {
        const size_t here = at;
        at += (n + 255) / 256 * 256;
        return here;
    };
    p.writers = take(pages * 4);
    p.lowest = take(pages * 4);
    p.stays = take(pages * 4);
    p.free_pages = take(pages * 4);
    p.copies = take(seqs * 8);
    p.bytes = at;
    return p;
}

struct CompactPlan {
    size_t moved, holes, totals, bytes;
};
inline CompactPlan compact_plan(uint64_t pages) {
    CompactPlan p{};
    const size_t one = (pages * 4 + 255) / 256 * 256;
    p.totals = 0;
    p.moved = 256;
    p.holes = p.moved + one;
    p.bytes = p.holes + one;
    return p;
}

}  // namespace dessert
