// How the row operators go about a call of given sizes, and the scratch memory that takes (host code, no HIP).
#pragma once
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

namespace dessert {

constexpr uint32_t LOGPROB_MAX_TOP = 64;   // one entry of the list a lane
constexpr uint32_t HEAD_GROUP = 128;       // channels of the vocabulary to a group

inline size_t align_bytes(size_t x, size_t a) { return (x + a - 1) / a * a; }

// ---- scaled products --------------------------------------------------------------------------------------------------------
// unit: the rows lie at multiples of 16 bytes, of 4, or of 1.
// Which numbers of tokens.  From 17 on the tiles' waves, which share what they read, are better where the channels are many or the columns
// very many: 32 tokens x 4096 x 1024 4.3 by columns, 5.7 us by tiles, x 8000 x 1024 7.5 / 6.9, x 32000 x 1024 15.9 / 14.5, x 4096 x 4096 9.7 /
// 12.5, x 1024 x 8192 15.1 / 11.9; 16 tokens x 16000 x 256 3.6 / 4.4, x 16000 x 2048 13.2 / 12.0.  Rows at odd bytes cost a wave more
// here, as the tiles' parts of the columns keep more waves busy (1 token x 1024 x 4097 10.0 / 12.8, x 8191 17.5 / 17.2; 16 x 1024 x 2049 9.5 /
// 10.3, x 4097 17.3 / 11.4; 32 x 1024 x 8193 46.6 / 18.7).
inline bool by_columns(uint64_t m, uint64_t n, uint32_t k, int unit) {
    if (k < 16) return false;
    if (m <= 16) return unit >= 4 || k < (m == 1 ? 8192 : 4096);
    return unit >= 4 && m <= 32 && k < 8192 && n <= 4096;
}

// Into how many parts the columns of a product in small tiles go, where the tiles alone leave CUs idle for long: 1 / 2 / 4 / 8 parts
// of 64 x 4096 x 4096 (64 tiles) 13.6 / 13.5 / 12.5 / 15.2 us, of 128 x 4096 x 4096 (128 tiles) 13.6 / 14.7 / 16.1 / 18.5, of 128 x 1024 x 8192
// (32 tiles) 21.5 / 18.8 / 13.6 / 12.6, of 128 x 4096 x 8192 (128 tiles) 23.1 / 20.9 / 18.2 / 25.1, of 64 x 4096 x 2048 (64 tiles) 8.8 / 10.2 / 10.4.
// At other addresses a step takes five times as long and parts pay sooner: 1 / 4 / 8 of 64 x 4096 x 8193 78 / 28.0 / 21.6, of 128 x 4096 x 8193 (128
// tiles) 78 / 29.7 / 35.5, of 64 x 1024 x 2049 19.4 / 11.3; 1 / 4 of 512 x 4096 x 8193 (512 tiles) 75 / 89.
inline uint32_t column_parts(uint64_t m, uint64_t n, uint32_t k, int unit) {
    const uint64_t tiles = ((m + 63) / 64) * ((n + 63) / 64);
    if (by_columns(m, n, k, unit)) return 1;
    if (unit >= 4) return k < 4096 || k < 64 * tiles ? 1 : k >= 8192 && k >= 256 * tiles ? 8 : 4;
    return k < 2048 || k < 16 * tiles || tiles > 256 ? 1 : k >= 4096 && tiles <= 64 ? 8 : 4;
}

inline size_t parts_bytes(uint64_t m, uint64_t n, uint32_t parts) { return parts < 2 ? 0 : (size_t)parts * m * ((n + 63) / 64 * 64) * 4; }

inline size_t scaled_matmul_workspace(uint64_t m, uint64_t n, uint32_t k) {
    uint32_t parts = 1;   // the most of any addresses that rows of k columns can have
    for (int unit : {1, 4, 16})
        if (k % unit == 0) parts = std::max(parts, column_parts(m, n, k, unit));
    return parts_bytes(m, n, parts);
}

// The most that any number of rows up to m needs.  For one number of parts the bytes grow with the rows, and the parts end where the tiles
// pass one of column_parts' limits (rows by columns need none): the last rows before each limit and m itself are all there is to look at.
inline size_t scaled_matmul_workspace_upto(uint64_t m, uint64_t n, uint32_t k) {
    const uint64_t across = std::max<uint64_t>((n + 63) / 64, 1);
    size_t bytes = scaled_matmul_workspace(m, n, k);
    for (uint64_t tiles : {(uint64_t)64, (uint64_t)256, (uint64_t)k / 16, (uint64_t)k / 64, (uint64_t)k / 256})
        bytes = std::max(bytes, scaled_matmul_workspace(std::min(m, tiles / across * 64), n, k));
    return bytes;
}

// ---- log probabilities ------------------------------------------------------------------------------------------------------
struct LogprobPlan {
    uint32_t splits, segment;   // of a row over workgroups
    size_t sums_bytes, bytes;   // workspace: of the sums, and altogether
};
// A row to a workgroup, or to several and a second launch that joins them: 1 workgroup / several for 384 rows x 4000 7.9 / 12.4 us, x 32000
// 20.2 / 24.1, x 128000 56.5 / 43.5, for 700 rows x 128000 65.1 / 60.4, for 1023 x 32000 27.5 / 33.3, x 128000 73.8 / 75.1 (bf16, 10 alternatives).
inline LogprobPlan logprob_plan(uint64_t rows, uint32_t vocab, uint32_t n_top) {
    LogprobPlan p{};
    if (rows >= 1024 || vocab <= 2048 || vocab <= 96 * rows) {
        p.segment = (vocab + 8191) / 8192 * 8192;
    } else {
        // a few workgroups a CU
        uint64_t splits = (2048 + rows - 1) / rows, most = (vocab + 2047) / 2048;
        if (splits > most) splits = most;
        p.segment = (uint32_t)(((vocab + splits - 1) / splits + 2047) / 2048 * 2048);
    }
    p.splits = (vocab + p.segment - 1) / p.segment;
    if (p.splits > 1) {
        p.sums_bytes = ((size_t)rows * p.splits * 12 + 255) / 256 * 256;
        p.bytes = p.sums_bytes + ((size_t)rows * p.splits * n_top * 8 + 255) / 256 * 256;
    }
    return p;
}

// Enough for any number of rows up to `rows`: their parts are at most 2047 + rows, and `most` a row.
inline size_t logprob_workspace_upto(uint64_t rows, uint32_t vocab, uint32_t n_top) {
    if (vocab <= 2048) return 0;
    const uint64_t r = std::min<uint64_t>(std::min<uint64_t>(rows, 1023), (vocab - 1) / 96);
    const uint64_t parts = std::min<uint64_t>(r * ((vocab + 2047) / 2048), 2047 + r);
    return align_bytes(parts * 12, 256) + align_bytes(parts * n_top * 8, 256);
}

// ---- log probabilities from states ------------------------------------------------------------------------------------------
// The head form goes through the rows in turns: by a product that writes the turn's 32-bit logits and a pass that reads them while they still lie in
// the 256 MB cache, or by groups of the vocabulary, without most of the logits (kernels.hpp).
// Of 16 calls that go by logits (1024 to 16384 rows, vocabularies of 4000 to 128000, 130 to 4096 columns, rows at 16, 4 and odd bytes) turns of at most
// 128 / 200 / 400 MB take 1.06 / 0.99 / 1.02 times what 256 MB take on average, and 0.87 to 1.67 / 0.89 to 1.20 / 0.90 to 1.13 times.
constexpr size_t HEAD_TURN_BYTES = 256u << 20;
struct HeadPlan {
    uint64_t rows;     // of a turn
    uint64_t stride;   // floats from row to row
    LogprobPlan pass;
    size_t logits_bytes, pass_bytes, bytes;
};
inline HeadPlan head_plan(uint64_t rows, uint32_t vocab, uint32_t k, uint32_t n_top) {
    HeadPlan h{};
    h.stride = ((uint64_t)vocab + 31) / 32 * 32;
    // Of the numbers of rows that fit, the one with the least time a row: whole rounds of 256 x 256 tiles over the 256 CUs, a third of a
    // round's time for each 256 tiles' worth of logits to read, and a seventh for two launches.  (The 16 calls above with every number of rows: this
    // choice takes 1.04 times the best one's time on average; 1.07 to 1.15 times where rows at odd bytes go in tiles of 128 x 128.)
    const uint64_t across = (vocab + 255) / 256, most = std::min<uint64_t>((rows + 255) / 256, HEAD_TURN_BYTES / (1024 * h.stride));
    double best = 1e30;
    h.rows = 256;
    for (uint64_t n = 1; n <= most && n <= 4096; ++n) {
        const uint64_t tiles = n * across, rounds = (tiles + 255) / 256;
        const double cost = (rounds + 0.35 * tiles / 256 + 0.15) / n;
        if (cost < best * 0.999) {
            best = cost;
            h.rows = n * 256;
        }
    }
    if (h.rows > rows) h.rows = rows;
    h.pass = logprob_plan(h.rows, vocab, n_top);
    h.logits_bytes = align_bytes((size_t)h.rows * h.stride * 4, 256);
    h.pass_bytes = align_bytes(h.pass.bytes, 256);
    h.bytes = h.logits_bytes + h.pass_bytes + scaled_matmul_workspace(h.rows, vocab, k);
    return h;
}

struct GroupPlan {
    uint64_t rows;     // of a turn, 0: does not pay
    uint32_t groups;
    size_t sums, counts, lists, picked, totals, logits, bytes;
};
// Where groups pay, in us: they save a logit's way to memory and back, 1.1 us for 10^6 of them, and spend three launches and, for each row and
// alternative, its picking and the products of a group.  Logits / groups: 4096 x 32000 x 2048 with 5, 10, 20, 33, 64 alternatives 423 / 308, 418 / 354,
// 427 / 431, 434 / 528, 448 / 764; x 128 columns 223 / 110, 227 / 132, 233 / 183, 242 / 242, 268 / 383; 1024 x 32000 x 1024 with 0, 5, 10, 20 77 / 46,
// 79 / 68, 80 / 76, 87 / 95; 300 x 128000 x 1024 with 5, 33, 64 130 / 114, 149 / 143, 155 / 168; 16384 x 4000 x 512 with 0, 1, 5 131 / 82, 134 / 130, 139 / 207;
// 128 x 50000 x 1024 with 0, 1 38 / 27, 41 / 45.  220 calls drawn apart from those that the numbers were fitted to (64 to 16384 rows, vocabularies of 2048
// to 150000, 32 to 4096 columns, 0 to 64 alternatives): 1.004 times the better one's time on average, 1.38 at most.
// The tiles of 256 x 256 that groups are formed in have to fill half of the 256 CUs: 512 x 4000 x 2048 (32 tiles) without alternatives
// 19 / 34, 64 x 32000 x 1024 (125) 23 / 25, 512 x 16000 x 1024 (126) 29 / 26.
inline bool groups_pay(uint64_t rows, uint32_t vocab, uint32_t k, uint32_t n_top) {
    if (((rows + 255) / 256) * ((vocab + 255) / 256) < 128) return false;
    return n_top == 0 || 1.1e-6 * rows * vocab > 9 + 1e-3 * rows * n_top * (0.9 + 0.0005 * k);
}

inline GroupPlan group_plan(uint64_t rows, uint32_t vocab, uint32_t k, uint32_t n_top) {
    GroupPlan p{};
    p.groups = (vocab + HEAD_GROUP - 1) / HEAD_GROUP;
    if (!groups_pay(rows, vocab, k, n_top)) return p;
    const size_t row_bytes = (size_t)p.groups * (16 + 4) + (size_t)n_top * (4 + 4 * HEAD_GROUP) + 8;
    p.rows = HEAD_TURN_BYTES / row_bytes / 256 * 256;
    if (p.rows < 256) p.rows = 256;
    if (p.rows > rows) p.rows = rows;
    const auto place = [&](size_t bytes) {
        const size_t at = p.bytes;
        p.bytes += align_bytes(bytes, 256);
        return at;
    };
    p.sums = place((size_t)p.rows * p.groups * 16);
    p.counts = place((size_t)p.groups * 4);
    p.lists = place(n_top ? (size_t)p.groups * p.rows * 4 : 0);
    p.picked = place((size_t)p.rows * n_top * 4);
    p.totals = place((size_t)p.rows * 8);
    p.logits = place((size_t)p.rows * n_top * HEAD_GROUP * 4);
    return p;
}

// Enough for any number of rows up to `rows`, whichever of the two it is (that depends on how the rows lie).  A turn's rows do not fall as the
// rows of the call rise.
inline size_t head_workspace_upto(uint64_t rows, uint32_t vocab, uint32_t k, uint32_t n_top) {
    const HeadPlan h = head_plan(rows, vocab, k, n_top);
    const size_t pass = align_bytes(logprob_workspace_upto(h.rows, vocab, n_top), 256);
    return std::max(h.logits_bytes + pass + scaled_matmul_workspace_upto(h.rows, vocab, k), group_plan(rows, vocab, k, n_top).bytes);
}

}  // namespace dessert
