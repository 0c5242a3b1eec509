// Pages of a paged cache: sequences that go on from others, and the pages in use brought together.  A page's count says how many tables hold
// it; a page that more than one holds is copied before a sequence writes to it.  Decisions are made by one workgroup (a few thousand numbers,
// in order), pages are moved by as many as fill the chip: bound by latency, then by memory.
#include "cache_common.hpp"

namespace dessert {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ inline uint32_t load_now(const uint32_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// A barrier behind which what the workgroup's waves stored and added is in L2, where load_now finds it.  (A fence over the whole device would also
// write L2 back, a few microseconds each time.)
__device__ inline void arrived() {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    barrier();
}

struct AdvanceWork {
    uint32_t *writers, *lowest, *stays;   // [pages], only at pages that some sequence writes to
    uint32_t* free_pages;                 // [pages] the lowest ones, as many as are asked for
    uint2* copies;                        // [n_new] from, to; or from = NO_PAGE
};

struct Parent {
    uint32_t seq, length, have;   // have: pages of its length in the table
};

__device__ inline Parent parent_of(const AdvanceArgs& a, uint32_t shift, uint32_t b) {
    Parent p;
    p.seq = a.parents ? a.parents[b] : b;
    const bool there = p.seq < a.p.n_seqs;
    p.length = there ? min(a.p.lengths[p.seq], CACHE_MOST) : 0u;
    p.have = min((uint32_t)(((uint64_t)p.length + (1u << shift) - 1) >> shift), a.p.table_pages);
    return p;
}

// Tables of the new sequences; counts of the pages that old ones no longer hold and new ones do.
__global__ __launch_bounds__(256) void advance_tables_kernel(AdvanceArgs a, AdvanceWork w, uint32_t n_pages, uint32_t shift) {
    const uint64_t stride = a.p.table_pages, n = (uint64_t)max(a.n_new, a.p.n_seqs) * stride;
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (uint64_t)gridDim.x * 256) {
        const uint32_t b = (uint32_t)(i / stride), j = (uint32_t)(i % stride);
        if (b < a.n_new) {
            const Parent p = parent_of(a, shift, b);
            const uint32_t page = j < p.have ? a.p.tables[(uint64_t)p.seq * stride + j] : NO_PAGE;
            a.out_tables[i] = page;
            if (page < n_pages) {
                if (a.counts) atomicAdd(a.p.refs + page, 1u);
                if (j + 1 == p.have) {
                    w.writers[page] = 0;
                    w.lowest[page] = NO_PAGE;
                    w.stays[page] = 0;
                }
            }
        }
        if (a.counts && b < a.p.n_seqs && j < (uint32_t)(((uint64_t)min(a.p.lengths[b], CACHE_MOST) + (1u << shift) - 1) >> shift)) {
            const uint32_t page = a.p.tables[i];
            if (page < n_pages) atomicSub(a.p.refs + page, 1u);
        }
    }
}

// Sums over a workgroup of 1024: of the threads in front, and of all.
__device__ inline uint32_t before_1024(uint32_t x, uint32_t* parts, uint32_t& total) {
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t y = x;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
        const uint32_t z = __shfl_up((int)y, o);
        if (lane >= (uint32_t)o) y += z;
    }
    barrier();
    if (lane == 63) parts[wave] = y;
    barrier();
    uint32_t before = 0;
    total = 0;
#pragma unroll
    for (uint32_t k = 0; k < 16; ++k) {
        const uint32_t z = parts[k];
        before += k < wave ? z : 0u;
        total += z;
    }
    return before + y - x;
}

// What a new sequence wants: its pages in all, whether they fit its table, its last page so far and whether it writes there.
struct Wish {
    uint32_t length, have, total, last;
    bool fits, writes;
};

__device__ inline Wish wish_of(const AdvanceArgs& a, uint32_t n_pages, uint32_t shift, uint32_t b) {
    const Parent p = parent_of(a, shift, b);
    Wish w;
    w.length = p.length;
    w.have = p.have;
    const uint64_t add = a.add[b], total = ((uint64_t)p.length + add + (1u << shift) - 1) >> shift;
    w.fits = total <= a.p.table_pages && (uint64_t)p.length + add <= CACHE_MOST;
    w.total = w.fits ? (uint32_t)total : 0u;
    w.last = p.have ? a.p.tables[(uint64_t)p.seq * a.p.table_pages + p.have - 1] : NO_PAGE;
    w.writes = w.fits && add > 0 && (p.length & ((1u << shift) - 1)) && w.last < n_pages;
    return w;
}

// Who copies, who is granted pages, which ones.  In the order of the new sequences: as long as the free pages last.
__global__ __launch_bounds__(1024) void advance_decide_kernel(AdvanceArgs a, AdvanceWork w, uint32_t n_pages, uint32_t shift) {
    __shared__ uint32_t parts[16];
    __shared__ uint32_t refused, taken;
    const uint32_t n = a.n_new;
    if (threadIdx.x == 0) refused = taken = 0;
    // a page that all its holders write to stays with the first of them
    for (uint32_t b = threadIdx.x; b < n; b += 1024) {
        const Wish x = wish_of(a, n_pages, shift, b);
        if (x.writes) {
            atomicAdd(w.writers + x.last, 1u);
            atomicMin(w.lowest + x.last, b);
        }
    }
    arrived();
    // the pages asked for
    uint32_t asked = 0;
    for (uint32_t b0 = 0; b0 < n; b0 += 1024) {
        const uint32_t b = b0 + threadIdx.x;
        uint32_t need = 0, total;
        if (b < n) {
            const Wish x = wish_of(a, n_pages, shift, b);
            const uint32_t holders = x.writes ? load_now(a.p.refs + x.last) : 0;
            const bool keeps = x.writes && holders > 1 && load_now(w.writers + x.last) == holders && load_now(w.lowest + x.last) == b;
            const bool copies = x.writes && holders > 1 && !keeps;
            need = x.fits ? x.total - x.have + copies : 0u;
        }
        const uint32_t mine = before_1024(need, parts, total);
        if (b < n) w.copies[b] = make_uint2(asked + mine, need);
        asked += total;      // fewer than 2^32: no more than there are places in the tables
    }
    // the free pages, lowest first
    uint32_t free_count = 0;
    for (uint32_t p0 = 0; p0 < n_pages; p0 += 4096) {
        const uint32_t p = p0 + threadIdx.x * 4;
        uint32_t empty = 0, total;
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) empty |= (uint32_t)(p + i < n_pages && load_now(a.p.refs + p + i) == 0) << i;
        uint32_t at = free_count + before_1024(__popc(empty), parts, total);
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i)
            if (empty >> i & 1) {
                if (at < asked) w.free_pages[at] = p + i;
                ++at;
            }
        free_count += total;
    }
    barrier();
    // copies that are not granted leave their page with the one that would keep it, which is not granted then either
    for (uint32_t b = threadIdx.x; b < n; b += 1024) {
        const Wish x = wish_of(a, n_pages, shift, b);
        const uint2 want = w.copies[b];
        const bool granted = x.fits && (want.y == 0 || (uint64_t)want.x + want.y <= free_count);
        const bool copies = x.fits && want.y > x.total - x.have;
        if (copies && !granted) atomicExch(w.stays + x.last, 1u);
    }
    arrived();
    for (uint32_t b0 = 0; b0 < n; b0 += 16) {      // a wave a sequence
        const uint32_t b = b0 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
        if (b >= n) continue;
        const Wish x = wish_of(a, n_pages, shift, b);
        const uint2 want = w.copies[b];
        const bool copies = x.fits && want.y > x.total - x.have;
        bool granted = x.fits && (want.y == 0 || (uint64_t)want.x + want.y <= free_count);
        if (x.writes && !copies && load_now(w.lowest + x.last) == b && load_now(w.stays + x.last)) granted = false;
        if (granted)
            for (uint32_t i = lane; i < want.y; i += 64) {
                const uint32_t page = w.free_pages[want.x + i];
                a.out_tables[(uint64_t)b * a.p.table_pages + x.have - copies + i] = page;
                atomicExch(a.p.refs + page, 1u);
            }
        if (lane == 0) {
            const bool copied = copies && granted;
            w.copies[b] = copied ? make_uint2(x.last, w.free_pages[want.x]) : make_uint2(NO_PAGE, NO_PAGE);
            if (copied) atomicSub(a.p.refs + x.last, 1u);
            a.out_lengths[b] = granted ? x.length + a.add[b] : x.length;
            if (!granted) atomicAdd(&refused, 1u);
            else atomicAdd(&taken, want.y);
        }
    }
    barrier();
    if (threadIdx.x == 0) {
        a.status[0] = free_count - taken;
        a.status[1] = refused;
    }
}

// The same of up to 1024 sequences, one a thread: what they want stays in registers and LDS, the tables are made on the way where they are
// small, and a call that has pages for all skips the passes for those that get none.  Latency of its phases: 16 sequences 6.0 us, 128 with the tables made in a
// launch of their own 7.6 and 4.4 (all in one 18).
constexpr uint32_t ADVANCE_FEW = 1024, FREE_IN_LDS = 2048, ADVANCE_ENTRIES = 2048;
__global__ __launch_bounds__(1024) void advance_few_kernel(AdvanceArgs a, AdvanceWork w, uint32_t n_pages, uint32_t shift, bool make_tables) {
    __shared__ uint32_t parts[16], parents[ADVANCE_FEW], lengths[ADVANCE_FEW], before[ADVANCE_FEW], first_new[ADVANCE_FEW], free_lds[FREE_IN_LDS];
    __shared__ uint32_t refused, taken;
    const uint32_t n = a.n_new, b = threadIdx.x, stride = a.p.table_pages, slots = (1u << shift) - 1;
    if (b == 0) refused = taken = 0;
    Parent p{NO_PAGE, 0, 0};
    Wish x{0, 0, 0, NO_PAGE, false, false};
    uint32_t add = 0;
    if (b < n) {
        add = a.add[b];
        p = parent_of(a, shift, b);
        parents[b] = p.seq;
        lengths[b] = p.length;
        const uint64_t total = ((uint64_t)p.length + add + slots) >> shift;
        x.length = p.length;
        x.have = p.have;
        x.fits = total <= stride && (uint64_t)p.length + add <= CACHE_MOST;
        x.total = x.fits ? (uint32_t)total : 0u;
        x.last = p.have ? a.p.tables[(uint64_t)p.seq * stride + p.have - 1] : NO_PAGE;
        x.writes = x.fits && add > 0 && (p.length & slots) && x.last < n_pages;
        if (make_tables && x.last < n_pages) {
            w.writers[x.last] = 0;
            w.lowest[x.last] = NO_PAGE;
            w.stays[x.last] = 0;
        }
    }
    barrier();
    if (make_tables) {
        for (uint32_t i = threadIdx.x; i < max(n, a.p.n_seqs) * stride; i += 1024) {
            const uint32_t s = i / stride, j = i % stride;
            if (s < n) {
                const bool inside = j < min((uint32_t)(((uint64_t)lengths[s] + slots) >> shift), stride);
                const uint32_t page = inside ? a.p.tables[(uint64_t)parents[s] * stride + j] : NO_PAGE;
                a.out_tables[i] = page;
                if (page < n_pages && a.counts) atomicAdd(a.p.refs + page, 1u);
            }
            if (a.counts && s < a.p.n_seqs && j < (uint32_t)(((uint64_t)min(a.p.lengths[s], CACHE_MOST) + slots) >> shift)) {
                const uint32_t page = a.p.tables[i];
                if (page < n_pages) atomicSub(a.p.refs + page, 1u);
            }
        }
        arrived();
    }
    if (x.writes) {
        atomicAdd(w.writers + x.last, 1u);
        atomicMin(w.lowest + x.last, b);
    }
    arrived();
    const uint32_t holders = x.writes ? load_now(a.p.refs + x.last) : 0;
    const bool keeps = holders > 1 && load_now(w.writers + x.last) == holders && load_now(w.lowest + x.last) == b, copies = holders > 1 && !keeps;
    const uint32_t need = x.fits ? x.total - x.have + copies : 0u;
    uint32_t asked;
    const uint32_t from = before_1024(need, parts, asked);
    if (b < n) before[b] = from;
    uint32_t free_count = 0;
    for (uint32_t p0 = 0; p0 < n_pages; p0 += 4096) {
        const uint32_t q = p0 + threadIdx.x * 4;
        uint32_t empty = 0, total;
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) empty |= (uint32_t)(q + i < n_pages && load_now(a.p.refs + min(q + i, n_pages - 1)) == 0) << i;
        uint32_t at = free_count + before_1024(__popc(empty), parts, total);
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i)
            if (empty >> i & 1) {
                if (at < min(asked, FREE_IN_LDS)) free_lds[at] = q + i;
                else if (at < asked) w.free_pages[at] = q + i;
                ++at;
            }
        free_count += total;
    }
    bool granted = b < n && x.fits && (need == 0 || from + need <= free_count);
    if (asked > free_count) {      // the same in all threads
        if (copies && !granted) atomicExch(w.stays + x.last, 1u);
        arrived();
        if (keeps && load_now(w.stays + x.last)) granted = false;
    }
    if (b < n) first_new[b] = granted ? x.have - copies : NO_PAGE;
    barrier();
    for (uint32_t i = threadIdx.x; i < min(asked, free_count); i += 1024) {
        uint32_t lo = 0, hi = n;           // the last sequence that begins at or before i and asks for something
        while (hi - lo > 1) {
            const uint32_t mid = (lo + hi) / 2;
            if (before[mid] <= i) lo = mid;
            else hi = mid;
        }
        if (first_new[lo] == NO_PAGE) continue;
        const uint32_t page = i < FREE_IN_LDS ? free_lds[i] : w.free_pages[i];
        a.out_tables[(uint64_t)lo * stride + first_new[lo] + i - before[lo]] = page;
        a.p.refs[page] = 1;
    }
    if (b < n) {
        const bool copied = copies && granted;
        w.copies[b] = copied ? make_uint2(x.last, from < FREE_IN_LDS ? free_lds[from] : w.free_pages[from]) : make_uint2(NO_PAGE, NO_PAGE);
        if (copied) atomicSub(a.p.refs + x.last, 1u);
        a.out_lengths[b] = granted ? x.length + add : x.length;
        if (!granted) atomicAdd(&refused, 1u);
        else if (need) atomicAdd(&taken, need);
    }
    barrier();
    if (b == 0) {
        a.status[0] = free_count - taken;
        a.status[1] = refused;
    }
}

struct PageCopy {
    CacheLayers layers;
    uint32_t heads, page_tokens, dim;
};

// A piece of a page of a layer: 8 KB of its keys, the same of its values, their part of the bounds; with the first the scales.  All is under
// way before the first is written.
constexpr uint32_t PIECE = 8192;
__device__ inline void copy_page(const PageCopy& c, uint32_t layer, uint32_t from, uint32_t to, uint32_t piece) {
    const uint64_t codes = (uint64_t)c.heads * c.page_tokens * c.dim / 16, bound = (uint64_t)c.heads * 2 * c.dim / 16;
    u32x4 *k = (u32x4*)c.layers.k[layer], *v = (u32x4*)c.layers.v[layer], *bounds = (u32x4*)c.layers.bounds[layer];
    const uint64_t i0 = (uint64_t)piece * (PIECE / 16) + threadIdx.x, i1 = i0 + 256, ib = (uint64_t)piece * 256 + threadIdx.x;
    const bool has0 = i0 < codes, has1 = i1 < codes, has_bound = bounds && ib < bound, scale = piece == 0 && threadIdx.x < c.heads;
    u32x4 k0, k1, v0, v1, b0;
    float ks, vs;
    if (has0) k0 = k[from * codes + i0], v0 = v[from * codes + i0];
    if (has1) k1 = k[from * codes + i1], v1 = v[from * codes + i1];
    if (has_bound) b0 = bounds[from * bound + ib];
    if (scale) ks = c.layers.ks[layer][(uint64_t)from * c.heads + threadIdx.x], vs = c.layers.vs[layer][(uint64_t)from * c.heads + threadIdx.x];
    if (has0) k[to * codes + i0] = k0, v[to * codes + i0] = v0;
    if (has1) k[to * codes + i1] = k1, v[to * codes + i1] = v1;
    if (has_bound) bounds[to * bound + ib] = b0;
    if (scale) c.layers.ks[layer][(uint64_t)to * c.heads + threadIdx.x] = ks, c.layers.vs[layer][(uint64_t)to * c.heads + threadIdx.x] = vs;
    if (piece == 0)
        for (uint32_t i = threadIdx.x + 256; i < c.heads; i += 256) {
            c.layers.ks[layer][(uint64_t)to * c.heads + i] = c.layers.ks[layer][(uint64_t)from * c.heads + i];
            c.layers.vs[layer][(uint64_t)to * c.heads + i] = c.layers.vs[layer][(uint64_t)from * c.heads + i];
        }
}

__global__ __launch_bounds__(256) void advance_copy_kernel(PageCopy c, const uint2* copies, uint32_t pieces) {
    const uint2 move = copies[blockIdx.x / pieces];
    if (move.x == NO_PAGE) return;
    for (uint32_t layer = blockIdx.y; layer < c.layers.n; layer += gridDim.y) copy_page(c, layer, move.x, move.y, blockIdx.x % pieces);
}

// ---- compaction -----------------------------------------------------------------------------------------------------------------
// Numbers after it: pages in use keep theirs below the number of them; those above go into the holes below, lowest to lowest.
__global__ __launch_bounds__(1024) void compact_decide_kernel(const uint32_t* refs, uint32_t n_pages, uint32_t* moved, uint32_t* holes, uint32_t* totals,
                                                              uint32_t* numbers, uint32_t* live_out) {
    __shared__ uint32_t parts[16];
    uint32_t count = 0, live;
    for (uint32_t p = threadIdx.x; p < n_pages; p += 1024) count += refs[p] != 0;
    (void)before_1024(count, parts, live);
    uint32_t n_moved = 0, n_holes = 0;
    for (uint32_t p0 = 0; p0 < n_pages; p0 += 4096) {
        const uint32_t p = p0 + threadIdx.x * 4;
        uint32_t used[4], mine = 0, all;       // pages that move, and holes in the upper half: at most 4096 of each
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) used[i] = refs[min(p + i, n_pages - 1)];
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i)
            if (p + i < n_pages) mine += used[i] ? (uint32_t)(p + i >= live) : (uint32_t)(p + i < live) << 16;
        const uint32_t before = before_1024(mine, parts, all);
        uint32_t at_moved = n_moved + (before & 0xFFFF), at_hole = n_holes + (before >> 16);
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i)
            if (p + i < n_pages) {
                if (used[i] && p + i >= live) moved[at_moved++] = p + i;
                else numbers[p + i] = used[i] ? p + i : NO_PAGE;
                if (!used[i] && p + i < live) holes[at_hole++] = p + i;
            }
        n_moved += all & 0xFFFF;
        n_holes += all >> 16;
    }
    arrived();
    for (uint32_t i = threadIdx.x; i < n_moved; i += 1024) numbers[load_now(moved + i)] = load_now(holes + i);
    if (threadIdx.x == 0) {
        totals[0] = n_moved;
        live_out[0] = live;
    }
}

// Moves the pages, and (with tables) the tables' entries and counts.  Bound by memory: 320 pages of 3 layers (262 MB read and written) 56 us, 4.7 TB/s.
__global__ __launch_bounds__(256) void compact_copy_kernel(PageCopy c, PagesArgs p, const uint32_t* moved, const uint32_t* holes, const uint32_t* totals,
                                                           const uint32_t* numbers, uint32_t n_pages, uint32_t shift, uint32_t pieces, bool tables) {
    const uint32_t n_moved = totals[0];
    if (tables) {
        const uint64_t first = (uint64_t)blockIdx.x * 256 + threadIdx.x, step = (uint64_t)gridDim.x * 256;
        for (uint64_t i = first; i < n_moved; i += step) {
            p.refs[holes[i]] = p.refs[moved[i]];
            p.refs[moved[i]] = 0;
        }
        for (uint64_t i = first; i < (uint64_t)p.n_seqs * p.table_pages; i += step) {
            const uint32_t b = (uint32_t)(i / p.table_pages), j = (uint32_t)(i % p.table_pages), page = p.tables[i];
            if (j < (uint32_t)(((uint64_t)min(p.lengths[b], CACHE_MOST) + (1u << shift) - 1) >> shift) && page < n_pages) p.tables[i] = numbers[page];
        }
    }
    const uint64_t n = (uint64_t)n_moved * c.layers.n * pieces;
    for (uint64_t i = blockIdx.x; i < n; i += gridDim.x) {
        const uint32_t piece = (uint32_t)(i % pieces), layer = (uint32_t)(i / pieces % c.layers.n), at = (uint32_t)(i / pieces / c.layers.n);
        copy_page(c, layer, moved[at], holes[at], piece);
    }
}

// Layers in turns of CACHE_LAYERS.
template <typename F>
void with_layers(const PagesArgs& p, F launch) {
    for (uint32_t l = 0; l < p.n_layers; l += CACHE_LAYERS) {
        PageCopy c{};
        c.heads = p.layers[0].heads;
        c.page_tokens = p.layers[0].page_tokens;
        c.dim = p.layers[0].dim;
        c.layers.n = std::min(CACHE_LAYERS, p.n_layers - l);
        for (uint32_t i = 0; i < c.layers.n; ++i) {
            const CachePages& x = p.layers[l + i];
            c.layers.k[i] = x.k;
            c.layers.v[i] = x.v;
            c.layers.ks[i] = x.ks;
            c.layers.vs[i] = x.vs;
            c.layers.bounds[i] = x.bounds;
        }
        launch(c);
    }
}

uint32_t entry_blocks(uint64_t entries) { return (uint32_t)std::min<uint64_t>(std::max<uint64_t>(1, divided_up(entries, 256)), 2048); }

uint32_t page_pieces(const CachePages& c) { return (uint32_t)divided_up((uint64_t)c.heads * c.page_tokens * c.dim, PIECE); }

}  // namespace

hipError_t launch_cache_advance(const AdvanceArgs& a, void* workspace, hipStream_t stream) {
    const CachePages& c = a.p.layers[0];
    const AdvancePlan plan = advance_plan(c.n_pages, a.n_new);
    char* ws = (char*)workspace;
    AdvanceWork w;
    w.writers = (uint32_t*)(ws + plan.writers);
    w.lowest = (uint32_t*)(ws + plan.lowest);
    w.stays = (uint32_t*)(ws + plan.stays);
    w.free_pages = (uint32_t*)(ws + plan.free_pages);
    w.copies = (uint2*)(ws + plan.copies);
    const uint64_t entries = (uint64_t)std::max(a.n_new, a.p.n_seqs) * a.p.table_pages;
    const bool few = a.n_new <= ADVANCE_FEW, with_tables = few && entries <= ADVANCE_ENTRIES;
    if (!with_tables) advance_tables_kernel<<<dim3(entry_blocks(entries)), dim3(256), 0, stream>>>(a, w, c.n_pages, c.shift);
    if (few) advance_few_kernel<<<dim3(1), dim3(1024), 0, stream>>>(a, w, c.n_pages, c.shift, with_tables);
    else advance_decide_kernel<<<dim3(1), dim3(1024), 0, stream>>>(a, w, c.n_pages, c.shift);
    if (a.n_new == 0) return hipGetLastError();
    const uint32_t pieces = page_pieces(c);
    with_layers(a.p, [&](const PageCopy& copy) {
        advance_copy_kernel<<<dim3(a.n_new * pieces, copy.layers.n), dim3(256), 0, stream>>>(copy, w.copies, pieces);
    });
    return hipGetLastError();
}

hipError_t launch_cache_compact(const CompactArgs& a, void* workspace, hipStream_t stream) {
    const CachePages& c = a.p.layers[0];
    const CompactPlan plan = compact_plan(c.n_pages);
    char* ws = (char*)workspace;
    uint32_t *totals = (uint32_t*)(ws + plan.totals), *moved = (uint32_t*)(ws + plan.moved), *holes = (uint32_t*)(ws + plan.holes);
    compact_decide_kernel<<<dim3(1), dim3(1024), 0, stream>>>(a.p.refs, c.n_pages, moved, holes, totals, a.numbers, a.live);
    const uint32_t pieces = page_pieces(c);
    const uint64_t entries = std::max<uint64_t>((uint64_t)a.p.n_seqs * a.p.table_pages, c.n_pages / 2);
    bool tables = true;
    with_layers(a.p, [&](const PageCopy& copy) {
        const uint64_t most = (uint64_t)(c.n_pages / 2) * copy.layers.n * pieces;    // as many pages move as there are holes
        const uint32_t blocks = (uint32_t)std::min<uint64_t>(std::max<uint64_t>(most, entry_blocks(entries)), 2048);
        compact_copy_kernel<<<dim3(blocks), dim3(256), 0, stream>>>(copy, a.p, moved, holes, totals, a.numbers, c.n_pages, c.shift, pieces, tables);
        tables = false;
    });
    return hipGetLastError();
}

}  // namespace dessert
