// Pages of a paged cache: sequences that go on from others, and the pages in use brought together.  A page's count says how many tables hold
// it; a page that more than one holds is copied before a sequence writes to it.  Decisions are made by one workgroup (a few thousand numbers,
// in order), pages are moved by as many as fill the chip: bound by latency, then by memory.
#include "cache_common.hpp"

namespace dessert {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ inline uint32_t load_now(const uint32_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

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
    __syncthreads();
    if (lane == 63) parts[wave] = y;
    __syncthreads();
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
    __threadfence();
    __syncthreads();
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
        // beyond 2^32 nobody is granted anything more
        asked = asked + total < asked ? 0xFFFFFFFFu : asked + total;
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
    __syncthreads();
    // copies that are not granted leave their page with the one that would keep it, which is not granted then either
    for (uint32_t b = threadIdx.x; b < n; b += 1024) {
        const Wish x = wish_of(a, n_pages, shift, b);
        const uint2 want = w.copies[b];
        const bool granted = x.fits && (want.y == 0 || (uint64_t)want.x + want.y <= free_count);
        const bool copies = x.fits && want.y > x.total - x.have;
        if (copies && !granted) atomicExch(w.stays + x.last, 1u);
    }
    __threadfence();
    __syncthreads();
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
    __syncthreads();
    if (threadIdx.x == 0) {
        a.status[0] = free_count - taken;
        a.status[1] = refused;
    }
}

// Bytes of a page of a layer, in this order: keys, values, bounds, scales.
struct PageCopy {
    CacheLayers layers;
    uint32_t heads, page_tokens, dim;
};

__device__ inline void copy_page(const PageCopy& c, uint32_t layer, uint32_t from, uint32_t to, uint32_t piece, uint32_t pieces) {
    const uint64_t codes = (uint64_t)c.heads * c.page_tokens * c.dim, bound = (uint64_t)c.heads * 2 * c.dim;
    auto move = [&](int8_t* base, uint64_t bytes) {
        const u32x4* x = (const u32x4*)(base + from * bytes);
        u32x4* y = (u32x4*)(base + to * bytes);
        const uint32_t n = (uint32_t)(bytes / 16);
        for (uint32_t i = piece * 256 + threadIdx.x; i < n; i += pieces * 256) y[i] = x[i];
    };
    move(c.layers.k[layer], codes);
    move(c.layers.v[layer], codes);
    if (c.layers.bounds[layer]) move(c.layers.bounds[layer], bound);
    if (piece == 0)
        for (uint32_t i = threadIdx.x; i < c.heads; i += 256) {
            c.layers.ks[layer][(uint64_t)to * c.heads + i] = c.layers.ks[layer][(uint64_t)from * c.heads + i];
            c.layers.vs[layer][(uint64_t)to * c.heads + i] = c.layers.vs[layer][(uint64_t)from * c.heads + i];
        }
}

__global__ __launch_bounds__(256) void advance_copy_kernel(PageCopy c, const uint2* copies, uint32_t pieces) {
    const uint2 move = copies[blockIdx.x / pieces];
    if (move.x == NO_PAGE) return;
    for (uint32_t layer = blockIdx.y; layer < c.layers.n; layer += gridDim.y) copy_page(c, layer, move.x, move.y, blockIdx.x % pieces, pieces);
}

// ---- compaction -----------------------------------------------------------------------------------------------------------------
// Numbers after it: pages in use keep theirs below the number of them; those above go into the holes below, lowest to lowest.
__global__ __launch_bounds__(1024) void compact_decide_kernel(const uint32_t* refs, uint32_t n_pages, uint32_t* moved, uint32_t* holes, uint32_t* totals,
                                                              uint32_t* numbers, uint32_t* live_out) {
    __shared__ uint32_t parts[16];
    uint32_t count = 0, live, rest;
    for (uint32_t p = threadIdx.x; p < n_pages; p += 1024) count += refs[p] != 0;
    (void)before_1024(count, parts, live);
    uint32_t n_moved = 0, n_holes = 0;
    for (uint32_t p0 = 0; p0 < n_pages; p0 += 1024) {
        const uint32_t p = p0 + threadIdx.x;
        const bool here = p < n_pages, used = here && refs[p] != 0;
        const bool moves = used && p >= live, hole = here && !used && p < live;
        const uint32_t at_moved = n_moved + before_1024(moves, parts, rest);
        n_moved += rest;
        const uint32_t at_hole = n_holes + before_1024(hole, parts, rest);
        n_holes += rest;
        if (moves) moved[at_moved] = p;
        if (hole) holes[at_hole] = p;
        if (here && !moves) numbers[p] = used ? p : NO_PAGE;
    }
    __threadfence();
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < n_moved; i += 1024) {
        const uint32_t from = load_now(moved + i), to = load_now(holes + i);
        numbers[from] = to;
    }
    if (threadIdx.x == 0) {
        totals[0] = n_moved;
        live_out[0] = live;
    }
}

__global__ __launch_bounds__(256) void compact_copy_kernel(PageCopy c, const uint32_t* moved, const uint32_t* holes, const uint32_t* totals, uint32_t pieces) {
    const uint64_t n = (uint64_t)totals[0] * c.layers.n * pieces;
    for (uint64_t i = blockIdx.x; i < n; i += gridDim.x) {
        const uint32_t piece = (uint32_t)(i % pieces), layer = (uint32_t)(i / pieces % c.layers.n), at = (uint32_t)(i / pieces / c.layers.n);
        copy_page(c, layer, moved[at], holes[at], piece, pieces);
    }
}

__global__ __launch_bounds__(256) void compact_tables_kernel(PagesArgs p, const uint32_t* moved, const uint32_t* holes, const uint32_t* totals,
                                                             const uint32_t* numbers, uint32_t n_pages, uint32_t shift) {
    const uint64_t first = (uint64_t)blockIdx.x * 256 + threadIdx.x, step = (uint64_t)gridDim.x * 256;
    for (uint64_t i = first; i < totals[0]; i += step) {
        p.refs[holes[i]] = p.refs[moved[i]];
        p.refs[moved[i]] = 0;
    }
    for (uint64_t i = first; i < (uint64_t)p.n_seqs * p.table_pages; i += step) {
        const uint32_t b = (uint32_t)(i / p.table_pages), j = (uint32_t)(i % p.table_pages);
        if (j >= (uint32_t)(((uint64_t)min(p.lengths[b], CACHE_MOST) + (1u << shift) - 1) >> shift)) continue;
        const uint32_t page = p.tables[i];
        if (page < n_pages) p.tables[i] = numbers[page];
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

// Workgroups that share a page: each moves 16 KB of its codes.
uint32_t page_pieces(const CachePages& c) { return (uint32_t)divided_up((uint64_t)c.heads * c.page_tokens * c.dim, 8192); }

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
    advance_tables_kernel<<<dim3(entry_blocks(entries)), dim3(256), 0, stream>>>(a, w, c.n_pages, c.shift);
    advance_decide_kernel<<<dim3(1), dim3(1024), 0, stream>>>(a, w, c.n_pages, c.shift);
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
    with_layers(a.p, [&](const PageCopy& copy) {
        const uint64_t most = (uint64_t)(c.n_pages / 2) * copy.layers.n * pieces;    // as many pages move as there are holes
        if (most) compact_copy_kernel<<<dim3((uint32_t)std::min<uint64_t>(most, 2048)), dim3(256), 0, stream>>>(copy, moved, holes, totals, pieces);
    });
    const uint64_t entries = std::max<uint64_t>((uint64_t)a.p.n_seqs * a.p.table_pages, c.n_pages / 2);
    compact_tables_kernel<<<dim3(entry_blocks(entries)), dim3(256), 0, stream>>>(a.p, moved, holes, totals, a.numbers, c.n_pages, c.shift);
    return hipGetLastError();
}

}  // namespace dessert
