// New tokens into a paged int8 cache, and the pages that a token looks at.
//   append   a page's scale s' = max(s, max|x| * (1 / 127)) over its new tokens (s: what it had for earlier ones), new codes x / s',
//            earlier ones c s / s', each the nearest integer to the real quotient, ties to even; the keys' smallest and largest codes a
//            channel beside them.  Bound by memory: tokens read, codes written.
//   select   a page's score for a query head is the most that a key between its bounds can come to, sum_d (q_d < 0 ? q_d min_d : q_d max_d)
//            in whole numbers, times the scales; the pages of the n highest, largest over the heads that share them.
#include "cache_common.hpp"
#include "launch_slices.hpp"

namespace dessert {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// The nearest integer to num / den (num = c * over: exact in 64 bits), ties to even; factor = over / den in 32 bits is off by at most 2^-23 of
// itself, the product with it by less than 2^-15 altogether: only products that close to a half need the 64-bit quotient, which is a half exactly
// where the real one is (two products of 24-bit numbers that differ do so by more than its rounding).
__device__ inline int nearest(float x, double over, double den, float factor) {
    const float t = x * factor;
    if (factor < 0x1p125f && factor > 0x1p-125f) {
        const float n = rintf(t);
        if (fabsf(t - n) < 0.5f - 0x1p-14f) return (int)fminf(fmaxf(n, -127.f), 127.f);
    }
    const double q = (double)x * over / den;
    return (int)fmin(fmax(rint(q), -127.0), 127.0);
}

struct PageScale {
    float before, now;
    bool none;     // new codes are 0: no scale, or one that is no number
    bool again;    // earlier codes go to the new scale

    // peak: bits of the largest magnitude; infinities and NaN, of which a page keeps scale NaN, are above all others
    __device__ PageScale(float had, uint32_t peak) : before(had) {
        const float most = __uint_as_float(peak);
        now = most < __builtin_huge_valf() && had == had ? fmaxf(had, most * (1.f / 127.f)) : __builtin_nanf("");
        none = !(now > 0.f && now < __builtin_huge_valf());
        again = now > before;
    }
    __device__ int moved(int c, float ratio) const { return again ? nearest((float)c, before, now, ratio) : c; }
    // Codes of 8 numbers.  Sums with 1.5 * 2^23 are rounded to whole numbers, which their last bits hold; factor = 1 / now.
    __device__ uint64_t codes(const float (&x)[8], float factor) const {
        constexpr float MAGIC = 12582912.f;
        uint32_t n[8];
        float off = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float t = x[i] * factor, m = t + MAGIC;
            n[i] = __float_as_uint(m);
            off = fmaxf(off, fabsf(t - (m - MAGIC)));
        }
        if (!(off < 0.5f - 0x1p-14f && factor < 0x1p125f && factor > 0x1p-125f)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) n[i] = none ? 0u : (uint32_t)nearest(x[i], 1.0, now, factor);
        }
        const uint32_t lo = __builtin_amdgcn_perm(n[1], n[0], 0x0C0C0400) | __builtin_amdgcn_perm(n[3], n[2], 0x04000C0C);
        const uint32_t hi = __builtin_amdgcn_perm(n[5], n[4], 0x0C0C0400) | __builtin_amdgcn_perm(n[7], n[6], 0x04000C0C);
        return (uint64_t)hi << 32 | lo;
    }
};

template <typename T>
__device__ inline uint32_t magnitude(T x) {
    return __float_as_uint((float)x) & 0x7FFFFFFFu;
}

// A workgroup of W waves sees to the keys or the values of one head in one page.  A lane has 8 channels of 4 consecutive slots, the workgroup
// a round of R = 4 * (lanes / (dim / 8)) slots (a multiple of 16): a page that is one round is read once, a larger one a second time from the
// caches.  Values go through LDS, from a lane's 4 slots of a channel to the 16 that are written at once.
// Bound by memory: 19500 tokens x 8 heads x 128 bf16 (120 MB read and, in int8, written) in 39 to 41 us, 3.0 TB/s,
// vector ALU 44 % busy; with a thread for 16 slots
// of a channel and 256 threads a page it took 67.
template <typename T, int W>
__global__ __launch_bounds__(64 * W) void append_kernel(CachePages c, CacheBatch b, const T* __restrict__ k, uint64_t k_stride, const T* __restrict__ v,
                                                        uint64_t v_stride, uint32_t places, uint64_t first_unit) {
    __shared__ uint32_t peaks[W];
    __shared__ int least[CACHE_MAX_DIM], most[CACHE_MAX_DIM];
    __shared__ uint32_t tile[W * 512 + CACHE_MAX_DIM];
    uint64_t id = first_unit + blockIdx.x;
    const bool values = id & 1;
    id >>= 1;
    const uint32_t h = (uint32_t)(id % c.heads);
    id /= c.heads;
    const uint32_t place_of = (uint32_t)(id % places), s = (uint32_t)(id / places);
    const NewTokens n = new_tokens(b, s);
    if (n.begin + (int32_t)n.count <= 0 || n.count == 0) return;
    const int32_t begin = max(n.begin, 0), end = n.begin + (int32_t)n.count;
    const uint32_t P = c.page_tokens, D = c.dim, place = ((uint32_t)begin >> c.shift) + place_of;
    const int32_t lo = max(begin, (int32_t)(place << c.shift)), hi = min(end, (int32_t)((place + 1) << c.shift));
    if (place >= b.table_pages || lo >= hi) return;
    const uint32_t page = page_at(b, b.tables + (uint64_t)s * b.table_pages, place, c.n_pages);
    const uint64_t at = (uint64_t)(page == NO_PAGE ? 0u : page) * c.heads + h;
    const uint32_t slot0 = lo & (P - 1), slot1 = slot0 + (uint32_t)(hi - lo);      // the new slots
    const uint64_t stride = values ? v_stride : k_stride;
    const T* x = (values ? v : k) + (uint64_t)(n.first + (uint32_t)(lo - n.begin)) * stride + (uint64_t)h * D;

    const uint32_t per = D / 8, quads = 64 * W / per & ~3u, R = 4 * quads, base = slot0 & ~15u, rounds = (slot1 - base + R - 1) / R;
    const uint32_t d8 = threadIdx.x % per, quad = threadIdx.x / per;
    T e[4][8];
    // slots outside the new ones get a neighbour's numbers, which changes no maximum and is not written
    auto load = [&](uint32_t round) {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            const uint32_t slot = min(max(base + round * R + 4 * min(quad, quads - 1) + i, slot0), slot1 - 1);
            __builtin_memcpy(e[i], x + (uint64_t)(slot - slot0) * stride + d8 * 8, sizeof(e[i]));
        }
    };
    float* scales = values ? c.vs : c.ks;
    load(0);       // does not wait for the page's number
    const float had = slot0 ? scales[at] : 0.f;
    if (page == NO_PAGE) return;
    uint32_t peak = 0;
    for (uint32_t round = 0; round < rounds; ++round) {
        if (round) load(round);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) peak = max(peak, magnitude(e[i][j]));
    }
#pragma unroll
    for (int o = 1; o < 64; o *= 2) peak = max(peak, (uint32_t)__shfl_xor((int)peak, o));
    int8_t* bounds = c.bounds ? c.bounds + at * 2 * D : nullptr;
    if constexpr (W > 1) {
        if ((threadIdx.x & 63) == 0) peaks[threadIdx.x >> 6] = peak;
        barrier();
#pragma unroll
        for (int w = 0; w < W; ++w) peak = max(peak, peaks[w]);
    }
    const PageScale scale(had, peak);
    const float factor = 1.f / scale.now, ratio = had / scale.now;
    barrier();      // every thread has read the scale
    if (threadIdx.x == 0) scales[at] = scale.now;

    if (!values) {
        int8_t* codes = c.k + at * P * D;
        if (scale.again && slot0)
            for (uint32_t i = threadIdx.x; i < slot0 * per; i += 64 * W) {
                int8_t q[8];
                __builtin_memcpy(q, codes + i * 8, 8);
#pragma unroll
                for (int j = 0; j < 8; ++j) q[j] = (int8_t)scale.moved(q[j], ratio);
                __builtin_memcpy(codes + i * 8, q, 8);
            }
        if (bounds)
            for (uint32_t d = threadIdx.x; d < D; d += 64 * W) {
                least[d] = slot0 ? scale.moved(bounds[d], ratio) : 127;
                most[d] = slot0 ? scale.moved(bounds[D + d], ratio) : -127;
            }
        int low[8], high[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            low[j] = 127;
            high[j] = -127;
        }
        for (uint32_t round = 0; round < rounds; ++round) {
            if (rounds > 1) load(round);
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) {
                const uint32_t slot = base + round * R + 4 * quad + i;
                float y[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] = (float)e[i][j];
                const uint64_t q = scale.codes(y, factor);
                if (quad < quads && slot >= slot0 && slot < slot1) {
                    __builtin_memcpy(codes + (uint64_t)slot * D + d8 * 8, &q, 8);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int z = (int8_t)(q >> 8 * j);
                        low[j] = min(low[j], z);
                        high[j] = max(high[j], z);
                    }
                }
            }
        }
        if (bounds) {
            barrier();
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                atomicMin(&least[d8 * 8 + j], low[j]);
                atomicMax(&most[d8 * 8 + j], high[j]);
            }
            barrier();
            for (uint32_t d = threadIdx.x; d < D; d += 64 * W) {
                bounds[d] = (int8_t)least[d];
                bounds[D + d] = (int8_t)most[d];
            }
        }
        return;
    }
    int8_t* codes = c.v + at * P * D;
    if (scale.again)      // whole groups of 16 in front of the first new slot's
        for (uint32_t i = threadIdx.x; i < base / 16 * D; i += 64 * W) {
            int8_t* to = codes + (uint64_t)(i / (base / 16)) * P + i % (base / 16) * 16;
            int8_t q[16];
            __builtin_memcpy(q, to, 16);
#pragma unroll
            for (int j = 0; j < 16; ++j) q[j] = (int8_t)scale.moved(q[j], ratio);
            __builtin_memcpy(to, q, 16);
        }
    const uint32_t row = R / 4 + 1;       // words of a channel's slots in LDS, one more than they fill: rows begin at other banks
    for (uint32_t round = 0; round < rounds; ++round) {
        if (rounds > 1) load(round);
        uint64_t q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = (float)e[i][j];
            q[i] = scale.codes(y, factor);
        }
        if (quad < quads)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                tile[(d8 * 8 + j) * row + quad] = (uint32_t)(q[0] >> 8 * j & 255) | (uint32_t)(q[1] >> 8 * j & 255) << 8 |
                                                  (uint32_t)(q[2] >> 8 * j & 255) << 16 | (uint32_t)(q[3] >> 8 * j & 255) << 24;
        barrier();
        const uint32_t groups = R / 16;
        for (uint32_t i = threadIdx.x; i < D * groups; i += 64 * W) {
            const uint32_t d = i / groups, g = i % groups, slot = base + round * R + g * 16;
            if (slot >= slot1) continue;
            u32x4 z = {tile[d * row + g * 4], tile[d * row + g * 4 + 1], tile[d * row + g * 4 + 2], tile[d * row + g * 4 + 3]};
            int8_t* to = codes + (uint64_t)d * P + slot;
            if (slot < slot0 || slot + 16 > slot1) {
                int8_t fresh[16], old[16];
                __builtin_memcpy(fresh, &z, 16);
                __builtin_memcpy(old, to, 16);
#pragma unroll
                for (int j = 0; j < 16; ++j) old[j] = slot + j < slot0 ? (int8_t)scale.moved(old[j], ratio) : slot + j < slot1 ? fresh[j] : old[j];
                __builtin_memcpy(&z, old, 16);
            }
            __builtin_memcpy(to, &z, 16);
        }
        barrier();
    }
}

// ---- pages by their bounds ----------------------------------------------------------------------------------------------------
// Scores as numbers that order the same; NaN as high as +inf, -0 as +0.  0: no page.
__device__ inline uint32_t ordered(float x) {
    if (!(x == x)) x = __builtin_huge_valf();
    const uint32_t u = x == 0.f ? 0u : __float_as_uint(x);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
constexpr uint32_t KEY_ALWAYS = 0xFFFFFFFFu;

__device__ inline bool select_row(const SelectArgs& a, uint32_t index, uint32_t& row, int32_t& pos, uint32_t& seq) {
    seq = index / a.batch.max_tokens;
    const uint32_t t = index % a.batch.max_tokens;
    const NewTokens n = new_tokens(a.batch, seq);
    row = n.first + t;
    pos = n.begin + (int32_t)t;
    return t < n.count;
}

// What a wave needs of a row to score pages: the negative and the positive parts of the codes of 16 query heads, as the right operand of
// products whose left one is pages' bounds (min and max side by side are a row of 2 dim numbers).
template <int ND>
__device__ inline void load_parts(const int8_t* q, uint32_t g, v4i (&parts)[ND]) {
    constexpr int D = ND * 32;
#pragma unroll
    for (int f = 0; f < ND; ++f) {
        const uint32_t at = 64 * f + 16 * g;
        const bool low = at < D;
        v4i e;
        __builtin_memcpy(&e, q + (low ? at : at - D), 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int sign = (int)(((uint32_t)e[j] >> 7 & 0x01010101u) * 255u);
            e[j] &= low ? sign : ~sign;
        }
        parts[f] = e;
    }
}

// Scores of the 64 places from `from` on (up to `last`), by a wave: all their bounds are on the way at once (2048 pages of 8 heads 6.6 us; 16 at a
// time 18).
template <int ND>
__device__ inline void score_places(const SelectArgs& a, const uint32_t* table, uint32_t row, uint32_t h, uint32_t from, uint32_t last, uint32_t* keys) {
    constexpr int D = ND * 32;
    const uint32_t lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const uint32_t own = page_at(a.batch, table, from + lane, a.cache.n_pages);
    const uint64_t q_row0 = (uint64_t)row * a.cache.heads * a.group + (uint64_t)h * a.group;
    v4i parts[ND];
    uint64_t q_row = q_row0 + min(r, a.group - 1);
    load_parts<ND>(a.q + q_row * D, g, parts);
    float sq = a.q_scales[q_row];
    v4i bounds[4][ND];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        const uint32_t page = (uint32_t)__shfl((int)own, 16 * s + r);
        const int8_t* at = a.cache.bounds + ((uint64_t)(page == NO_PAGE ? 0u : page) * a.cache.heads + h) * 2 * D + 16 * g;
#pragma unroll
        for (int f = 0; f < ND; ++f) bounds[s][f] = *(const v4i*)(at + 64 * f);
    }
    const float own_ks = a.cache.ks[(uint64_t)(own == NO_PAGE ? 0u : own) * a.cache.heads + h];
    float best[4][4];
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i) best[s][i] = -__builtin_huge_valf();
    for (uint32_t g0 = 0; g0 < a.group; g0 += 16) {
        if (g0) {
            q_row = q_row0 + min(g0 + r, a.group - 1);
            load_parts<ND>(a.q + q_row * D, g, parts);
            sq = a.q_scales[q_row];
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            v4i sum = {};
#pragma unroll
            for (int f = 0; f < ND; ++f) sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(bounds[s][f], parts[f], sum, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float x = (float)sum[i] * (sq * __shfl(own_ks, 16 * s + 4 * g + i));
                if (!(x == x)) x = __builtin_huge_valf();
                best[s][i] = fmaxf(best[s][i], x);
            }
        }
    }
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        float mine = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int o = 1; o < 16; o *= 2) best[s][i] = fmaxf(best[s][i], __shfl_xor(best[s][i], o));
            if ((r & 3) == (uint32_t)i) mine = best[s][i];
        }
        // the score of place 16 s + 4 g + r % 4
        const uint32_t at = 16 * s + 4 * g + (r & 3), j = from + at;
        const bool there = (uint32_t)__shfl((int)own, at) != NO_PAGE, always = j < a.n_first || j + a.n_last > last;
        if (r < 4 && j <= last) keys[j] = !there ? 0u : always ? KEY_ALWAYS : ordered(mine);
    }
}

// Sum over a workgroup of W waves: of the threads in front, and of all.
template <int W>
__device__ inline uint32_t sum_before(uint32_t x, uint32_t* parts, uint32_t& total) {
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
    for (uint32_t w = 0; w < W; ++w) {
        if (w < wave) before += parts[w];
        total += parts[w];
    }
    return before + y - x;
}

// The n_select highest of up to 64 W EACH keys, ties to the lower place, written in the order of places.  A thread holds EACH consecutive
// ones; the key of the last one is found bit by bit, by counting the keys that are not below it, from the highest bit in which the keys
// differ (those aside that are always taken) until just n_select are left.  64 of 2048 keys 7.1 us, 48 of 512 5.0 (12 by histograms of 8 bits, whose counts
// fall on few addresses).
template <int W, int EACH>
__device__ inline void pick(const uint32_t* keys, uint32_t n, uint32_t n_select, uint32_t* out, uint32_t* parts) {
    uint32_t key[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const uint32_t at = threadIdx.x * EACH + i;
        key[i] = at < n ? keys[at] : 0u;
    }
    uint32_t border = 0, ties = 0;      // keys above the border are taken, and the first `ties` at it (0 is no page)
    if (n > n_select) {
        uint32_t lo = 0xFFFFFFFFu, hi = 0, there = 0;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            if (key[i] != 0 && key[i] != KEY_ALWAYS) {
                lo = min(lo, key[i]);
                hi = max(hi, key[i]);
            }
            there += key[i] != 0;
        }
#pragma unroll
        for (int o = 1; o < 64; o *= 2) {
            lo = min(lo, (uint32_t)__shfl_xor((int)lo, o));
            hi = max(hi, (uint32_t)__shfl_xor((int)hi, o));
            there += (uint32_t)__shfl_xor((int)there, o);
        }
        if ((threadIdx.x & 63) == 0) {
            parts[threadIdx.x >> 6] = lo;
            parts[W + (threadIdx.x >> 6)] = hi;
            parts[2 * W + (threadIdx.x >> 6)] = there;
        }
        barrier();
        there = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            lo = min(lo, parts[w]);
            hi = max(hi, parts[W + w]);
            there += parts[2 * W + w];
        }
        barrier();
        if (there > n_select && hi) {
            const uint32_t differ = lo ^ hi;
            int bit = differ ? 31 - __clz((int)differ) : -1;
            border = bit < 0 ? hi : bit == 31 ? 0u : hi >> (bit + 1) << (bit + 1);
            for (bool exact = false; bit >= 0 && !exact; --bit) {
                const uint32_t trial = border | 1u << bit;
                uint32_t count = 0;
#pragma unroll
                for (int i = 0; i < EACH; ++i) count += (uint32_t)__popcll(__ballot(key[i] >= trial));
                uint32_t* slot = parts + (bit & 1) * W;      // by turns: one barrier a bit
                if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = count;
                barrier();
                count = 0;
#pragma unroll
                for (int w = 0; w < W; ++w) count += slot[w];
                if (count >= n_select) border = trial;
                exact = count == n_select;
            }
        }
        uint32_t above = 0, all;
#pragma unroll
        for (int i = 0; i < EACH; ++i) above += key[i] > border;
        (void)sum_before<W>(above, parts, all);
        ties = border ? n_select - all : 0u;
    }
    uint32_t above = 0, at = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        above += key[i] > border;
        at += key[i] == border;
    }
    uint32_t all_above, all_at;
    const uint32_t above_before = sum_before<W>(above, parts, all_above);
    uint32_t tie = sum_before<W>(at, parts, all_at), place = above_before + min(tie, ties);
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const bool tied = key[i] == border;
        if (key[i] > border || (tied && tie < ties)) out[place++] = threadIdx.x * EACH + i;
        tie += tied;
    }
    for (uint32_t i = all_above + min(all_at, ties) + threadIdx.x; i < n_select; i += 64 * W) out[i] = NO_PAGE;
}

// Places of a row that there are, up to its token's own.
__device__ inline uint32_t row_places(const SelectArgs& a, int32_t pos) {
    return pos < 0 ? 0u : min(((uint32_t)pos >> a.cache.shift) + 1, a.batch.table_pages);
}

// A wave for 64 pages.  (Scored and picked by one workgroup a row instead: 43 us for 29 with 2048 pages of 8 rows, chosen and attended to, 49 for 40
// with 1024 of 16 rows at dim 256, the same for 512 of 128 rows.)
template <int ND>
__global__ __launch_bounds__(256) void select_score_kernel(SelectArgs a, uint32_t blocks) {
    uint32_t id = blockIdx.x;
    const uint32_t from = id % blocks * 256 + (threadIdx.x >> 6) * 64;
    id /= blocks;
    const uint32_t h = id % a.cache.heads;
    uint32_t row, seq;
    int32_t pos;
    if (!select_row(a, id / a.cache.heads, row, pos, seq)) return;
    const uint32_t n = row_places(a, pos);
    if (from >= n) return;
    score_places<ND>(a, a.batch.tables + (uint64_t)seq * a.batch.table_pages, row, h, from, n - 1,
                     a.keys + ((uint64_t)row * a.cache.heads + h) * a.batch.table_pages);
}

template <int W, int EACH>
__global__ __launch_bounds__(64 * W) void select_pick_kernel(SelectArgs a) {
    __shared__ uint32_t parts[3 * W];
    const uint32_t h = blockIdx.x % a.cache.heads;
    uint32_t row, seq;
    int32_t pos;
    if (!select_row(a, blockIdx.x / a.cache.heads, row, pos, seq)) return;
    const uint64_t at = (uint64_t)row * a.cache.heads + h;
    pick<W, EACH>(a.keys + at * a.batch.table_pages, row_places(a, pos), a.n_select, a.out + at * a.n_select, parts);
}

// More pages than a workgroup's registers hold: the border by four passes of 8 bits, then one pass over consecutive runs of places a thread.
__global__ __launch_bounds__(1024) void select_pages_kernel(SelectArgs a) {
    __shared__ uint32_t counts[256], parts[16], found[2];
    const uint32_t h = blockIdx.x % a.cache.heads;
    uint32_t row, seq;
    int32_t pos;
    if (!select_row(a, blockIdx.x / a.cache.heads, row, pos, seq)) return;
    const uint32_t n = row_places(a, pos);
    const uint32_t* keys = a.keys + ((uint64_t)row * a.cache.heads + h) * a.batch.table_pages;
    uint32_t* out = a.out + ((uint64_t)row * a.cache.heads + h) * a.n_select;
    uint32_t border = 0, ties = 0;
    if (n > a.n_select) {
        uint32_t want = a.n_select, mask = 0;
        for (int shift = 24; shift >= 0; shift -= 8) {
            if (threadIdx.x < 256) counts[threadIdx.x] = 0;
            barrier();
            for (uint32_t i = threadIdx.x; i < n; i += 1024) {
                const uint32_t key = keys[i];
                if ((key & mask) == border) atomicAdd(&counts[key >> shift & 255], 1u);
            }
            barrier();
            // digits from the highest: thread i sees to digit 255 - i
            const uint32_t here = threadIdx.x < 256 ? counts[255 - threadIdx.x] : 0u;
            uint32_t total;
            const uint32_t before = sum_before<16>(here, parts, total);
            if (before < want && want <= before + here) {
                found[0] = 255 - threadIdx.x;
                found[1] = want - before;
            }
            barrier();
            border |= found[0] << shift;
            want = found[1];
            mask |= 255u << shift;
            barrier();
        }
        ties = border ? want : 0u;
    }
    const uint32_t each = (n + 1023) / 1024, from = min(threadIdx.x * each, n), to = min(from + each, n);
    uint32_t above = 0, at = 0;
    for (uint32_t i = from; i < to; ++i) {
        const uint32_t key = keys[i];
        above += key > border;
        at += key == border;
    }
    uint32_t all_above, all_at;
    const uint32_t above_before = sum_before<16>(above, parts, all_above);
    uint32_t tie = sum_before<16>(at, parts, all_at), place = above_before + min(tie, ties);
    for (uint32_t i = from; i < to; ++i) {
        const uint32_t key = keys[i];
        const bool tied = key == border;
        if (key > border || (tied && tie < ties)) out[place++] = i;
        tie += tied;
    }
    for (uint32_t i = all_above + min(all_at, ties) + threadIdx.x; i < a.n_select; i += 1024) out[i] = NO_PAGE;
}

template <int ND>
void launch_select(const SelectArgs& a, hipStream_t stream) {
    const uint32_t rows = a.batch.n_seqs * a.batch.max_tokens * a.cache.heads, pages = a.batch.table_pages;
    const uint32_t blocks = (pages + 255) / 256;
    select_score_kernel<ND><<<dim3(rows * blocks), dim3(256), 0, stream>>>(a, blocks);
    if (pages <= 512) select_pick_kernel<4, 2><<<dim3(rows), dim3(256), 0, stream>>>(a);
    else if (pages <= 2048) select_pick_kernel<4, 8><<<dim3(rows), dim3(256), 0, stream>>>(a);
    else if (pages <= 16384) select_pick_kernel<16, 16><<<dim3(rows), dim3(1024), 0, stream>>>(a);
    else select_pages_kernel<<<dim3(rows), dim3(1024), 0, stream>>>(a);
}

template <typename T>
void launch_append(const CachePages& c, const CacheBatch& b, const T* k, uint64_t k_stride, const T* v, uint64_t v_stride, hipStream_t stream) {
    const uint32_t places = (uint32_t)append_places(b.max_tokens, c.page_tokens);
    // waves: as many as see to the new slots of a page in one round, four at most; enough for rounds of 16 slots
    const uint32_t per = c.dim / 8, slots = std::min<uint64_t>(c.page_tokens, std::max<uint64_t>(16, (uint64_t)b.max_tokens + 15));
    uint32_t waves = 1;
    while (waves < 4 && 4 * (64 * waves / per & ~3u) < std::max(16u, slots)) waves *= 2;
    const uint64_t units = (uint64_t)b.n_seqs * places * c.heads * 2;
    in_launches(units, 1, 256, [&](uint64_t first, uint64_t, uint32_t workgroups) {
        const dim3 grid(workgroups);
        if (waves == 1) append_kernel<T, 1><<<grid, dim3(64), 0, stream>>>(c, b, k, k_stride, v, v_stride, places, first);
        else if (waves == 2) append_kernel<T, 2><<<grid, dim3(128), 0, stream>>>(c, b, k, k_stride, v, v_stride, places, first);
        else append_kernel<T, 4><<<grid, dim3(256), 0, stream>>>(c, b, k, k_stride, v, v_stride, places, first);
    });
}

}  // namespace

hipError_t launch_cache_append(const CachePages& c, const CacheBatch& b, const void* k, uint64_t k_stride, const void* v, uint64_t v_stride,
                               uint32_t dtype, hipStream_t stream) {
    if (dtype == TYPE_F16) launch_append<f16_t>(c, b, (const f16_t*)k, k_stride, (const f16_t*)v, v_stride, stream);
    else if (dtype == TYPE_BF16) launch_append<bf16_t>(c, b, (const bf16_t*)k, k_stride, (const bf16_t*)v, v_stride, stream);
    else launch_append<float>(c, b, (const float*)k, k_stride, (const float*)v, v_stride, stream);
    return hipGetLastError();
}

hipError_t launch_cache_select(const SelectArgs& a, hipStream_t stream) {
    switch (a.cache.dim / 32) {
        case 1: launch_select<1>(a, stream); break;
        case 2: launch_select<2>(a, stream); break;
        case 3: launch_select<3>(a, stream); break;
        case 4: launch_select<4>(a, stream); break;
        case 5: launch_select<5>(a, stream); break;
        case 6: launch_select<6>(a, stream); break;
        case 7: launch_select<7>(a, stream); break;
        default: launch_select<8>(a, stream); break;
    }
    return hipGetLastError();
}

}  // namespace dessert
