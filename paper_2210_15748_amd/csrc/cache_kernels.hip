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
    __device__ int code(float x, float factor) const { return none ? 0 : nearest(x, 1.0, now, factor); }
    __device__ int moved(int c, float factor) const { return again ? nearest((float)c, before, now, factor) : c; }
};

template <typename T>
__device__ inline uint32_t magnitude(T x) {
    return __float_as_uint((float)x) & 0x7FFFFFFFu;
}

// A workgroup sees to the keys or the values of one head in one page: the page's new tokens are read twice, for the scale and for the
// codes (the second time from the caches).
template <typename T>
__global__ __launch_bounds__(256) void append_kernel(CachePages c, CacheBatch b, const T* __restrict__ k, uint64_t k_stride, const T* __restrict__ v,
                                                     uint64_t v_stride, uint32_t places, uint64_t first) {
    __shared__ uint32_t peaks[4];
    __shared__ int least[CACHE_MAX_DIM], most[CACHE_MAX_DIM];
    uint64_t id = first + blockIdx.x;
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
    if (page == NO_PAGE) return;
    const uint64_t at = (uint64_t)page * c.heads + h;
    const uint32_t tokens = hi - lo, slot0 = lo & (P - 1);
    const uint64_t stride = values ? v_stride : k_stride;
    const T* x = (values ? v : k) + (uint64_t)(n.first + (uint32_t)(lo - n.begin)) * stride + (uint64_t)h * D;

    const uint32_t per = D / 8, runs = tokens * per;
    uint32_t peak = 0;
    for (uint32_t i = threadIdx.x; i < runs; i += 256) {
        T e[8];
        __builtin_memcpy(e, x + (uint64_t)(i / per) * stride + i % per * 8, sizeof(e));
#pragma unroll
        for (int j = 0; j < 8; ++j) peak = max(peak, magnitude(e[j]));
    }
#pragma unroll
    for (int o = 1; o < 64; o *= 2) peak = max(peak, (uint32_t)__shfl_xor((int)peak, o));
    if ((threadIdx.x & 63) == 0) peaks[threadIdx.x >> 6] = peak;
    float* scales = values ? c.vs : c.ks;
    const float had = slot0 ? scales[at] : 0.f;
    int8_t* bounds = c.bounds ? c.bounds + at * 2 * D : nullptr;
    __syncthreads();
    peak = max(max(peaks[0], peaks[1]), max(peaks[2], peaks[3]));
    const PageScale scale(had, peak);
    const float factor = 1.f / scale.now, ratio = had / scale.now;
    if (threadIdx.x == 0) scales[at] = scale.now;      // every thread has read it: it is behind the barrier

    if (!values) {
        int8_t* codes = c.k + at * P * D;
        if (scale.again && slot0)
            for (uint32_t i = threadIdx.x; i < slot0 * D / 8; i += 256) {
                int8_t e[8];
                __builtin_memcpy(e, codes + i * 8, 8);
#pragma unroll
                for (int j = 0; j < 8; ++j) e[j] = (int8_t)scale.moved(e[j], ratio);
                __builtin_memcpy(codes + i * 8, e, 8);
            }
        if (bounds) {
            for (uint32_t d = threadIdx.x; d < D; d += 256) {
                least[d] = slot0 ? scale.moved(bounds[d], ratio) : 127;
                most[d] = slot0 ? scale.moved(bounds[D + d], ratio) : -127;
            }
            __syncthreads();
        }
        for (uint32_t i = threadIdx.x; i < runs; i += 256) {
            const uint32_t t = i / per, d = i % per * 8;
            T e[8];
            __builtin_memcpy(e, x + (uint64_t)t * stride + d, sizeof(e));
            int8_t q[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                q[j] = (int8_t)scale.code((float)e[j], factor);
                if (bounds) {
                    atomicMin(&least[d + j], (int)q[j]);
                    atomicMax(&most[d + j], (int)q[j]);
                }
            }
            __builtin_memcpy(codes + (uint64_t)(slot0 + t) * D + d, q, 8);
        }
        if (bounds) {
            __syncthreads();
            for (uint32_t d = threadIdx.x; d < D; d += 256) {
                bounds[d] = (int8_t)least[d];
                bounds[D + d] = (int8_t)most[d];
            }
        }
        return;
    }
    // values: 16 tokens of a channel at a time, which lie side by side
    int8_t* codes = c.v + at * P * D;
    const uint32_t g0 = scale.again ? 0 : slot0 / 16, g1 = (slot0 + tokens + 15) / 16;
    for (uint32_t i = threadIdx.x; i < (g1 - g0) * D; i += 256) {
        const uint32_t g = g0 + i / D, d = i % D;
        int8_t* to = codes + (uint64_t)d * P + g * 16;
        int8_t q[16];
        if (g * 16 < slot0 || g * 16 + 16 > slot0 + tokens) __builtin_memcpy(q, to, 16);
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const uint32_t slot = g * 16 + j;
            if (slot >= slot0 && slot < slot0 + tokens) q[j] = (int8_t)scale.code((float)x[(uint64_t)(slot - slot0) * stride + d], factor);
            else if (slot < slot0) q[j] = (int8_t)scale.moved(q[j], ratio);
        }
        __builtin_memcpy(to, q, 16);
    }
}

// ---- pages by their bounds ----------------------------------------------------------------------------------------------------
// Scores as numbers that order the same; NaN as high as +inf.  0: no page.
__device__ inline uint32_t ordered(float x) {
    if (!(x == x)) x = __builtin_huge_valf();
    const uint32_t u = __float_as_uint(x);
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

// Scores of 64 pages a wave, 16 at a time: bounds (min and max side by side are a row of 2 dim numbers) times the negative and positive
// parts of the codes, on the matrix cores.
template <int ND>
__global__ __launch_bounds__(256) void select_score_kernel(SelectArgs a, uint32_t blocks) {
    constexpr int D = ND * 32;
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
    uint32_t id = blockIdx.x;
    const uint32_t block = id % blocks;
    id /= blocks;
    const uint32_t h = id % a.cache.heads;
    uint32_t row, seq;
    int32_t pos;
    if (!select_row(a, id / a.cache.heads, row, pos, seq) || pos < 0) return;
    const uint32_t last = min((uint32_t)pos >> a.cache.shift, a.batch.table_pages - 1);
    const uint32_t* table = a.batch.tables + (uint64_t)seq * a.batch.table_pages;
    uint32_t* keys = a.keys + ((uint64_t)row * a.cache.heads + h) * a.batch.table_pages;
    const uint32_t from = block * 256 + wave * 64;
    for (uint32_t p0 = from; p0 < from + 64 && p0 <= last; p0 += 16) {
        const uint32_t mine = page_at(a.batch, table, p0 + r, a.cache.n_pages);
        const int8_t* bounds = a.cache.bounds + ((uint64_t)(mine == NO_PAGE ? 0u : mine) * a.cache.heads + h) * 2 * D + 16 * g;
        v4i bv[ND];
#pragma unroll
        for (int f = 0; f < ND; ++f) bv[f] = *(const v4i*)(bounds + 64 * f);
        float best[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) best[i] = -__builtin_huge_valf();
        bool nan[4] = {};
        float ks[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t page = page_at(a.batch, table, p0 + 4 * g + i, a.cache.n_pages);
            ks[i] = a.cache.ks[(uint64_t)(page == NO_PAGE ? 0u : page) * a.cache.heads + h];
        }
        for (uint32_t g0 = 0; g0 < a.group; g0 += 16) {
            const uint64_t q_row = (uint64_t)row * a.cache.heads * a.group + (uint64_t)h * a.group + min(g0 + r, a.group - 1);
            const int8_t* q = a.q + q_row * D;
            v4i sum = {};
#pragma unroll
            for (int f = 0; f < ND; ++f) {
                // place 64 f + 16 g of the row of 2 dim: the first half goes with the negative parts
                const uint32_t at = 64 * f + 16 * g;
                const bool low = at < D;
                int8_t e[16];
                __builtin_memcpy(e, q + (low ? at : at - D), 16);
#pragma unroll
                for (int j = 0; j < 16; ++j) e[j] = low ? min(e[j], (int8_t)0) : max(e[j], (int8_t)0);
                sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(bv[f], __builtin_bit_cast(v4i, e), sum, 0, 0, 0);
            }
            const float sq = a.q_scales[q_row];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float x = (float)sum[i] * (sq * ks[i]);
                nan[i] = nan[i] || !(x == x);
                best[i] = fmaxf(best[i], x);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (nan[i]) best[i] = __builtin_huge_valf();
#pragma unroll
            for (int o = 1; o < 16; o *= 2) best[i] = fmaxf(best[i], __shfl_xor(best[i], o));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t j = p0 + 4 * g + i;
            if (r == (uint32_t)i && j <= last) {
                const bool there = page_at(a.batch, table, j, a.cache.n_pages) != NO_PAGE;
                const bool always = j < a.n_first || j + a.n_last > last;
                keys[j] = !there ? 0u : always ? KEY_ALWAYS : ordered(best[i]);
            }
        }
    }
}

// Sum over the workgroup's threads in front of this one, and of all of them.
__device__ inline uint32_t sum_before(uint32_t x, uint32_t* parts, uint32_t& total) {
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
    for (uint32_t w = 0; w < blockDim.x / 64; ++w) {
        if (w < wave) before += parts[w];
        total += parts[w];
    }
    return before + y - x;
}

// The n_select highest keys of a row, ties to the lower place, in the order of places: the key of the last one by four passes of 8 bits,
// then one pass over consecutive runs of places a thread.
__global__ __launch_bounds__(256) void select_pages_kernel(SelectArgs a) {
    __shared__ uint32_t counts[256], parts[4], found[2];
    const uint32_t index = blockIdx.x, h = index % a.cache.heads;
    uint32_t row, seq;
    int32_t pos;
    if (!select_row(a, index / a.cache.heads, row, pos, seq)) return;
    const uint32_t n = pos < 0 ? 0u : min(((uint32_t)pos >> a.cache.shift) + 1, a.batch.table_pages);
    const uint32_t* keys = a.keys + ((uint64_t)row * a.cache.heads + h) * a.batch.table_pages;
    uint32_t* out = a.out + ((uint64_t)row * a.cache.heads + h) * a.n_select;
    uint32_t border = 0, ties = 0xFFFFFFFFu;     // keys above the border are taken, and the first `ties` at it
    if (n > a.n_select) {
        uint32_t want = a.n_select, mask = 0;
        for (int shift = 24; shift >= 0; shift -= 8) {
            counts[threadIdx.x] = 0;
            __syncthreads();
            for (uint32_t i = threadIdx.x; i < n; i += 256) {
                const uint32_t key = keys[i];
                if ((key & mask) == border) atomicAdd(&counts[key >> shift & 255], 1u);
            }
            __syncthreads();
            // digits from the highest: thread i sees to digit 255 - i
            const uint32_t here = counts[255 - threadIdx.x];
            uint32_t total;
            const uint32_t before = sum_before(here, parts, total);
            if (before < want && want <= before + here) {
                found[0] = 255 - threadIdx.x;
                found[1] = want - before;
            }
            __syncthreads();
            border |= found[0] << shift;
            want = found[1];
            mask |= 255u << shift;
            __syncthreads();
        }
        ties = want;
    }
    const uint32_t each = (n + 255) / 256, from = min(threadIdx.x * each, n), to = min(from + each, n);
    uint32_t above = 0, at = 0;
    for (uint32_t i = from; i < to; ++i) {
        const uint32_t key = keys[i];
        above += key > border;
        at += key == border && key != 0;
    }
    uint32_t all_above, all_at;
    const uint32_t above_before = sum_before(above, parts, all_above), at_before = sum_before(at, parts, all_at);
    uint32_t tie = at_before, place = above_before + min(at_before, ties);
    for (uint32_t i = from; i < to; ++i) {
        const uint32_t key = keys[i];
        const bool tied = key == border && key != 0;
        if (key > border || (tied && tie < ties)) out[place++] = i;
        tie += tied;
    }
    for (uint32_t i = all_above + min(all_at, ties) + threadIdx.x; i < a.n_select; i += 256) out[i] = NO_PAGE;
}

template <typename T>
void launch_append(const CachePages& c, const CacheBatch& b, const void* k, uint64_t k_stride, const void* v, uint64_t v_stride, hipStream_t stream) {
    const uint32_t places = (uint32_t)append_places(b.max_tokens, c.page_tokens);
    in_launches((uint64_t)b.n_seqs * places * c.heads * 2, 1, 256, [&](uint64_t first, uint64_t, uint32_t workgroups) {
        append_kernel<T><<<dim3(workgroups), dim3(256), 0, stream>>>(c, b, (const T*)k, k_stride, (const T*)v, v_stride, places, first);
    });
}

}  // namespace

hipError_t launch_cache_append(const CachePages& c, const CacheBatch& b, const void* k, uint64_t k_stride, const void* v, uint64_t v_stride,
                               uint32_t dtype, hipStream_t stream) {
    if (dtype == TYPE_F16) launch_append<f16_t>(c, b, k, k_stride, v, v_stride, stream);
    else if (dtype == TYPE_BF16) launch_append<bf16_t>(c, b, k, k_stride, v, v_stride, stream);
    else launch_append<float>(c, b, k, k_stride, v, v_stride, stream);
    return hipGetLastError();
}

hipError_t launch_cache_select(const SelectArgs& a, hipStream_t stream) {
    const uint32_t rows = a.batch.n_seqs * a.batch.max_tokens * a.cache.heads, blocks = (a.batch.table_pages + 255) / 256;
    const dim3 grid(rows * blocks);
    switch (a.cache.dim / 32) {
        case 1: select_score_kernel<1><<<grid, dim3(256), 0, stream>>>(a, blocks); break;
        case 2: select_score_kernel<2><<<grid, dim3(256), 0, stream>>>(a, blocks); break;
        case 3: select_score_kernel<3><<<grid, dim3(256), 0, stream>>>(a, blocks); break;
        case 4: select_score_kernel<4><<<grid, dim3(256), 0, stream>>>(a, blocks); break;
        case 5: select_score_kernel<5><<<grid, dim3(256), 0, stream>>>(a, blocks); break;
        case 6: select_score_kernel<6><<<grid, dim3(256), 0, stream>>>(a, blocks); break;
        case 7: select_score_kernel<7><<<grid, dim3(256), 0, stream>>>(a, blocks); break;
        default: select_score_kernel<8><<<grid, dim3(256), 0, stream>>>(a, blocks); break;
    }
    select_pages_kernel<<<dim3(rows), dim3(256), 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace dessert
