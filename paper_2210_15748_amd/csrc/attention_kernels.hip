// Attention of new tokens over a paged int8 cache: for the rows of a key head (its query heads, the new tokens)
//   s_j = scale * k_scale(page of j) * q . k_j     over the visible j: not behind the row's position, inside the window, on a page
//   out = sum_j e^(s_j - m) v_scale(page of j) v_j / sum_j e^(s_j - m),   lse = m + log sum_j e^(s_j - m),   m = max_j s_j
// in one pass over the keys with a running m.  All products go to the matrix cores in fp16, which holds codes exactly; queries of bf16 are
// first scaled by a power of two a row, which makes their 8 bits exact in fp16 (but for parts below 2^-37 of the row's largest).
// e^s v_scale is rounded to fp16 (off by at most 2^-11 of itself: the rounding of an fp16 result), 2^12 being the largest of a row so far, which
// keeps all down to 2^-26 of the largest a normal number however far apart the scales of pages are and of whatever size; sums, maxima and
// the outputs, means from the first division on, are held in 32 bits.  Below, exponents are in powers of two: m the largest s log2(e), top
// the largest s log2(e) + log2(v_scale).
// Scores are formed as K Q^T: a lane then holds consecutive tokens of one row, and these are what it has to give as its part of P for
// O^T = V^T P^T, so P goes from one product to the next in registers.
#include "cache_common.hpp"

namespace dessert {

namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;
constexpr float NEVER = -__builtin_huge_valf();
// What products (at most 2^31) are multiplied by is at least this, which changes no score by more than 2^-29: -inf, where a key is not seen, stays that.
constexpr float LEAST_SCALE = 0x1p-60f;
constexpr float P_TOP = 12.f;      // the largest of P so far is 2^12,
constexpr float SLACK = 3.f;       // or of many rows up to 2^15

__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// In a branch: keeps the compiler from working it out for all and choosing afterwards.
__device__ inline void rarely() { asm volatile("; seldom"); }

// log2 of a scale, a subnormal one too (v_log_f32 takes those for 0).
__device__ inline float log2_scale(float x) { return __builtin_amdgcn_logf(__builtin_amdgcn_frexp_mantf(x)) + (float)__builtin_amdgcn_frexp_expf(x); }

// A value scale by its logarithm: m - top is about -log2(v_scale), and what is raised to it alone would leave the range of a float with scales that do
// not.  (A logarithm that is rounded to 2^-17 at most is right to that part of P, which goes on with 2^-11.)
__device__ inline float or_zero(float x) { return x == NEVER ? 0.f : x; }
// log2 of what a scale makes of a largest s log2(e); scales that are no numbers raise nothing.
__device__ inline float raised(float peak, float log2_vs) { return log2_vs < __builtin_huge_valf() ? peak + log2_vs : NEVER; }
// What e^(s - m) is multiplied by to be a part of P.
__device__ inline float p_factor(float log2_vs, float m, float top) { return exp2_fast(log2_vs + (or_zero(m) - or_zero(top) + P_TOP)); }
// What is added to s log2(e) for P's exponent, without that factor, which may be too large for a float where e^(s - m) is too small for one.
__device__ inline float p_shift(float log2_vs, float top) { return log2_vs + (P_TOP - or_zero(top)); }
// With factors below this P comes of products with e^(s - m): where that is below the normal numbers, they are nothing in fp16.
constexpr float MOST_FACTOR = 0x1p100f;

// What a key scale is multiplied by: a call's factor and the power of two that undoes a query row's, in two factors of half that power each.  Rows of tiny
// numbers over huge keys (or the other way round) have scores of an ordinary size: no product on the way to them may be a subnormal number.
struct RowScale {
    float first, second;
    __device__ RowScale(float factor, int power) : first(ldexpf(factor, power / 2)), second(ldexpf(1.f, power - power / 2)) {}
    __device__ float times(float ks) const { return ks * first * second; }
};

// 2^x as part * 2^power, 1/2 <= part < 1: what is multiplied by both in turn may be as large as 2^x is small.
struct Power {
    float part;
    int power;
    Power() = default;
    __device__ Power(float part, int power) : part(part), power(power) {}
    __device__ explicit Power(float x) {
        x = fmaxf(x, -1000.f);
        const float n = floorf(x) + 1.f;
        part = exp2_fast(x - n);
        power = (int)n;
    }
    __device__ float as_float() const { return ldexpf(part, power); }
    __device__ Power times(float w) const { return {part * __builtin_amdgcn_frexp_mantf(w), power + __builtin_amdgcn_frexp_expf(w)}; }
};

__device__ inline f32x4 times(f32x4 x, const Power& p) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = ldexpf(x[i] * p.part, p.power);
    return x;
}

// The larger of a lane's and the one 32 lanes on.
__device__ inline float over_halves(float x) {
    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
}

// 4 signed bytes to fp16, exactly: 1024 + (c + 128) is 0x6400 | byte.
__device__ inline void bytes_to_half(uint32_t w, half2_t& lo, half2_t& hi) {
    const uint32_t x = w ^ 0x80808080u;
    const uint32_t a = __builtin_amdgcn_perm(0x64646464u, x, 0x04010400u), b = __builtin_amdgcn_perm(0x64646464u, x, 0x04030402u);
    const half2_t bias = {(_Float16)1152.f, (_Float16)1152.f};
    lo = __builtin_bit_cast(half2_t, a) - bias;
    hi = __builtin_bit_cast(half2_t, b) - bias;
}

__device__ inline half8 codes_to_half(uint32_t w0, uint32_t w1) {
    half2_t r[4];
    bytes_to_half(w0, r[0], r[1]);
    bytes_to_half(w1, r[2], r[3]);
    return __builtin_bit_cast(half8, r);
}

// 8 elements of a query row.  (All of a row's are loaded before the first is looked at.)
__device__ inline void convert_query(u32x4 bits, uint32_t dtype, float (&x)[8]) {
    if (dtype == TYPE_F16) {
        const half8 v = __builtin_bit_cast(half8, bits);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (float)v[i];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(bits[i] << 16);
            x[2 * i + 1] = __uint_as_float(bits[i] & 0xFFFF0000u);
        }
    }
}

__device__ inline u32x4 load_query(const void* q, uint64_t at) {
    u32x4 x;
    __builtin_memcpy(&x, (const uint16_t*)q + at, 16);
    return x;
}

// An element as the products take it; of a row that holds an infinity or NaN all are NaN, which it then gives wherever it sees a key.
__device__ inline f16_t query_element(float x, float peak, int e) { return peak < __builtin_huge_valf() ? (f16_t)ldexpf(x, e) : (f16_t)__builtin_nanf(""); }

// The power of two that brings a bf16 row's largest magnitude to [2^13, 2^14); 1 for fp16, rows of zeros, infinities and NaN.
__device__ inline int query_exponent(float peak, uint32_t dtype) {
    if (dtype == TYPE_F16 || !(peak > 0.f && peak < __builtin_huge_valf())) return 0;
    int e;
    (void)frexpf(peak, &e);
    return 14 - e;
}

template <int N>
__device__ inline void store_out(void* out, uint64_t at, uint32_t dtype, const float (&x)[N]) {
    if (dtype == TYPE_F16) store_run((f16_t*)out + at, x);
    else store_run((bf16_t*)out + at, x);
}

// A unit's rows: the query heads of key head h for tokens of one sequence (or, with lists of pages, of one token).
struct Unit {
    uint32_t seq, head, first_token;   // first_token: its row in q
    uint32_t rows;                     // rows of the unit
    int32_t begin;                     // the first token's position
    uint32_t lo, hi;                   // keys that some row sees lie at lo .. hi of the axis (with lists: of the listed pages)
};

__device__ inline Unit unit_of(const AttendArgs& a, uint32_t index, uint32_t head) {
    Unit u;
    u.head = head;
    const bool lists = a.pages != nullptr;
    u.seq = lists ? index / a.batch.max_tokens : index;
    const uint32_t t = lists ? index % a.batch.max_tokens : 0;
    const NewTokens n = new_tokens(a.batch, u.seq);
    const uint32_t tokens = lists ? (t < n.count ? 1u : 0u) : n.count;
    u.first_token = n.first + t;
    u.begin = n.begin + (int32_t)t;
    u.rows = tokens * a.group;
    const int32_t last = u.begin + (int32_t)tokens - 1;
    u.lo = 0;
    if (lists) {
        u.hi = a.n_select << a.cache.shift;
    } else {
        u.hi = last < 0 ? 0u : min((uint32_t)last + 1u, a.batch.table_pages << a.cache.shift);
        if (a.window && u.begin >= 0 && (uint32_t)u.begin + 1u > a.window) u.lo = (uint32_t)u.begin + 1u - a.window;
    }
    return u;
}

// The unit as the rows of one of its tiles see it.
__device__ inline Unit tile_of(const AttendArgs& a, Unit u, uint32_t tile, uint32_t rows) {
    const uint32_t t0 = tile * rows / a.group, t1 = min((tile + 1) * rows - 1, u.rows - 1) / a.group;
    const int32_t p0 = u.begin + (int32_t)t0, p1 = u.begin + (int32_t)t1;
    u.hi = p1 < 0 ? 0u : min(u.hi, (uint32_t)p1 + 1u);
    u.lo = a.window && p0 >= 0 && (uint32_t)p0 + 1u > a.window ? (uint32_t)p0 + 1u - a.window : 0u;
    return u;
}

__device__ inline uint32_t unit_parts(const AttendArgs& a, const Unit& u) {
    const uint32_t first = u.lo / ATTEND_CHUNK, end = (u.hi + ATTEND_CHUNK - 1) / ATTEND_CHUNK;
    if (end <= first) return 1;
    return min((end - first + a.part_chunks - 1) / a.part_chunks, a.parts);
}

// The steps of a part; the last part of a call goes on to the end, however long a sequence is.
__device__ inline void part_range(const AttendArgs& a, const Unit& u, uint32_t part, uint32_t& begin, uint32_t& end) {
    const uint32_t first = u.lo / ATTEND_CHUNK, last = (u.hi + ATTEND_CHUNK - 1) / ATTEND_CHUNK;
    begin = first + part * a.part_chunks;
    end = part + 1 == a.parts ? last : min(last, begin + a.part_chunks);
}

// The page (or NO_PAGE) that a token of the axis lies on, and its place in the table.
template <bool LISTS>
__device__ inline uint32_t page_of(const AttendArgs& a, const uint32_t* table, const uint32_t* list, uint32_t token, uint32_t& place) {
    place = token >> a.cache.shift;
    bool there = true;
    if constexpr (LISTS) {
        there = place < a.n_select;
        place = list[min(place, a.n_select - 1)];
    }
    const uint32_t page = page_at(a.batch, table, place, a.cache.n_pages);
    return there ? page : NO_PAGE;
}

// ---- few rows: 16 to a workgroup, each of its W waves takes every W-th step of 64 tokens --------------------------------------
// Keys and values come from memory straight into the layout of the products: a lane reads 16 bytes of a key (or of a value channel's
// 16 tokens), converts them, and no LDS is used before the waves' results are joined.  Bound by memory: one token over 131072 of 8 heads of
// 128 channels (268 MB) 52 us, 5.2 TB/s, and 6.5 for the join; 64 sequences up to 4096 in pages of 16 (340 MB) 73 us, 4.7 TB/s; 4 sequences up to 500 of
// 64 channels 6.5 us.  Two waves to a SIMD with all registers they ask for: with three the spilled ones cost a third.
template <int ND, int W, bool LISTS>
__global__ __launch_bounds__(64 * W, ND <= 5 ? 2 : 1) void attend_few_kernel(AttendArgs a) {
    constexpr int D = ND * 32, NV = D / 16;
    __shared__ f32x4 joined[W / 2][NV][64];
    __shared__ float sums[W][16][2];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
    uint32_t id = a.first + blockIdx.x;
    const uint32_t part = id % a.parts;
    id /= a.parts;
    const uint32_t group_index = id;
    const uint32_t tile = id % a.tiles;
    id /= a.tiles;
    const Unit u = unit_of(a, id / a.cache.heads, id % a.cache.heads);
    if (tile * 16 >= u.rows || part >= unit_parts(a, u)) return;
    uint32_t c0, c1;
    part_range(a, u, part, c0, c1);
    const uint32_t* table = a.batch.tables + (uint64_t)u.seq * a.batch.table_pages;
    const uint32_t* list = LISTS ? a.pages + ((uint64_t)u.first_token * a.cache.heads + u.head) * a.n_select : nullptr;
    const uint32_t heads = a.cache.heads, q_heads = heads * a.group;

    // the row of this lane
    const uint32_t row = min(tile * 16 + r, u.rows - 1);
    const uint32_t token = u.first_token + row / a.group, q_head = u.head * a.group + row % a.group;
    const int32_t pos = u.begin + (int32_t)(row / a.group);
    const int32_t least = a.window ? max(pos - (int32_t)min(a.window, CACHE_MOST) + 1, 0) : 0;
    u32x4 raw[ND];
#pragma unroll
    for (int f = 0; f < ND; ++f)
        raw[f] = load_query(a.q, (uint64_t)token * a.q_stride + (uint64_t)q_head * D + (f < ND / 2 * 2 ? 64 * (f / 2) + 16 * (int)g + 8 * (f % 2) : 32 * f + 8 * (int)g));

    f32x4 o[NV] = {};
    float m = NEVER, top = NEVER, l = 0.f;
    // A step's codes are asked for as soon as the registers of the one before are free: keys behind the first product, values behind the
    // second.
    u32x4 kc[4][ND / 2 + 1], vc[NV];
    u32x2 kt[4];
    float ks = 0.f, vs = 0.f;
    const uint32_t slots = a.cache.page_tokens - 1;
    auto key_token = [&](uint32_t c) { return c * 64 + 16 * (r >> 2); };    // the first of the 16 around the key this lane reads
    auto value_token = [&](uint32_t c) { return c * 64 + 16 * g; };         // of those whose values it reads and whose scores it holds
    auto fetch_keys = [&](uint32_t page, uint32_t token) {
        page = page == NO_PAGE ? 0u : page;
        const int8_t* k = a.cache.k + (((uint64_t)page * heads + u.head) * a.cache.page_tokens + (token & slots) + (r & 3)) * D;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
            for (int f = 0; f < ND / 2; ++f) kc[t][f] = *(const u32x4*)(k + 4 * t * D + 64 * f + 16 * g);
            if constexpr (ND % 2) kt[t] = *(const u32x2*)(k + 4 * t * D + 32 * (ND - 1) + 8 * g);
        }
    };
    auto fetch_values = [&](uint32_t page, uint32_t token) {
        page = page == NO_PAGE ? 0u : page;
        const int8_t* v = a.cache.v + ((uint64_t)page * heads + u.head) * D * a.cache.page_tokens + (uint64_t)r * a.cache.page_tokens + (token & slots);
        ks = a.cache.ks[(uint64_t)page * heads + u.head];
        vs = a.cache.vs[(uint64_t)page * heads + u.head];
#pragma unroll
        for (int d = 0; d < NV; ++d) vc[d] = *(const u32x4*)(v + (uint64_t)(16 * d) * a.cache.page_tokens);
    };
    uint32_t c = c0 + wave;
    uint32_t k_place, v_place;
    uint32_t k_page = page_of<LISTS>(a, table, list, key_token(c), k_place), v_page = page_of<LISTS>(a, table, list, value_token(c), v_place);
    if (c < c1) {
        fetch_keys(k_page, key_token(c));
        fetch_values(v_page, value_token(c));
    }
    half8 q[ND];
    int e;
    {
        float x[8], peak = 0.f;
#pragma unroll
        for (int f = 0; f < ND; ++f) {
            convert_query(raw[f], a.dtype, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) peak = fmaxf(peak, x[i] == x[i] ? fabsf(x[i]) : __builtin_huge_valf());
        }
        peak = fmaxf(peak, __shfl_xor(peak, 16));
        peak = fmaxf(peak, __shfl_xor(peak, 32));
        e = query_exponent(peak, a.dtype);
#pragma unroll
        for (int f = 0; f < ND; ++f) {
            convert_query(raw[f], a.dtype, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) q[f][i] = query_element(x[i], peak, e);
        }
    }
    const RowScale row_scale(a.scale * LOG2E, -e);
    for (; c < c1; c += W) {
        // where the scores of this lane lie; a missing page's lie behind every row
        const int32_t at0 = v_page == NO_PAGE ? 0x7FFFFFFF - 64 : (int32_t)((v_place << a.cache.shift) + (value_token(c) & slots));
        k_page = page_of<LISTS>(a, table, list, key_token(c + W), k_place);
        v_page = page_of<LISTS>(a, table, list, value_token(c + W), v_place);
        f32x4 s[4] = {};
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
            for (int f = 0; f < ND / 2; ++f) {
                s[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_to_half(kc[t][f].x, kc[t][f].y), q[2 * f], s[t], 0, 0, 0);
                s[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_to_half(kc[t][f].z, kc[t][f].w), q[2 * f + 1], s[t], 0, 0, 0);
            }
            if constexpr (ND % 2) s[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_to_half(kt[t].x, kt[t].y), q[ND - 1], s[t], 0, 0, 0);
        }
        if (c + W < c1) fetch_keys(k_page, key_token(c + W));
        const bool whole = __all(at0 + 15 <= pos && at0 >= least);
        const float by = row_scale.times(ks);
        float peak = NEVER;
#pragma unroll
        for (int t = 0; t < 4; ++t) s[t] *= by;
        if (!whole) {
            rarely();
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int32_t at = at0 + 4 * t + i;
                    s[t][i] = ((at <= pos) & (at >= least)) ? s[t][i] : NEVER;
                }
        }
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) peak = fmaxf(peak, s[t][i]);
        const float log2_vs = log2_scale(vs);
        float high = raised(peak, log2_vs);
        high = fmaxf(high, __shfl_xor(high, 16));
        high = fmaxf(high, __shfl_xor(high, 32));
        peak = fmaxf(peak, __shfl_xor(peak, 16));
        peak = fmaxf(peak, __shfl_xor(peak, 32));
        if (__any(peak > m || high > top)) {
            const float m_new = fmaxf(m, peak), top_new = fmaxf(top, high);
            if (m_new != m) l *= exp2_fast(m - m_new);
            if (top_new != top) {
                const float keep = exp2_fast(top - top_new);
#pragma unroll
                for (int d = 0; d < NV; ++d) o[d] *= keep;
            }
            m = m_new;
            top = top_new;
        }
        const float base = or_zero(m);
        const float weight = p_factor(log2_vs, m, top);
        half8 p[2];
        if (__builtin_expect(__any(!(fabsf(weight) < MOST_FACTOR)), 0)) {
            rarely();      // scales very far apart, or no numbers; what is not seen may have any scale
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    l += exp2_fast(s[t][i] - base);
                    p[t / 2][t % 2 * 4 + i] = s[t][i] == NEVER ? (f16_t)0.f : (f16_t)exp2_fast(s[t][i] + p_shift(log2_vs, top));
                }
        } else {
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float e = exp2_fast(s[t][i] - base);
                    l += e;
                    p[t / 2][t % 2 * 4 + i] = (f16_t)(e * weight);
                }
        }
#pragma unroll
        for (int d = 0; d < NV; ++d) {
            o[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_to_half(vc[d].x, vc[d].y), p[0], o[d], 0, 0, 0);
            o[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_to_half(vc[d].z, vc[d].w), p[1], o[d], 0, 0, 0);
        }
        if (c + W < c1) fetch_values(v_page, value_token(c + W));
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    // the waves' results, in halves: the upper half's outputs go to the lower one through LDS, lane to lane
    if (g == 0) {
        sums[wave][r][0] = m;
        sums[wave][r][1] = l;
    }
    barrier();
    float most = NEVER, total = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) most = fmaxf(most, sums[w][r][0]);
#pragma unroll
    for (int w = 0; w < W; ++w) total += sums[w][r][1] * (sums[w][r][0] == most ? 1.f : exp2_fast(sums[w][r][0] - most));
    Power mine(top - P_TOP - or_zero(most));
    mine.part *= total == 0.f ? 0.f : 1.f / total;      // means, of a part too: sums may pass the largest number where the values are near it
#pragma unroll
    for (int d = 0; d < NV; ++d) o[d] = times(o[d], mine);
#pragma unroll
    for (int half = W / 2; half >= 1; half /= 2) {
        if (wave >= half && wave < 2 * half)
#pragma unroll
            for (int d = 0; d < NV; ++d) joined[wave - half][d][lane] = o[d];
        barrier();
        if (wave < half)
#pragma unroll
            for (int d = 0; d < NV; ++d) o[d] += joined[wave][d][lane];
        if (half > 1) barrier();
    }
    if (wave != 0 || tile * 16 + r >= u.rows) return;
    if (a.parts == 1) {
        const uint64_t at = (uint64_t)token * q_heads + q_head;
#pragma unroll
        for (int d = 0; d < NV; ++d) {
            const float y[4] = {o[d][0], o[d][1], o[d][2], o[d][3]};
            store_out(a.out, at * D + 16 * d + 4 * g, a.dtype, y);
        }
        if (a.lse && g == 0) a.lse[at] = total == 0.f ? NEVER : (most + log2f(total)) * LN2;
    } else {
        const uint64_t slot = ((uint64_t)group_index * a.parts + part) * 16 + r;
#pragma unroll
        for (int d = 0; d < NV; ++d) *(f32x4*)(a.part_out + slot * D + 16 * d + 4 * g) = o[d];
        if (g == 0) a.part_sums[slot] = make_float2(most, total);
    }
}

// ---- many rows: 128 or 256 to a workgroup, 32 to a wave, all over the same steps of 64 tokens ---------------------------------------
// Keys and values are converted once for the workgroup's waves on their way into LDS, two steps' worth of it: while one is computed
// with, the next one's codes are under way from memory.  Rows in LDS are 16 bytes apart from a multiple of their length: a wave's 16-byte
// reads then spread over all banks.  3584 tokens of 32 heads of 128 channels over up to 8192 (350 GFLOP): 430 to 500 us by card, 700 to 815 TFLOP/s; matrix cores
// 31 % busy, vector ALU 47 % (32 exponentials a lane and step, the codes' conversion), mostly one after the other.
// ONE: a step lies on one page (of 64 tokens or more), so its page and scales are the same for all.
template <int ND, int W, bool ONE>
__global__ __launch_bounds__(64 * W, W == 8 || ND <= 4 ? 2 : 1) void attend_many_kernel(AttendArgs a) {
    constexpr uint32_t ROWS = 32 * W;
    constexpr int NG = ONE ? 1 : 4;     // groups of a step's tokens with scales of their own
    constexpr int D = ND * 32, KS = D + 8, VS = 64 + 8, UNITS = D * 4, PER = (UNITS + 64 * W - 1) / (64 * W);
    __shared__ f16_t k_tile[2][64 * KS];
    __shared__ f16_t v_tile[2][D * VS];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 31, h = lane >> 5;
    // Workgroups go to the 8 XCDs in turn: where the heads of all sequences are a multiple of 8, an XCD gets all tiles of some of them, one after the
    // other, and their keys and values stay in its L2.  A head's longest tiles come first.  (Tiles of a long and a short sequence by turns
    // would be as bad as can be: an XCD's workgroups go to its parts in turn as well, and some would get the long ones only.)
    uint32_t id = a.first + blockIdx.x;
    const uint32_t xcds = a.unit_heads % 8 ? 1 : 8, lane_of = id % xcds;
    id /= xcds;
    const uint32_t tile = a.tiles - 1 - id % a.tiles;
    id /= a.tiles;
    const uint32_t part = id % a.parts, unit_head = id / a.parts * xcds + lane_of;
    const Unit whole_unit = unit_of(a, unit_head / a.cache.heads, unit_head % a.cache.heads);
    if (tile * ROWS >= whole_unit.rows) return;
    const Unit u = tile_of(a, whole_unit, tile, ROWS);
    if (part >= unit_parts(a, u)) return;
    uint32_t c0, c1;
    part_range(a, u, part, c0, c1);
    const uint32_t* table = a.batch.tables + (uint64_t)u.seq * a.batch.table_pages;
    const uint32_t heads = a.cache.heads, q_heads = heads * a.group, T = a.cache.page_tokens;

    const uint32_t row = tile * ROWS + wave * 32 + r;
    const bool there = row < u.rows;
    const uint32_t safe = min(row, u.rows - 1);
    const uint32_t token = u.first_token + safe / a.group, q_head = u.head * a.group + safe % a.group;
    const int32_t pos = u.begin + (int32_t)(safe / a.group);
    const int32_t least = a.window ? max(pos - (int32_t)min(a.window, CACHE_MOST) + 1, 0) : 0;
    // of the wave's rows
    const uint32_t w0 = min(tile * ROWS + wave * 32, u.rows - 1), w1 = min(tile * ROWS + wave * 32 + 31, u.rows - 1);
    const int32_t pos_first = u.begin + (int32_t)(w0 / a.group), pos_last = u.begin + (int32_t)(w1 / a.group);
    const int32_t least_first = a.window ? max(pos_first - (int32_t)min(a.window, CACHE_MOST) + 1, 0) : 0;
    const int32_t least_last = a.window ? max(pos_last - (int32_t)min(a.window, CACHE_MOST) + 1, 0) : 0;

    half8 q[D / 16];
    int e;
    {
        u32x4 raw[D / 16];
#pragma unroll
        for (int f = 0; f < D / 16; ++f) raw[f] = load_query(a.q, (uint64_t)token * a.q_stride + (uint64_t)q_head * D + 8 * h + 16 * f);
        float x[8], peak = 0.f;
#pragma unroll
        for (int f = 0; f < D / 16; ++f) {
            convert_query(raw[f], a.dtype, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) peak = fmaxf(peak, x[i] == x[i] ? fabsf(x[i]) : __builtin_huge_valf());
        }
        peak = fmaxf(peak, __shfl_xor(peak, 32));
        e = query_exponent(peak, a.dtype);
#pragma unroll
        for (int f = 0; f < D / 16; ++f) {
            convert_query(raw[f], a.dtype, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) q[f][i] = query_element(a.scale < 0.f ? -x[i] : x[i], peak, e);
        }
    }
    const RowScale row_scale(fabsf(a.scale) * LOG2E, -e);

    // a step's codes: `PER` runs of 16 keys' channels and 16 values' tokens a thread; the pages of its four 16 tokens and their scales
    u32x4 kc[PER], vc[PER];
    uint32_t absent, next_absent;
    float ks[NG], v_log2[NG], next_ks, next_vs;
    uint64_t odd;       // scales of the step that are no numbers, or values' of 0
    // A lane keeps the page and the scales of one of the four: vector loads, which come in order with the codes, a step ahead of their use.
    uint32_t own_page = page_at(a.batch, table, (c0 * 64 + 16 * (lane & 3)) >> a.cache.shift, a.cache.n_pages);
    auto fetch = [&](uint32_t c) {
        uint32_t page[NG];
        next_absent = 0;
#pragma unroll
        for (int j = 0; j < NG; ++j) {
            page[j] = (uint32_t)__builtin_amdgcn_readlane((int)own_page, j);
            next_absent |= page[j] == NO_PAGE ? (ONE ? 15u : 1u << j) : 0u;
            page[j] = page[j] == NO_PAGE ? 0u : page[j];
        }
        const uint64_t at = (uint64_t)(own_page == NO_PAGE ? 0u : own_page) * heads + u.head;
        next_ks = a.cache.ks[at];
        next_vs = a.cache.vs[at];
        own_page = page_at(a.batch, table, ((c + 1) * 64 + 16 * (lane & 3)) >> a.cache.shift, a.cache.n_pages);
        if constexpr (ONE) {
            const int8_t* k = a.cache.k + (((uint64_t)page[0] * heads + u.head) * T + ((c * 64) & (T - 1))) * D;     // the same for all
            const int8_t* v = a.cache.v + ((uint64_t)page[0] * heads + u.head) * D * T + ((c * 64) & (T - 1));
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const uint32_t n = min(threadIdx.x + 64 * W * i, (uint32_t)UNITS - 1);
                kc[i] = *(const u32x4*)(k + 16 * n);
                vc[i] = *(const u32x4*)(v + ((n >> 2) * T + 16 * (n & 3)));
            }
        } else {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const uint32_t n = min(threadIdx.x + 64 * W * i, (uint32_t)UNITS - 1);
                const uint32_t t = n / (D / 16), d = n % (D / 16) * 16, j = t >> 4;
                const uint32_t kp = j < 2 ? (j == 0 ? page[0] : page[1 % NG]) : (j == 2 ? page[2 % NG] : page[3 % NG]);
                kc[i] = *(const u32x4*)(a.cache.k + (((uint64_t)kp * heads + u.head) * T + ((c * 64 + t) & (T - 1))) * D + d);
                const uint32_t jv = n & 3, dv = n >> 2;
                const uint32_t vp = jv < 2 ? (jv == 0 ? page[0] : page[1 % NG]) : (jv == 2 ? page[2 % NG] : page[3 % NG]);
                vc[i] = *(const u32x4*)(a.cache.v + (((uint64_t)vp * heads + u.head) * D + dv) * T + ((c * 64 + 16 * jv) & (T - 1)));
            }
        }
    };
    auto put = [&](int buffer) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const uint32_t n = min(threadIdx.x + 64 * W * i, (uint32_t)UNITS - 1);
            f16_t* k = &k_tile[buffer][n / (D / 16) * KS + n % (D / 16) * 16];
            *(half8*)k = codes_to_half(kc[i].x, kc[i].y);
            *(half8*)(k + 8) = codes_to_half(kc[i].z, kc[i].w);
            f16_t* v = &v_tile[buffer][(n >> 2) * VS + (n & 3) * 16];
            *(half8*)v = codes_to_half(vc[i].x, vc[i].y);
            *(half8*)(v + 8) = codes_to_half(vc[i].z, vc[i].w);
        }
    };
    auto next = [&]() {
        absent = next_absent;
        const float v = log2_scale(next_vs);      // by the lane that has the page
        odd = __ballot(!(fabsf(next_ks) < __builtin_huge_valf() && fabsf(v) < __builtin_huge_valf())) & (ONE ? 1 : 15);
#pragma unroll
        for (int j = 0; j < NG; ++j) {
            ks[j] = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(next_ks), j));
            v_log2[j] = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), j));
        }
    };

    f32x16 o[ND] = {};
    float m = NEVER, top = NEVER, l = 0.f;
    // row m of a product's 32 tokens is token 16 (m / 16) + 8 (m / 4 % 2) + 4 (m / 8 % 2) + m % 4: a lane's 16 scores are then two runs of 8 tokens
    const uint32_t k_row = 16 * (r >> 4) + 8 * ((r >> 2) & 1) + 4 * ((r >> 3) & 1) + (r & 3);
    if (c0 < c1) {
        fetch(c0);
        put(0);
        next();
        fetch(c0 + 1);
    }
    for (uint32_t c = c0; c < c1; ++c) {
        const int buffer = (c - c0) & 1;
        barrier();
        const int32_t from = (int32_t)(c * 64);
        const bool seen = from <= pos_last && from + 63 >= least_first && tile * ROWS + wave * 32 < u.rows;
        f32x16 s[2] = {};
        if (seen) {
#pragma unroll
            for (int f = 0; f < D / 16; ++f)
#pragma unroll
                for (int mt = 0; mt < 2; ++mt)
                    s[mt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(*(const half8*)&k_tile[buffer][(32 * mt + k_row) * KS + 16 * f + 8 * h], q[f], s[mt], 0, 0, 0);
        }
        // behind the barrier nobody reads the other buffer: the next step goes there beside the products (behind the last step nothing of use)
        put(buffer ^ 1);
        float by[NG], log2_vs[NG];
        uint32_t gone = absent;
        const bool numbers = odd == 0;
#pragma unroll
        for (int j = 0; j < NG; ++j) {
            by[j] = row_scale.times(ks[j]);
            by[j] = by[j] < LEAST_SCALE ? LEAST_SCALE : by[j];
            log2_vs[j] = v_log2[j];
        }
        next();
        fetch(c + 2);
        if (!seen) continue;
        const bool inside = from + 63 <= pos_first && from >= least_last && !gone;
        if (!inside) {
            rarely();
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int j = 2 * mt + i / 8;
                    const int32_t at = from + 16 * j + 8 * (int32_t)h + i % 8;
                    s[mt][i] = ((at <= pos) & (at >= least) & !(gone >> j & 1)) ? s[mt][i] : NEVER;
                }
        }
        float peak = NEVER, high = NEVER, peaks[NG];
#pragma unroll
        for (int j = 0; j < NG; ++j) {
            float x = s[j / 2][j % 2 * 8];
#pragma unroll
            for (int i = 1; i < 32 / NG; ++i) x = fmaxf(x, s[(8 * j + i) / 16][(8 * j + i) % 16]);
            peaks[j] = x * by[j];
            peak = fmaxf(peak, peaks[j]);
            high = fmaxf(high, peaks[j] + log2_vs[j]);
        }
        if (!numbers) {
            rarely();
            high = NEVER;
#pragma unroll
            for (int j = 0; j < NG; ++j) high = fmaxf(high, raised(peaks[j], log2_vs[j]));
        }
        peak = over_halves(peak);
        high = over_halves(high);
        // The references m and top follow the largest only when it has passed them by SLACK: what they are does not matter, as long as P stays in range.
        if (__any(peak > m + SLACK || high > top + SLACK)) {
            const float m_new = fmaxf(m, peak), top_new = fmaxf(top, high);
            if (m_new != m) l *= exp2_fast(m - m_new);
            const float keep = top_new != top ? exp2_fast(top - top_new) : 1.f;
#pragma unroll
            for (int d = 0; d < ND; ++d) o[d] *= keep;
            m = m_new;
            top = top_new;
        }
        half8 vf[ND];      // of wide heads, one wave to a SIMD: the first values' way from LDS is hidden behind the exponentials
        auto first_values = [&]() {
            if constexpr (ND >= 7) {
#pragma unroll
                for (int d = 0; d < ND; ++d) vf[d] = *(const half8*)&v_tile[buffer][(32 * d + r) * VS + 8 * h];
            }
        };
        const float base = or_zero(m);
        half8 p[4];
        // A step's P and sums from the same exponentials e^(s - m) weight where the weight, 2^(shift + base), is an ordinary number for all rows and the
        // keys' scale one at all, otherwise (scales very far apart, or 0, or no numbers) from e^(s - m).
        const float shift = p_shift(log2_vs[0], top);
        if (ONE && numbers && __all(fabsf(shift + base) < 60.f)) {
            first_values();
            float part[4] = {};
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float e = exp2_fast(fmaf(s[j / 2][j % 2 * 8 + i], by[0], shift));
                    part[j] += e;
                    p[j][i] = (f16_t)e;
                }
            l += (part[0] + part[1] + (part[2] + part[3])) * exp2_fast(-shift - base);
        } else {
            float weight[NG];
#pragma unroll
            for (int j = 0; j < NG; ++j) weight[j] = p_factor(log2_vs[j], m, top);
            float most = weight[0];
#pragma unroll
            for (int j = 1; j < NG; ++j) most = fmaxf(most, weight[j]);
            const bool apart = !numbers || __any(most >= MOST_FACTOR);
            float base_of = base, kept = l;
            if (__builtin_expect(apart, 0)) {
                rarely();      // scales very far apart, or no numbers; what is not seen may have any scale: P's exponents in place of the scores
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float shift_of = p_shift(log2_vs[ONE ? 0 : j], top);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        float x = s[j / 2][j % 2 * 8 + i];
                        const bool shown = x != NEVER;
                        x *= by[ONE ? 0 : j];
                        kept += shown ? exp2_fast(x - base) : 0.f;
                        x = shown ? x + shift_of : NEVER;
                        s[j / 2][j % 2 * 8 + i] = x;
                    }
                }
#pragma unroll
                for (int j = 0; j < NG; ++j) by[j] = weight[j] = 1.f;
                base_of = 0.f;
            }
            first_values();
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float e = exp2_fast(fmaf(s[j / 2][j % 2 * 8 + i], by[ONE ? 0 : j], -base_of));
                    s[j / 2][j % 2 * 8 + i] = e;
                    p[j][i] = (f16_t)(e * weight[ONE ? 0 : j]);
                }
            if (!ONE || !apart) {      // small pages: no branch here, which parted the exponentials from the products (128 channels 527 for 547 us)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float part = 0.f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) part += s[j / 2][j % 2 * 8 + i];
                    l += part;
                }
            }
            l = apart ? kept : l;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int d = 0; d < ND; ++d)
                o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ND >= 7 && j == 0 ? vf[d] : *(const half8*)&v_tile[buffer][(32 * d + r) * VS + 16 * j + 8 * h],
                                                              p[j], o[d], 0, 0, 0);
    }
    l += __shfl_xor(l, 32);
    if (!there) return;
    const Power mine(top - P_TOP - or_zero(m));
    const float by = mine.part * (l == 0.f ? 0.f : 1.f / l);      // means, of a part too
    const uint64_t at = (uint64_t)token * q_heads + q_head;
    const uint64_t slot = (((uint64_t)unit_head * a.tiles + tile) * a.parts + part) * ROWS + wave * 32 + r;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int ch = 32 * d + 8 * j + 4 * (int)h;
            float y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = ldexpf(o[d][4 * j + i] * by, mine.power);
            if (a.parts == 1) store_out(a.out, at * D + ch, a.dtype, y);
            else __builtin_memcpy(a.part_out + slot * D + ch, y, 16);
        }
    if (h == 0) {
        if (a.parts > 1) a.part_sums[slot] = make_float2(m, l);
        else if (a.lse) a.lse[at] = l == 0.f ? NEVER : (m + log2f(l)) * LN2;
    }
}

// ---- the parts of the keys' axis joined: a workgroup a row ---------------------------------------------------------------------
// First the parts' factors, a thread a part, then their outputs, the parts spread over groups of lanes that hold 4 channels each.  Latency: 64 parts of 32
// rows 6.5 us (47 when every thread went through all the sums).
constexpr uint32_t MOST_PARTS = ATTEND_MOST_GROUPS;

__device__ inline float over_workgroup(float x, bool max, float* parts) {
#pragma unroll
    for (int o = 1; o < 64; o *= 2) x = max ? fmaxf(x, __shfl_xor(x, o)) : x + __shfl_xor(x, o);
    if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = x;
    barrier();
    return max ? fmaxf(fmaxf(parts[0], parts[1]), fmaxf(parts[2], parts[3])) : parts[0] + parts[1] + parts[2] + parts[3];
}

__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs a, uint32_t rows, uint32_t used) {
    __shared__ f32x4 joined[256];
    __shared__ Power factors[MOST_PARTS];
    __shared__ float most4[4], sum4[4];
    const uint32_t D = a.cache.dim, per = D / 4, lanes = 256 / per;
    uint32_t id = blockIdx.x;
    const uint32_t rr = id % used;       // used: rows of a workgroup that a unit can have
    id /= used;
    const uint32_t group_index = id, tile = id % a.tiles;
    id /= a.tiles;
    Unit u = unit_of(a, id / a.cache.heads, id % a.cache.heads);
    const uint32_t row = tile * rows + rr;
    if (row >= u.rows) return;
    if (rows != ATTEND_FEW) u = tile_of(a, u, tile, rows);
    const uint32_t parts = unit_parts(a, u);
    const uint64_t slot0 = (uint64_t)group_index * a.parts * rows + rr;
    float m = NEVER, l = 0.f;
    for (uint32_t i = threadIdx.x; i < parts; i += 256) m = fmaxf(m, a.part_sums[slot0 + (uint64_t)i * rows].x);
    m = over_workgroup(m, true, most4);
    for (uint32_t i = threadIdx.x; i < parts; i += 256) {
        const float2 s = a.part_sums[slot0 + (uint64_t)i * rows];
        const Power f = Power(s.x == m ? 0.f : s.x - m).times(s.y);
        factors[i] = f;
        l += f.as_float();
    }
    l = over_workgroup(l, false, sum4);
    const float by = l == 0.f ? 0.f : 1.f / l;
    const uint32_t part0 = threadIdx.x / per, d = threadIdx.x % per * 4;
    f32x4 x = {};
    if (part0 < lanes) {
        const float* from = a.part_out + slot0 * D + d;
        const uint64_t apart = (uint64_t)rows * D;
#pragma unroll 4
        for (uint32_t i = part0; i < parts; i += lanes) x += times(*(const f32x4*)(from + i * apart), factors[i].times(by));
    }
    joined[threadIdx.x] = x;
    barrier();
    if (part0 != 0) return;
    for (uint32_t i = 1; i < lanes; ++i) x += joined[i * per + threadIdx.x];
    const uint64_t at = (uint64_t)(u.first_token + row / a.group) * (a.cache.heads * a.group) + u.head * a.group + row % a.group;
    const float y[4] = {x[0], x[1], x[2], x[3]};
    store_out(a.out, at * D + d, a.dtype, y);
    if (a.lse && d == 0) a.lse[at] = l == 0.f ? NEVER : (m + log2f(l)) * LN2;
}

// Of up to 32 parts: a wave a row (4 us for 32 rows of 16 parts).
__global__ __launch_bounds__(256) void attend_join_few_kernel(AttendArgs a, uint32_t rows, uint32_t used, uint64_t n) {
    const uint32_t D = a.cache.dim, per = D / 4, lane = threadIdx.x & 63;
    const uint64_t index = (uint64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (index >= n) return;
    uint32_t id = (uint32_t)(index / used);
    const uint32_t rr = (uint32_t)(index % used), group_index = id, tile = id % a.tiles;
    id /= a.tiles;
    Unit u = unit_of(a, id / a.cache.heads, id % a.cache.heads);
    const uint32_t row = tile * rows + rr;
    if (row >= u.rows) return;
    if (rows != ATTEND_FEW) u = tile_of(a, u, tile, rows);
    const uint32_t parts = unit_parts(a, u);
    const uint64_t slot0 = (uint64_t)group_index * a.parts * rows + rr;
    const float2 s = lane < parts ? a.part_sums[slot0 + (uint64_t)lane * rows] : make_float2(NEVER, 0.f);
    float m = s.x;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) m = fmaxf(m, __shfl_xor(m, o));
    m = __shfl(m, 0);
    Power f = Power(s.x == m ? 0.f : s.x - m).times(s.y);
    float l = f.as_float();
#pragma unroll
    for (int o = 1; o < 32; o *= 2) l += __shfl_xor(l, o);
    l = __shfl(l, 0);
    f = f.times(l == 0.f ? 0.f : 1.f / l);
    // of heads of up to 128 channels each half of the wave sees to every other part
    const uint32_t halves = per <= 32 ? 2 : 1, half = halves == 2 ? lane >> 5 : 0, at4 = halves == 2 ? lane & 31 : lane;
    f32x4 x = {};
    const float* from = a.part_out + slot0 * D + min(at4, per - 1) * 4;
    const uint64_t apart = (uint64_t)rows * D;
    for (uint32_t i0 = 0; i0 < parts; i0 += 8) {
        f32x4 v[8];
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j)
            if (j < 8 / halves) v[j] = *(const f32x4*)(from + min(i0 + j * halves + half, parts - 1) * apart);
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j)
            if (j < 8 / halves) {
                const uint32_t i = i0 + j * halves + half;
                const Power by{__shfl(f.part, i & 63), __shfl(f.power, i & 63)};
                if (i < parts) x += times(v[j], by);
            }
    }
    if (halves == 2)
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] += __shfl_xor(x[i], 32);
    if (half || at4 >= per) return;
    const uint64_t at = (uint64_t)(u.first_token + row / a.group) * (a.cache.heads * a.group) + u.head * a.group + row % a.group;
    const float y[4] = {x[0], x[1], x[2], x[3]};
    store_out(a.out, at * D + lane * 4, a.dtype, y);
    if (a.lse && lane == 0) a.lse[at] = l == 0.f ? NEVER : (m + log2f(l)) * LN2;
}

template <int ND>
void launch_attend(const AttendArgs& a, const AttendPlan& p, uint32_t workgroups, hipStream_t stream) {
    const dim3 grid(workgroups);
    if (p.few && p.waves == 4) {
        if (a.pages) attend_few_kernel<ND, 4, true><<<grid, dim3(256), 0, stream>>>(a);
        else attend_few_kernel<ND, 4, false><<<grid, dim3(256), 0, stream>>>(a);
    } else if (p.few) {
        if constexpr (ND <= 5) {
            if (a.pages) attend_few_kernel<ND, 8, true><<<grid, dim3(512), 0, stream>>>(a);
            else attend_few_kernel<ND, 8, false><<<grid, dim3(512), 0, stream>>>(a);
        }
    }
    else if (p.rows == 256) {
        if constexpr (ND >= 4 && ND <= 6) {
            if (a.cache.page_tokens >= 64) attend_many_kernel<ND, 8, true><<<grid, dim3(512), 0, stream>>>(a);
            else attend_many_kernel<ND, 8, false><<<grid, dim3(512), 0, stream>>>(a);
        }
    } else {
        if (a.cache.page_tokens >= 64) attend_many_kernel<ND, 4, true><<<grid, dim3(256), 0, stream>>>(a);
        else attend_many_kernel<ND, 4, false><<<grid, dim3(256), 0, stream>>>(a);
    }
}

}  // namespace

hipError_t launch_cache_attention(AttendArgs a, const AttendPlan& p, void* workspace, hipStream_t stream) {
    a.parts = p.parts;
    a.part_chunks = p.part_chunks;
    a.tiles = p.tiles;
    a.unit_heads = p.units * a.cache.heads;
    a.part_out = (float*)workspace;
    a.part_sums = (float2*)((char*)workspace + p.sums);
    attend_launches(p, [&](uint32_t first, uint32_t workgroups) {
        a.first = first;
        switch (a.cache.dim / 32) {
            case 1: launch_attend<1>(a, p, workgroups, stream); break;
            case 2: launch_attend<2>(a, p, workgroups, stream); break;
            case 3: launch_attend<3>(a, p, workgroups, stream); break;
            case 4: launch_attend<4>(a, p, workgroups, stream); break;
            case 5: launch_attend<5>(a, p, workgroups, stream); break;
            case 6: launch_attend<6>(a, p, workgroups, stream); break;
            case 7: launch_attend<7>(a, p, workgroups, stream); break;
            default: launch_attend<8>(a, p, workgroups, stream); break;
        }
    });
    if (p.parts > 1) {
        const uint32_t used = (uint32_t)std::min<uint64_t>(p.rows, (uint64_t)a.group * (a.pages ? 1 : a.batch.max_tokens));
        const uint64_t rows = p.groups * used;
        if (p.parts <= 32) attend_join_few_kernel<<<dim3((uint32_t)divided_up(rows, 4)), dim3(256), 0, stream>>>(a, p.rows, used, rows);
        else attend_join_kernel<<<dim3((uint32_t)rows), dim3(256), 0, stream>>>(a, p.rows, used);
    }
    return hipGetLastError();
}

}  // namespace dessert
