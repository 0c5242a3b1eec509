// Log probabilities of given tokens, the entropy and the best alternatives of rows of logits, in one pass over the logits.
// With m = max_j l_j, s = sum_j e^(l_j - m) and t = sum_j e^(l_j - m) (l_j - m):
//     log p(token) = (l_token - m) - log s,    entropy = log s - t / s,
// and two parts of a row join by moving both to the larger m: s' = e^d s, t' = e^d (t + d s) with d = m - m'.
// Entries of -inf have no probability and are never an alternative; a row with +inf or NaN has s = NaN and gives NaN.
#include "kernels.hpp"
#include "launch_slices.hpp"
#include "number_formats.hpp"

namespace dessert {

namespace {

constexpr float LOG2E = 1.44269504088896340736f;
constexpr float MINUS_INF = -__builtin_huge_valf();
constexpr uint32_t NONE = 0xFFFFFFFFu;

struct Sums {
    float m, s, t;
};

__device__ inline float exp_of(float d) { return __builtin_amdgcn_exp2f(d * LOG2E); }

// The parts' sums moved to the larger maximum and added.
__device__ inline Sums join(Sums a, Sums b) {
    Sums o;
    o.m = fmaxf(a.m, b.m);
    o.s = o.t = 0.f;
    if (a.m != MINUS_INF) {   // else nothing in it (s = 0), or NaN
        const float d = a.m - o.m, e = exp_of(d);
        o.s = e * a.s;
        o.t = e == 0.f ? 0.f : e * (a.t + d * a.s);
    } else {
        o.s = a.s;
    }
    if (b.m != MINUS_INF) {
        const float d = b.m - o.m, e = exp_of(d);
        o.s += e * b.s;
        o.t += e == 0.f ? 0.f : e * (b.t + d * b.s);
    } else {
        o.s += b.s;
    }
    return o;
}

// A key orders entries by value, then by lower column; 0 stands for none.  Values are whole floats; -0 counts as +0.
__device__ inline uint32_t order_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ inline float value_of(uint32_t order) { return __uint_as_float(order & 0x80000000u ? order & 0x7FFFFFFFu : ~order); }
__device__ inline uint64_t key_of(uint32_t order, uint32_t col) { return (uint64_t)order << 32 | (uint32_t)~col; }
constexpr uint32_t ORDER_FLOOR = 0x007FFFFFu;   // of -inf, which is no alternative

// LDS written by some lanes of a wave and read by others of it: their order in the code is the order that they are done in.
__device__ inline void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

constexpr uint32_t POOL = 256;   // keys a wave keeps

// The entries that a wave has found no reason to leave out of the n_top best: in no order, in LDS.  bound: the order of a value that
// n_top entries seen are not below; what is below it is out.
struct Pool {
    uint64_t* keys;
    uint32_t count = 0, bound = ORDER_FLOOR;
    uint32_t grown = 0;             // keys since the bound was last looked for
    uint32_t peaks[4] = {0, 0, 0, 0};   // the orders of the largest of four parts of the entries that the lane has had

    // The n_top largest of `count` keys, sorted: a key's place is the number of larger ones (no two are equal).
    __device__ void compress(uint32_t n_top, uint32_t lane) {
        uint64_t mine[POOL / 64];
        uint32_t place[POOL / 64];
#pragma unroll
        for (uint32_t j = 0; j < POOL / 64; ++j) {
            mine[j] = j * 64 + lane < count ? keys[j * 64 + lane] : 0;
            place[j] = 0;
        }
        for (uint32_t i = 0; i < count; i += 2) {
            const uint64_t k0 = keys[i], k1 = i + 1 < count ? keys[i + 1] : 0;
#pragma unroll
            for (uint32_t j = 0; j < POOL / 64; ++j) place[j] += (uint32_t)(k0 > mine[j]) + (uint32_t)(k1 > mine[j]);
        }
        wave_sync();
#pragma unroll
        for (uint32_t j = 0; j < POOL / 64; ++j)
            if (mine[j] && place[j] < n_top) keys[place[j]] = mine[j];
        wave_sync();
        if (count >= n_top) {
            count = n_top;
            bound = max(bound, (uint32_t)__builtin_amdgcn_readfirstlane((int)(keys[n_top - 1] >> 32)));
        }
    }
    // A key from every lane that wants one in; there has to be room.
    __device__ void add(bool want, uint64_t key) {
        const uint64_t all = __ballot(want);
        if (!all) return;
        grown += __popcll(all);
        if (want) keys[count + __builtin_amdgcn_mbcnt_hi((uint32_t)(all >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)all, 0))] = key;
        count += __popcll(all);
    }
    // now: the orders of the largest of four parts of the entries that the lane has now.  false: none can be among the best.  The n_top-th
    // largest of the peaks so far bounds the n_top-th largest entry so far from below; its upper 18 bits, by bisection, leave in little
    // more than n_top entries of the first ones and few of the later ones.  (The lanes' own peaks do for a few alternatives; of 64 they
    // would be the least.)
    // IN_ORDER: entries come with rising columns, so that a later one that only equals the bound is out.
    template <bool IN_ORDER>
    __device__ bool raise(const uint32_t (&now)[4], uint32_t n_top) {
        const uint32_t best = max(max(now[0], now[1]), max(now[2], now[3]));
        const uint32_t above = __popcll(__ballot(IN_ORDER ? best > bound : best >= max(bound, ORDER_FLOOR + 1)));
#pragma unroll
        for (int q = 0; q < 4; ++q) peaks[q] = max(peaks[q], now[q]);
        if (above == 0) return false;
        if (grown + above < n_top) return true;
        grown = 0;
        uint32_t b = 0;
        if (n_top <= 16) {
            const uint32_t peak = max(max(peaks[0], peaks[1]), max(peaks[2], peaks[3]));
#pragma unroll
            for (int bit = 31; bit >= 14; --bit) {
                const uint32_t t = b | 1u << bit;
                if ((uint32_t)__popcll(__ballot(peak >= t)) >= n_top) b = t;
            }
        } else {
#pragma unroll 1
            for (int bit = 31; bit >= 14; --bit) {
                const uint32_t t = b | 1u << bit;
                uint32_t n = 0;
#pragma unroll
                for (int q = 0; q < 4; ++q) n += __popcll(__ballot(peaks[q] >= t));
                if (n >= n_top) b = t;
            }
        }
        bound = max(bound, b);
        return true;
    }
};

// The best n_top of the four waves' pools and the row's sums, to the outputs (or, of a part of a row, to the parts).  `finals` and `totals`
// are the workgroup's; all 256 threads take part.
struct Totals {
    Sums sums[4];
    uint32_t bound[4], count, above[2][4];
};

// The bound once more, over the whole workgroup's `count` keys (at most 1024), where they are many: those below it go.  All threads take part;
// `spare` has room for the keys.
__device__ inline uint32_t thin_out(uint64_t* finals, uint64_t* spare, Totals& totals, uint32_t count, uint32_t n_top) {
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint64_t mine[POOL / 64];
#pragma unroll
    for (uint32_t j = 0; j < POOL / 64; ++j) mine[j] = threadIdx.x + 256 * j < count ? finals[threadIdx.x + 256 * j] : 0;
    uint32_t b = 0;
#pragma unroll 1
    for (int bit = 31; bit >= 14; --bit) {
        const uint32_t t = b | 1u << bit;
        uint32_t n = 0;
#pragma unroll
        for (uint32_t j = 0; j < POOL / 64; ++j) n += __popcll(__ballot((uint32_t)(mine[j] >> 32) >= t));
        uint32_t* above = totals.above[bit & 1];   // the other turn's are read until the next barrier
        if (lane == 0) above[wave] = n;
        __syncthreads();
        if (above[0] + above[1] + above[2] + above[3] >= n_top) b = t;
    }
    if (threadIdx.x == 0) totals.count = 0;
    __syncthreads();
#pragma unroll
    for (uint32_t j = 0; j < POOL / 64; ++j)
        if (mine[j] && (uint32_t)(mine[j] >> 32) >= b) spare[atomicAdd(&totals.count, 1u)] = mine[j];
    __syncthreads();
    const uint32_t left = totals.count;
    for (uint32_t i = threadIdx.x; i < left; i += 256) finals[i] = spare[i];
    __syncthreads();
    return left;
}
__device__ inline Sums wave_total(Sums z) {
    float m = z.m;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) m = fmaxf(m, __shfl_xor(m, o));
    z = join(z, Sums{m, 0.f, 0.f});   // moved to the wave's maximum
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
        z.s += __shfl_xor(z.s, o);
        z.t += __shfl_xor(z.t, o);
    }
    return z;
}

// The row's sums over the four waves, in all threads.
__device__ inline Sums row_total(Sums z, const Pool& pool, Totals& totals) {
    z = wave_total(z);
    if ((threadIdx.x & 63) == 0) {
        totals.sums[threadIdx.x >> 6] = z;
        totals.bound[threadIdx.x >> 6] = pool.bound;
        if (threadIdx.x == 0) totals.count = 0;
    }
    __syncthreads();
    return join(join(totals.sums[0], totals.sums[1]), join(totals.sums[2], totals.sums[3]));
}

// After row_total: sink(place, key) for every place < n_top, by one thread each; key 0 where there is no entry.
template <typename Sink>
__device__ inline void rank_best(uint32_t n_top, const Pool& pool, uint64_t* pools, uint64_t* finals, Totals& totals, Sink sink) {
    const uint32_t bound = max(max(totals.bound[0], totals.bound[1]), max(totals.bound[2], totals.bound[3]));
    for (uint32_t i = threadIdx.x & 63; i < pool.count; i += 64)
        if ((uint32_t)(pool.keys[i] >> 32) >= bound) finals[atomicAdd(&totals.count, 1u)] = pool.keys[i];
    __syncthreads();
    uint32_t count = totals.count;
    if (count > 2 * n_top && count > 96) count = thin_out(finals, pools, totals, count, n_top);
    for (uint32_t j = threadIdx.x; j < max(count, n_top); j += 256) {
        const uint64_t mine = j < count ? finals[j] : 0;
        uint32_t place = j;   // behind the last key: an unused slot
        if (j < count) {
            place = 0;
            for (uint32_t i = 0; i < count; i += 8) {   // what lies behind the last key is read, but not counted
                uint64_t other[8];
#pragma unroll
                for (uint32_t u = 0; u < 8; ++u) other[u] = finals[i + u];
#pragma unroll
                for (uint32_t u = 0; u < 8; ++u) place += (uint32_t)(i + u < count) & (uint32_t)(other[u] > mine);
            }
        }
        if (place < n_top) sink(place, mine);
    }
}

// A row's log probability and entropy, by one thread; logit: of its token, where that is in the vocabulary.
__device__ inline void write_row(const LogprobArgs& g, uint64_t row, uint32_t token, Sums z, float log_s, float logit) {
    const bool nan = z.s != z.s, empty = z.s == 0.f;
    if (g.entropy) g.entropy[row] = empty ? 0.f : log_s - z.t / z.s;
    if (g.tokens) {
        const float lp = nan ? z.s : empty || token >= g.vocab ? MINUS_INF : (logit - z.m) - log_s;
        g.logprobs[row] = token == NONE ? 0.f : lp;
    }
}

__device__ inline void write_place(const LogprobArgs& g, uint64_t row, uint32_t place, uint64_t key, float m, float log_s) {
    const bool nan = log_s != log_s, some = key && !nan;
    g.top_ids[row * g.n_top + place] = some ? ~(uint32_t)key : NONE;
    g.top_logprobs[row * g.n_top + place] = nan ? log_s : some ? (value_of((uint32_t)(key >> 32)) - m) - log_s : MINUS_INF;
}

// part: all ones for a whole row, else where its parts go.
template <typename T>
__device__ inline void finish(const LogprobArgs& g, uint64_t row, Sums z, Pool& pool, uint64_t* pools, uint64_t* finals, Totals& totals, uint64_t part) {
    z = row_total(z, pool, totals);
    const bool whole = part == ~0ull;
    const float log_s = logf(z.s);
    if (threadIdx.x == 0) {
        if (whole) {
            const uint32_t token = g.tokens ? g.tokens[row] : NONE;
            write_row(g, row, token, z, log_s, token < g.vocab ? (float)((const T*)g.logits)[row * g.stride + token] : 0.f);
        } else {
            g.part_sums[3 * part] = z.m;
            g.part_sums[3 * part + 1] = z.s;
            g.part_sums[3 * part + 2] = z.t;
        }
    }
    if (!g.n_top) return;
    rank_best(g.n_top, pool, pools, finals, totals, [&](uint32_t place, uint64_t key) {
        if (whole) write_place(g, row, place, key, z.m, log_s);
        else g.part_keys[part * g.n_top + place] = key;
    });
}

// Entries c0 + (256 j + thread) * 8 ... of a row, 8 for each j, as they lie in memory; -inf from `end` on.
template <typename T, int V>
struct Entries {
    static constexpr int WORDS = 8 * sizeof(T) / 16;   // of 16 bytes a run
    uint4 raw[V / 8][WORDS];

    __device__ void load(const T* x, uint32_t c0, uint32_t end) {
        const uint32_t c = c0 + threadIdx.x * 8;
        if (c0 + 256 * V <= end) {   // the loads of all runs are on their way at once
#pragma unroll
            for (int j = 0; j < V / 8; ++j) __builtin_memcpy(raw[j], x + c + j * 2048, sizeof(raw[j]));
        } else {
#pragma unroll
            for (int j = 0; j < V / 8; ++j) {
                if (c + j * 2048 + 8 <= end) {
                    __builtin_memcpy(raw[j], x + c + j * 2048, sizeof(raw[j]));
                } else {
                    T part[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) part[i] = c + j * 2048 + i < end ? x[c + j * 2048 + i] : (T)MINUS_INF;
                    __builtin_memcpy(raw[j], part, sizeof(raw[j]));
                }
            }
        }
    }
    __device__ void values(float (&v)[V]) const {
#pragma unroll
        for (int j = 0; j < V / 8; ++j) {
            T part[8];
            __builtin_memcpy(part, raw[j], sizeof(part));
#pragma unroll
            for (int i = 0; i < 8; ++i) v[j * 8 + i] = (float)part[i];
        }
    }
};

// A workgroup takes a segment of a row, 256 * V entries at a time.  (Loading the next ones ahead gained nothing: 2048 x 32000 bf16 without
// alternatives 33.8 -> 35.5 us; 8 workgroups a CU have enough loads on their way.)  Bound by the vector ALU, an exponential and a test against the
// bound for every entry: 2048 x 32000 with 10 alternatives 40.7 us in bf16 (3.2 TB/s), 58.3 in fp32 (4.5 TB/s).
template <typename T, int V>
__global__ __launch_bounds__(256) void token_logprobs_kernel(LogprobArgs g) {
    __shared__ uint64_t pools[4][POOL], finals[4 * POOL + 8];
    __shared__ Totals totals;
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint64_t w = blockIdx.x, row = w / g.splits;
    const uint32_t begin = (uint32_t)(w % g.splits) * g.segment;
    const uint32_t end = g.vocab - begin < g.segment ? g.vocab : begin + g.segment;
    const T* x = (const T*)g.logits + row * g.stride;
    const auto column = [&](uint32_t c0, int i) { return c0 + (i / 8 * 256 + threadIdx.x) * 8 + i % 8; };
    Sums z{MINUS_INF, 0.f, 0.f};
    Pool pool{pools[wave]};
    for (uint32_t c0 = begin; c0 < end; c0 += 256 * V) {
        float v[V];
        Entries<T, V> entries;
        entries.load(x, c0, end);
        entries.values(v);
        float peaks[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            peaks[q] = v[q * (V / 4)];
#pragma unroll
            for (int i = 1; i < V / 4; ++i) peaks[q] = fmaxf(peaks[q], v[q * (V / 4) + i]);
        }
        const float peak = fmaxf(fmaxf(peaks[0], peaks[1]), fmaxf(peaks[2], peaks[3])), m = fmaxf(z.m, peak);
        const float base = m == MINUS_INF ? 0.f : m;
        z = join(z, Sums{m, 0.f, 0.f});
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float d = v[i] - base, e = exp_of(d);
            z.s += e;
            z.t = fmaf(e, fmaxf(d, -1000.f), z.t);   // an entry of -inf adds 0, not 0 * inf; e^-1000 is 0 as well
        }
        if (!g.n_top) continue;
        const uint32_t orders[4] = {order_of(peaks[0]), order_of(peaks[1]), order_of(peaks[2]), order_of(peaks[3])};
        if (!pool.raise<true>(orders, g.n_top)) continue;
        const float from = value_of(max(pool.bound, ORDER_FLOOR + 1));   // floats compare as their orders do
        uint32_t n = V * __popcll(__ballot(peak >= from));   // at most, and counted where that is too many
        if (pool.count + n > POOL) {
            n = 0;
#pragma unroll
            for (int i = 0; i < V; ++i) n += __popcll(__ballot(v[i] >= from));
        }
        if (pool.count + n <= POOL) {
#pragma unroll
            for (int i = 0; i < V; ++i) pool.add(v[i] >= from, key_of(order_of(v[i]), column(c0, i)));
            wave_sync();
        } else {   // equal entries, or one lane's above all others: from memory again, with room made on the way
#pragma unroll 1
            for (int i = 0; i < V; ++i) {
                const uint32_t c = column(c0, i);
                const uint32_t order = c < end ? order_of((float)x[c]) : 0;
                if (pool.count > POOL - 64) pool.compress(g.n_top, lane);
                pool.add(order >= max(pool.bound, ORDER_FLOOR + 1), key_of(order, c));
                wave_sync();
            }
        }
    }
    finish<T>(g, row, z, pool, pools[0], finals, totals, g.splits == 1 ? ~0ull : w);
}

// Joins the segments' parts of a row.  Bound by latency: 5 of the 10.1 us of 8 x 50257 in fp32.
template <typename T>
__global__ __launch_bounds__(256) void join_logprobs_kernel(LogprobArgs g) {
    __shared__ uint64_t pools[4][POOL], finals[4 * POOL + 8];
    __shared__ Totals totals;
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint64_t row = blockIdx.x;
    Sums z{MINUS_INF, 0.f, 0.f};
    const float* sums = g.part_sums + 3 * row * g.splits;
    for (uint32_t i = threadIdx.x; i < g.splits; i += 256) z = join(z, Sums{sums[3 * i], sums[3 * i + 1], sums[3 * i + 2]});
    Pool pool{pools[wave]};
    const uint64_t* keys = g.part_keys + row * g.splits * g.n_top;
    const uint32_t n = g.splits * g.n_top;
    for (uint32_t i = wave * 64; i < n; i += 256) {
        const uint64_t key = i + lane < n ? keys[i + lane] : 0;
        const uint32_t order = (uint32_t)(key >> 32), orders[4] = {order, 0, 0, 0};
        if (!pool.raise<true>(orders, g.n_top)) continue;
        if (pool.count > POOL - 64) pool.compress(g.n_top, lane);
        pool.add(order >= max(pool.bound, ORDER_FLOOR + 1), key);
        wave_sync();
    }
    finish<T>(g, row, z, pool, pools[0], finals, totals, ~0ull);
}

// A row's sums over its groups, its outputs but for the alternatives, and the groups these are among: the n_top with the largest logits,
// ties to the first.  (Each of those has an entry that beats whatever is in another group, or equals it and comes first.)
__global__ __launch_bounds__(256) void head_rows_kernel(HeadArgs h) {
    __shared__ uint64_t pools[4][POOL], finals[4 * POOL + 8];
    __shared__ Totals totals;
    __shared__ int dots[4];
    const LogprobArgs& g = h.outputs;
    const MatmulArgs& p = h.product;
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint64_t row = blockIdx.x;
    const float4* sums = h.sums + row * h.groups;
    float4 next = threadIdx.x < h.groups ? sums[threadIdx.x] : make_float4(MINUS_INF, 0.f, 0.f, 0.f);
    // the token's logit
    const uint32_t token = g.tokens ? g.tokens[row] : NONE;
    int dot = 0;
    float scale = 0.f;
    if (token < g.vocab) {
        scale = p.sa[row] * p.sb[token];
        const int8_t *a = p.a + row * p.lda, *b = p.b + token * p.ldb;
        for (uint32_t c = threadIdx.x * 16; c < p.k; c += 4096) {
            const v4i x = *(const v4i*)(a + c), y = *(const v4i*)(b + c);
#pragma unroll
            for (int i = 0; i < 4; ++i) dot = __builtin_amdgcn_sdot4(x[i], y[i], dot, false);
        }
    }
#pragma unroll
    for (int o = 1; o < 64; o *= 2) dot += __shfl_xor(dot, o);
    if (lane == 0) dots[wave] = dot;
    Sums z{MINUS_INF, 0.f, 0.f};
    Pool pool{pools[wave]};
    for (uint32_t i = wave * 64; i < h.groups; i += 256) {
        const float4 v = next;
        next = i + 256 + lane < h.groups ? sums[i + 256 + lane] : make_float4(MINUS_INF, 0.f, 0.f, 0.f);
        z = join(z, Sums{v.x, v.y, v.z});
        if (!h.n_top) continue;
        const uint32_t order = order_of(v.x), orders[4] = {order, 0, 0, 0};
        if (!pool.raise<true>(orders, h.n_top)) continue;
        if (pool.count > POOL - 64) pool.compress(h.n_top, lane);
        pool.add(order >= max(pool.bound, ORDER_FLOOR + 1), key_of(order, i + lane));
        wave_sync();
    }
    z = row_total(z, pool, totals);
    const float log_s = logf(z.s);
    if (threadIdx.x == 0) {
        write_row(g, row, token, z, log_s, (float)(dots[0] + dots[1] + dots[2] + dots[3]) * scale);
        h.totals[row] = make_float2(z.m, log_s);
    }
    if (!h.n_top) return;
    rank_best(h.n_top, pool, pools[0], finals, totals, [&](uint32_t place, uint64_t key) {
        const uint32_t group = ~(uint32_t)key, entry = (uint32_t)(row * h.n_top + place);
        h.picked[entry] = key ? group : NONE;
    });
}

// A workgroup a group: who picked it.  (With a counter per group and an entry written by whoever picks it the counters of groups that many
// rows pick decide the time: head_rows_kernel took 28 us for 4096 rows with 5 of 250
// groups each, now 13.5 and this kernel 9.7; 14.4 where all rows pick the same groups.)
__global__ __launch_bounds__(256) void head_lists_kernel(HeadArgs h) {
    constexpr uint32_t AHEAD = 8;
    __shared__ uint32_t count;
    const uint32_t group = blockIdx.x, lane = threadIdx.x & 63, all = (uint32_t)h.product.m * h.n_top;
    uint32_t* list = h.lists + (uint64_t)group * h.product.m;
    if (threadIdx.x == 0) count = 0;
    __syncthreads();
    for (uint32_t i = threadIdx.x; i - threadIdx.x < all; i += 256 * AHEAD) {
        uint32_t picked[AHEAD];
#pragma unroll
        for (uint32_t u = 0; u < AHEAD; ++u) picked[u] = i + 256 * u < all ? h.picked[i + 256 * u] : NONE;
#pragma unroll
        for (uint32_t u = 0; u < AHEAD; ++u) {
            const uint64_t mine = __ballot(picked[u] == group);
            if (!mine) continue;
            uint32_t at = 0;
            if (lane == 0) at = atomicAdd(&count, (uint32_t)__popcll(mine));
            at = __builtin_amdgcn_readfirstlane((int)at);
            if (picked[u] == group)
                list[at + __builtin_amdgcn_mbcnt_hi((uint32_t)(mine >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mine, 0))] = i + 256 * u;
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) h.counts[group] = count;
}

// The best entries of a row's picked groups.  4096 rows of 5 groups: 10.7 us.
__global__ __launch_bounds__(256) void head_best_kernel(HeadArgs h) {
    __shared__ uint64_t pools[4][POOL], finals[4 * POOL + 8];
    __shared__ Totals totals;
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint64_t row = blockIdx.x;
    Pool pool{pools[wave]};
    const uint32_t entries = h.n_top * HEAD_GROUP;
    for (uint32_t i = wave * 64; i < entries; i += 1024) {   // four times 64 entries of one group each
        uint32_t group[4], orders[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) group[j] = i + 256 * j < entries ? h.picked[row * h.n_top + (i + 256 * j) / HEAD_GROUP] : NONE;
#pragma unroll
        for (int j = 0; j < 4; ++j) orders[j] = group[j] != NONE ? order_of(h.logits[row * entries + i + 256 * j + lane]) : 0;
        if (!pool.raise<false>(orders, h.n_top)) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (pool.count > POOL - 64) pool.compress(h.n_top, lane);
            pool.add(orders[j] >= max(pool.bound, ORDER_FLOOR + 1), key_of(orders[j], group[j] * HEAD_GROUP + (i + 256 * j) % HEAD_GROUP + lane));
            wave_sync();
        }
    }
    row_total(Sums{MINUS_INF, 0.f, 0.f}, pool, totals);
    const float2 total = h.totals[row];
    rank_best(h.n_top, pool, pools[0], finals, totals,
              [&](uint32_t place, uint64_t key) { write_place(h.outputs, row, place, key, total.x, total.y); });
}

template <typename T>
hipError_t launch_rows(const LogprobArgs& g, hipStream_t stream) {
    const dim3 grid((uint32_t)(g.rows * g.splits));
    if (g.segment <= 2048) token_logprobs_kernel<T, 8><<<grid, dim3(256), 0, stream>>>(g);
    else token_logprobs_kernel<T, 16><<<grid, dim3(256), 0, stream>>>(g);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_type(const LogprobArgs& g, hipStream_t stream) {
    hipError_t e = hipSuccess;
    if (g.splits == 1) {   // any number of rows
        in_launches(g.rows, 1, 256, [&](uint64_t first, uint64_t n, uint32_t) {
            LogprobArgs part = g;
            part.rows = n;
            part.logits = (const T*)g.logits + first * g.stride;
            if (g.tokens) part.tokens = g.tokens + first;
            if (g.logprobs) part.logprobs = g.logprobs + first;
            if (g.entropy) part.entropy = g.entropy + first;
            if (g.n_top) part.top_ids = g.top_ids + first * g.n_top;
            if (g.n_top) part.top_logprobs = g.top_logprobs + first * g.n_top;
            if (e == hipSuccess) e = launch_rows<T>(part, stream);
        });
        return e;
    }
    e = launch_rows<T>(g, stream);   // fewer than 1024 rows (logprob_plan)
    if (e != hipSuccess) return e;
    join_logprobs_kernel<T><<<dim3((uint32_t)g.rows), dim3(256), 0, stream>>>(g);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_token_logprobs(LogprobArgs g, uint32_t dtype, const LogprobPlan& p, void* workspace, hipStream_t stream) {
    if (g.rows == 0) return hipSuccess;
    g.splits = p.splits;
    g.segment = p.segment;
    g.part_sums = (float*)workspace;
    g.part_keys = (uint64_t*)((char*)workspace + p.sums_bytes);
    if (dtype == TYPE_F16) return launch_type<f16_t>(g, stream);
    if (dtype == TYPE_BF16) return launch_type<bf16_t>(g, stream);
    return launch_type<float>(g, stream);
}

hipError_t launch_head_rows(const HeadArgs& h, hipStream_t stream) {
    head_rows_kernel<<<dim3((uint32_t)h.product.m), dim3(256), 0, stream>>>(h);
    return hipGetLastError();
}

hipError_t launch_head_lists(const HeadArgs& h, hipStream_t stream) {
    head_lists_kernel<<<dim3(h.groups), dim3(256), 0, stream>>>(h);
    return hipGetLastError();
}

hipError_t launch_head_best(const HeadArgs& h, hipStream_t stream) {
    head_best_kernel<<<dim3((uint32_t)h.product.m), dim3(256), 0, stream>>>(h);
    return hipGetLastError();
}

}  // namespace dessert
