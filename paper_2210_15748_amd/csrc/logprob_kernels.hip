// Log probabilities of given tokens, the entropy and the best alternatives of rows of logits, in one pass over the logits.
// With m = max_j l_j, s = sum_j e^(l_j - m) and t = sum_j e^(l_j - m) (l_j - m):
//     log p(token) = (l_token - m) - log s,    entropy = log s - t / s,
// and two parts of a row join by moving both to the larger m: s' = e^d s, t' = e^d (t + d s) with d = m - m'.
// Entries of -inf have no probability and are never an alternative; a row with +inf or NaN has s = NaN and gives NaN.
#include "kernels.hpp"
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

    // The n_top largest of `count` keys, sorted: a key's place is the number of larger ones (no two are equal).
    __device__ void compress(uint32_t n_top, uint32_t lane) {
        uint64_t mine[POOL / 64];
        uint32_t place[POOL / 64];
#pragma unroll
        for (uint32_t j = 0; j < POOL / 64; ++j) {
            mine[j] = j * 64 + lane < count ? keys[j * 64 + lane] : 0;
            place[j] = 0;
        }
        for (uint32_t i = 0; i < count; ++i) {
            const uint64_t k = keys[i];
#pragma unroll
            for (uint32_t j = 0; j < POOL / 64; ++j) place[j] += k > mine[j];
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
    __device__ void add(bool want, uint64_t key, uint32_t n_top, uint32_t lane) {
        const uint64_t all = __ballot(want);
        if (!all) return;
        if (count > POOL - 64) compress(n_top, lane);
        if (want) keys[count + __builtin_amdgcn_mbcnt_hi((uint32_t)(all >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)all, 0))] = key;
        count += __popcll(all);
        wave_sync();
    }
    // `peak`: the order of the largest entry of each lane.  The n_top-th largest of the 64 peaks bounds the n_top-th largest entry from
    // below; its upper 18 bits, by bisection, leave in little more than n_top entries of a wave's.
    __device__ bool raise(uint32_t peak, uint32_t n_top) {
        if (!__ballot(peak > bound)) return false;
        uint32_t b = 0;
#pragma unroll
        for (int bit = 31; bit >= 14; --bit) {
            const uint32_t t = b | 1u << bit;
            if ((uint32_t)__popcll(__ballot(peak >= t)) >= n_top) b = t;
        }
        bound = max(bound, b);
        return true;
    }
};

// The best n_top of the four waves' pools and the row's sums, to the outputs (or, of a part of a row, to the parts).  `finals` and `totals`
// are the workgroup's; all 256 threads take part.
struct Totals {
    Sums sums[4];
    uint32_t bound[4], count;
};
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

template <typename T>
__device__ inline void finish(const LogprobArgs& g, uint64_t row, Sums z, Pool& pool, uint64_t* finals, Totals& totals, uint64_t part) {
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    z = wave_total(z);
    if (lane == 0) {
        totals.sums[wave] = z;
        totals.bound[wave] = pool.bound;
        if (wave == 0) totals.count = 0;
    }
    __syncthreads();
    z = join(join(totals.sums[0], totals.sums[1]), join(totals.sums[2], totals.sums[3]));
    const bool whole = part == ~0ull, nan = z.s != z.s, empty = z.s == 0.f;
    const float log_s = logf(z.s);
    if (threadIdx.x == 0) {
        if (!whole) {
            g.part_sums[3 * part] = z.m;
            g.part_sums[3 * part + 1] = z.s;
            g.part_sums[3 * part + 2] = z.t;
        } else {
            if (g.entropy) g.entropy[row] = empty ? 0.f : log_s - z.t / z.s;
            if (g.tokens) {
                const uint32_t token = g.tokens[row];
                float lp = nan ? z.s : MINUS_INF;
                if (!nan && !empty && token < g.vocab) lp = ((float)((const T*)g.logits)[row * g.stride + token] - z.m) - log_s;
                g.logprobs[row] = token == NONE ? 0.f : lp;
            }
        }
    }
    if (!g.n_top) return;
    const uint32_t bound = max(max(totals.bound[0], totals.bound[1]), max(totals.bound[2], totals.bound[3]));
    for (uint32_t i = lane; i < pool.count; i += 64)
        if ((uint32_t)(pool.keys[i] >> 32) >= bound) finals[atomicAdd(&totals.count, 1u)] = pool.keys[i];
    __syncthreads();
    const uint32_t count = totals.count;
    for (uint32_t j = threadIdx.x; j < max(count, g.n_top); j += 256) {
        const uint64_t mine = j < count ? finals[j] : 0;
        uint32_t place = j;   // behind the last key: an unused slot
        if (j < count) {
            place = 0;
            for (uint32_t i = 0; i < count; ++i) place += finals[i] > mine;
        }
        if (place >= g.n_top) continue;
        if (!whole) {
            g.part_keys[part * g.n_top + place] = mine;
        } else {
            const bool some = mine && !nan;
            g.top_ids[row * g.n_top + place] = some ? ~(uint32_t)mine : NONE;
            g.top_logprobs[row * g.n_top + place] = nan ? z.s : some ? (value_of((uint32_t)(mine >> 32)) - z.m) - log_s : MINUS_INF;
        }
    }
}

// A workgroup takes a segment of a row, 256 * V entries at a time.
template <typename T, int V>
__global__ __launch_bounds__(256) void token_logprobs_kernel(LogprobArgs g) {
    constexpr int RUN = 8;
    __shared__ uint64_t pools[4][POOL], finals[4 * POOL];
    __shared__ Totals totals;
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint64_t w = blockIdx.x, row = w / g.splits;
    const uint32_t begin = (uint32_t)(w % g.splits) * g.segment;
    const uint32_t end = g.vocab - begin < g.segment ? g.vocab : begin + g.segment;
    const T* x = (const T*)g.logits + row * g.stride;
    Sums z{MINUS_INF, 0.f, 0.f};
    Pool pool{pools[wave]};
    for (uint32_t c0 = begin; c0 < end; c0 += 256 * V) {
        float v[V];
        if (c0 + 256 * V <= end) {   // the loads of all runs are on their way at once
#pragma unroll
            for (int j = 0; j < V / RUN; ++j) load_run<T, RUN>(x + c0 + (j * 256 + threadIdx.x) * RUN, *(float(*)[RUN])(v + j * RUN));
        } else {
#pragma unroll
            for (int j = 0; j < V / RUN; ++j) {
                const uint32_t c = c0 + (j * 256 + threadIdx.x) * RUN;
                float part[RUN];
                if (c + RUN <= end) load_run<T, RUN>(x + c, part);
                else
#pragma unroll
                    for (int i = 0; i < RUN; ++i) part[i] = c + i < end ? (float)x[c + i] : MINUS_INF;
#pragma unroll
                for (int i = 0; i < RUN; ++i) v[j * RUN + i] = part[i];
            }
        }
        float peak = MINUS_INF;
#pragma unroll
        for (int i = 0; i < V; ++i) peak = fmaxf(peak, v[i]);
        const float m = fmaxf(z.m, peak);
        const float base = m == MINUS_INF ? 0.f : m;
        z = join(z, Sums{m, 0.f, 0.f});
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float d = v[i] - base, e = exp_of(d);
            z.s += e;
            z.t = fmaf(e, fmaxf(d, -1000.f), z.t);   // an entry of -inf adds 0, not 0 * inf; e^-1000 is 0 as well
        }
        if (g.n_top && pool.raise(order_of(peak), g.n_top)) {
#pragma unroll
            for (int i = 0; i < V; ++i)   // floats compare as their orders do
                pool.add(v[i] >= value_of(max(pool.bound, ORDER_FLOOR + 1)), key_of(order_of(v[i]), c0 + ((i / RUN) * 256 + threadIdx.x) * RUN + i % RUN), g.n_top, lane);
        }
    }
    finish<T>(g, row, z, pool, finals, totals, g.splits == 1 ? ~0ull : w);
}

// Joins the segments' parts of a row.
template <typename T>
__global__ __launch_bounds__(256) void join_logprobs_kernel(LogprobArgs g) {
    __shared__ uint64_t pools[4][POOL], finals[4 * POOL];
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
        if (pool.raise((uint32_t)(key >> 32), g.n_top)) pool.add(key && (uint32_t)(key >> 32) >= pool.bound, key, g.n_top, lane);
    }
    finish<T>(g, row, z, pool, finals, totals, ~0ull);
}

template <typename T>
hipError_t launch_type(const LogprobArgs& g, hipStream_t stream) {
    const dim3 grid((uint32_t)(g.rows * g.splits));
    if (g.segment <= 2048) token_logprobs_kernel<T, 8><<<grid, dim3(256), 0, stream>>>(g);
    else token_logprobs_kernel<T, 32><<<grid, dim3(256), 0, stream>>>(g);
    if (g.splits > 1) {
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        join_logprobs_kernel<T><<<dim3((uint32_t)g.rows), dim3(256), 0, stream>>>(g);
    }
    return hipGetLastError();
}

}  // namespace

LogprobPlan logprob_plan(uint64_t rows, uint32_t vocab, uint32_t n_top) {
    LogprobPlan p{};
    if (rows >= 1024 || vocab <= 2048) {
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

}  // namespace dessert
