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
constexpr uint64_t KEY_FLOOR = (uint64_t)ORDER_FLOOR << 32 | 0xFFFFFFFFu;

__device__ inline uint64_t read_lane(uint64_t v, uint32_t lane) {
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), (int)lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, (int)lane);
}

// A wave's list of the best entries it has seen: lane j holds the j-th largest key, 0 where there is none.
struct Best {
    uint64_t list = 0, least = KEY_FLOOR;   // least: what a key has to beat, list[n_top - 1] or the floor

    // One key, the same in all lanes, that beats `least`.
    __device__ void insert(uint64_t key, uint32_t n_top, uint32_t lane) {
        const uint32_t at = __popcll(__ballot(list > key));
        // the neighbour's entry: the whole wave moves up by one lane
        const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(list >> 32), 0x138, 0xF, 0xF, false);
        const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)list, 0x138, 0xF, 0xF, false);
        if (lane == at) list = key;
        else if (lane > at) list = (uint64_t)hi << 32 | lo;
        const uint64_t last = read_lane(list, n_top - 1);
        least = last > KEY_FLOOR ? last : KEY_FLOOR;
    }
    // A key from every lane.
    __device__ void offer(uint64_t key, uint32_t n_top, uint32_t lane) {
        uint64_t want = __ballot(key > least);
        while (want) {
            const uint32_t from = __ffsll((unsigned long long)want) - 1;
            insert(read_lane(key, from), n_top, lane);
            want &= want - 1;
            want &= __ballot(key > least);
        }
    }
    // V values from every lane, `peak` the largest of a lane's; col(i) the column of value i.  An entry can be among the n_top best
    // only if it is not below the n_top-th largest of the 64 peaks: that bound (its upper 18 bits, by bisection) leaves little more
    // than n_top values to insert, where an empty list would let in n_top * ln(64 V / n_top) more.
    template <int V, typename Col>
    __device__ void offer_all(const float (&v)[V], float peak, uint32_t n_top, uint32_t lane, Col col) {
        const uint32_t top = order_of(peak);
        if (!__ballot(top >= (uint32_t)(least >> 32))) return;
        uint32_t bound = 0;
#pragma unroll
        for (int bit = 31; bit >= 14; --bit) {
            const uint32_t t = bound | 1u << bit;
            if ((uint32_t)__popcll(__ballot(top >= t)) >= n_top) bound = t;
        }
        const uint32_t floor = (uint32_t)(least >> 32);
        if (bound < floor) bound = floor;
        const float from = value_of(bound);   // compared as floats: no order to be formed for entries that are out
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (__ballot(v[i] >= from)) offer(v[i] >= from ? key_of(order_of(v[i]), col(i)) : 0, n_top, lane);
    }
};

__device__ inline void finish(const LogprobArgs& g, uint64_t row, Sums z, float given, uint64_t list, uint32_t lane) {
    const float log_s = logf(z.s);
    const bool nan = z.s != z.s, empty = z.s == 0.f;
    if (lane == 0) {
        if (g.entropy) g.entropy[row] = empty ? 0.f : log_s - z.t / z.s;
        if (g.tokens) {
            const uint32_t token = g.tokens[row];
            float lp = nan ? z.s : token >= g.vocab || empty ? MINUS_INF : (given - z.m) - log_s;
            g.logprobs[row] = token == NONE ? 0.f : lp;
        }
    }
    if (lane < g.n_top) {
        const bool some = list > KEY_FLOOR && !nan;
        g.top_ids[row * g.n_top + lane] = some ? ~(uint32_t)list : NONE;
        g.top_logprobs[row * g.n_top + lane] = nan ? z.s : some ? (value_of((uint32_t)(list >> 32)) - z.m) - log_s : MINUS_INF;
    }
}

template <typename T>
__device__ inline float given_logit(const LogprobArgs& g, uint64_t row) {
    if (!g.tokens) return 0.f;
    const uint32_t token = g.tokens[row];
    return token < g.vocab ? (float)((const T*)g.logits)[row * g.stride + token] : 0.f;
}

// A workgroup takes a segment of a row, 256 * V entries at a time.
template <typename T, int V>
__global__ __launch_bounds__(256) void token_logprobs_kernel(LogprobArgs g) {
    constexpr int RUN = 8;
    __shared__ uint64_t s_list[4][64];
    __shared__ Sums s_sums[4];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (uint64_t w = blockIdx.x; w < g.rows * g.splits; w += gridDim.x) {
        const uint64_t row = w / g.splits;
        const uint32_t split = (uint32_t)(w % g.splits);
        const uint32_t begin = split * g.segment;
        const uint32_t end = g.vocab - begin < g.segment ? g.vocab : begin + g.segment;
        const T* x = (const T*)g.logits + row * g.stride;
        Sums z{MINUS_INF, 0.f, 0.f};
        Best best;
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
            if (z.m != MINUS_INF) {
                const float d = z.m - base, e = exp_of(d);
                z.t = e == 0.f ? 0.f : e * (z.t + d * z.s);
                z.s *= e;
            }
            z.m = m;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float d = v[i] - base, e = exp_of(d);
                z.s += e;
                z.t = fmaf(e, fmaxf(d, -1000.f), z.t);   // an entry of -inf adds 0, not 0 * inf; e^-1000 is 0 as well
            }
            if (g.n_top)
                best.offer_all<V>(v, peak, g.n_top, lane,
                                  [&](int i) { return c0 + ((i / RUN) * 256 + threadIdx.x) * RUN + i % RUN; });
        }
#pragma unroll
        for (int o = 1; o < 64; o *= 2) z = join(z, Sums{__shfl_xor(z.m, o), __shfl_xor(z.s, o), __shfl_xor(z.t, o)});
        __syncthreads();
        if (lane == 0) s_sums[wave] = z;
        s_list[wave][lane] = best.list;
        __syncthreads();
        if (wave == 0) {
            for (int o = 1; o < 4; ++o) {
                z = join(z, s_sums[o]);
                if (g.n_top) best.offer(lane < g.n_top ? s_list[o][lane] : 0, g.n_top, lane);
            }
            if (g.splits == 1) {
                finish(g, row, z, given_logit<T>(g, row), best.list, lane);
            } else {
                if (lane == 0) {
                    g.part_sums[3 * w] = z.m;
                    g.part_sums[3 * w + 1] = z.s;
                    g.part_sums[3 * w + 2] = z.t;
                }
                if (lane < g.n_top) g.part_keys[w * g.n_top + lane] = best.list;
            }
        }
        __syncthreads();
    }
}

// One wave a row joins the segments' parts.
template <typename T>
__global__ __launch_bounds__(64) void join_logprobs_kernel(LogprobArgs g) {
    const uint32_t lane = threadIdx.x;
    for (uint64_t row = blockIdx.x; row < g.rows; row += gridDim.x) {
        Sums z{MINUS_INF, 0.f, 0.f};
        const float* sums = g.part_sums + 3 * row * g.splits;
        for (uint32_t i = lane; i < g.splits; i += 64) z = join(z, Sums{sums[3 * i], sums[3 * i + 1], sums[3 * i + 2]});
#pragma unroll
        for (int o = 1; o < 64; o *= 2) z = join(z, Sums{__shfl_xor(z.m, o), __shfl_xor(z.s, o), __shfl_xor(z.t, o)});
        Best best;
        const uint64_t* keys = g.part_keys + row * g.splits * g.n_top;
        for (uint32_t i = 0; i < g.splits * g.n_top; i += 64)
            best.offer(i + lane < g.splits * g.n_top ? keys[i + lane] : 0, g.n_top, lane);
        finish(g, row, z, given_logit<T>(g, row), best.list, lane);
    }
}

template <typename T>
hipError_t launch_type(const LogprobArgs& g, hipStream_t stream) {
    const uint64_t work = g.rows * g.splits, most = 1u << 20;
    const dim3 grid((uint32_t)(work < most ? work : most));
    if (g.segment <= 2048) token_logprobs_kernel<T, 8><<<grid, dim3(256), 0, stream>>>(g);
    else token_logprobs_kernel<T, 32><<<grid, dim3(256), 0, stream>>>(g);
    if (g.splits > 1) {
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        join_logprobs_kernel<T><<<dim3((uint32_t)(g.rows < most ? g.rows : most)), dim3(64), 0, stream>>>(g);
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
