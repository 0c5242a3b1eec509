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
__device__ inline uint64_t key_of(float x, uint32_t col) {
    uint32_t u = __float_as_uint(x + 0.f);
    u = u & 0x80000000u ? ~u : u | 0x80000000u;
    return (uint64_t)u << 32 | (uint32_t)~col;
}
__device__ inline float key_value(uint64_t key) {
    const uint32_t u = (uint32_t)(key >> 32);
    return __uint_as_float(u & 0x80000000u ? u & 0x7FFFFFFFu : ~u);
}
constexpr uint64_t KEY_FLOOR = (uint64_t)0x007FFFFFu << 32 | 0xFFFFFFFFu;   // an entry of -inf: no key up to this one is an alternative

// The wave's list: lane j holds the j-th largest key.
__device__ inline void insert(uint64_t& list, uint64_t key, uint32_t lane) {
    const uint32_t at = __popcll(__ballot(list > key));
    const uint64_t left = __shfl_up(list, 1);
    if (lane == at) list = key;
    else if (lane > at) list = left;
}
// Offer one key a lane; the list's entry at n_top - 1 is the threshold.
__device__ inline void offer(uint64_t& list, uint64_t key, uint32_t n_top, uint32_t lane) {
    uint64_t least = __shfl(list, (int)n_top - 1);
    if (least < KEY_FLOOR) least = KEY_FLOOR;
    uint64_t want = __ballot(key > least);
    while (want) {
        const int from = __ffsll((unsigned long long)want) - 1;
        const uint64_t k = __shfl(key, from);
        if (lane == (uint32_t)from) key = 0;
        insert(list, k, lane);
        least = __shfl(list, (int)n_top - 1);
        if (least < KEY_FLOOR) least = KEY_FLOOR;
        want = __ballot(key > least);
    }
}

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
        g.top_logprobs[row * g.n_top + lane] = nan ? z.s : some ? (key_value(list) - z.m) - log_s : MINUS_INF;
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
        uint64_t list = 0;
        for (uint32_t c0 = begin; c0 < end; c0 += 256 * V) {
            float v[V];
            float peak = MINUS_INF;
#pragma unroll
            for (int j = 0; j < V / RUN; ++j) {
                const uint32_t c = c0 + (j * 256 + threadIdx.x) * RUN;
                float part[RUN];
                if (c + RUN <= end) load_run<T, RUN>(x + c, part);
                else
#pragma unroll
                    for (int i = 0; i < RUN; ++i) part[i] = c + i < end ? (float)x[c + i] : MINUS_INF;
#pragma unroll
                for (int i = 0; i < RUN; ++i) {
                    v[j * RUN + i] = part[i];
                    peak = fmaxf(peak, part[i]);
                }
            }
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
                z.t += e * fmaxf(d, -3.4e38f);   // an entry of -inf adds 0, not 0 * inf
            }
            if (g.n_top) {
#pragma unroll
                for (int i = 0; i < V; ++i)
                    offer(list, key_of(v[i], c0 + ((i / RUN) * 256 + threadIdx.x) * RUN + i % RUN), g.n_top, lane);
            }
        }
#pragma unroll
        for (int o = 1; o < 64; o *= 2) z = join(z, Sums{__shfl_xor(z.m, o), __shfl_xor(z.s, o), __shfl_xor(z.t, o)});
        __syncthreads();
        if (lane == 0) s_sums[wave] = z;
        s_list[wave][lane] = list;
        __syncthreads();
        if (wave == 0) {
            for (int o = 1; o < 4; ++o) {
                z = join(z, s_sums[o]);
                if (g.n_top) offer(list, lane < g.n_top ? s_list[o][lane] : 0, g.n_top, lane);
            }
            if (g.splits == 1) {
                finish(g, row, z, given_logit<T>(g, row), list, lane);
            } else {
                if (lane == 0) {
                    g.part_sums[3 * w] = z.m;
                    g.part_sums[3 * w + 1] = z.s;
                    g.part_sums[3 * w + 2] = z.t;
                }
                if (lane < g.n_top) g.part_keys[w * g.n_top + lane] = list;
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
        uint64_t list = 0;
        const uint64_t* keys = g.part_keys + row * g.splits * g.n_top;
        for (uint32_t i = 0; i < g.splits * g.n_top; i += 64)
            offer(list, i + lane < g.splits * g.n_top ? keys[i + lane] : 0, g.n_top, lane);
        finish(g, row, z, given_logit<T>(g, row), list, lane);
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
