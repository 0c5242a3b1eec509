// int8 x int8 products with a scale for each token (row of a) and each channel (row of b):
//     out[i][j] = T( float(sum_c a[i][c] * b[j][c]) * (sa[i] * sb[j]) + bias[j] )
// The sums are exact in int32 whatever their order, so any split of the columns gives the same bits.  Both operands lie with
// their columns side by side, which is the order that v_mfma_i32_16x16x64_i8 takes: 16 bytes of one row per lane.
#include <algorithm>
#include <type_traits>

#include "kernels.hpp"
#include "launch_slices.hpp"
#include "number_formats.hpp"

namespace dessert {

namespace {

[[maybe_unused]] constexpr int LINE = 128;   // bytes

// ---- tiles ------------------------------------------------------------------------------------------------------------------
// A workgroup of WM x WN waves goes through tiles of TM tokens x TN channels, STEP columns a step.  A step's rows lie in LDS,
// double-buffered: while the waves multiply one step, the next one is on its way, across the border between two tiles
// too, so that a tile's results leave while the next tile's first columns arrive.  Rows at whole 4 bytes (DIRECT) go from memory to LDS
// directly, others through registers: 203 x 50021 x 1028 48 us through registers, 32 directly, x 1029 54.
//
// The buffers are four arrays by name and the two steps of a round stand one after the other in the code: the compiler then knows
// that reads of one buffer do not wait for what is arriving in the other.  The products appear once per buffer and nowhere else
// (no tail outside the loop): a second copy of the accumulators would not fit the registers.
template <int TM_, int TN_, int WM_, int WN_, int STEP_, bool DIRECT_, bool WORDS_ = true>
struct Tile {
    static constexpr int TM = TM_, TN = TN_, WM = WM_, WN = WN_, STEP = STEP_;
    static constexpr bool DIRECT = DIRECT_;
    static constexpr bool WORDS = WORDS_;                        // the columns may end within a 16-byte part, at whole 4 bytes
    static constexpr int W = WM * WN;
    static constexpr int FM = TM / WM / 16, FQ = TN / WN / 64;   // a wave's fragments: of 16 tokens, and 4 x 16 channels
    static constexpr int PARTS = STEP / 16, ROWS = 64 / PARTS;   // 16-byte parts of a row; rows in a piece of 1 KB, which a wave fetches at a time
    static constexpr int LA = TM / ROWS / W, LB = TN / ROWS / W; // pieces that a wave fetches per step
};

#if defined(__HIP_DEVICE_COMPILE__)
// 16 bytes of a row from column c on; columns from k on read as zero, k < 16.
__device__ inline v4i load_few(const int8_t* row, uint32_t c, uint32_t k) {
    uint64_t lo = 0, hi = 0;
#pragma unroll 1
    for (uint32_t i = c; i < k; ++i) {
        const uint64_t byte = (uint8_t)row[i];
        if (i - c < 8) lo |= byte << 8 * (i - c);
        else hi |= byte << 8 * (i - c - 8);
    }
    const v4i v = {(int)lo, (int)(lo >> 32), (int)hi, (int)(hi >> 32)};
    return v;
}

// Where a part of 16 columns from c on would pass the columns' end, the last 16 are read instead, of tokens and channels alike (the sum does not
// mind the order); of the tokens' the first `seen`, which an earlier part has, become zeros.
__device__ inline v4i unseen(v4i v, uint32_t seen) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int bytes = (int)seen - 4 * i;
        v[i] = bytes <= 0 ? v[i] : bytes >= 4 ? 0 : v[i] & (int)(~0u << 8 * bytes);
    }
    return v;
}

__device__ inline v4i mfma(v4i x, v4i y, v4i acc) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(x, y, acc, 0, 0, 0); }

// In LDS the 16-byte parts of a row are permuted by a key of the row (part ^ key), so that lanes that read together, the same part of
// neighbouring rows, meet different banks: 8 parts of 128-byte rows, 16 of longer ones (no conflicts in the products; 256-byte rows with 8
// keys had conflicts in half of the reads' cycles).
template <typename G>
__device__ inline uint32_t row_key(uint32_t row) { return row & (G::PARTS < 16 ? 7 : 15); }

// Workgroups go to the 8 dies in turn, each of which has an L2 of its own: a die takes tiles side by side, in bands of 4 rows of tiles.
__device__ inline void place_tile(uint32_t id, uint32_t tiles_m, uint32_t tiles_n, uint32_t& tm, uint32_t& tn) {
    constexpr uint32_t DIES = 8, BAND = 4;
    const uint32_t total = tiles_m * tiles_n, per = total / DIES, rest = total % DIES, die = id % DIES;
    const uint32_t at = die * per + (die < rest ? die : rest) + id / DIES;
    const uint32_t first = at / (BAND * tiles_n) * BAND, high = tiles_m - first < BAND ? tiles_m - first : BAND, in = at - first * tiles_n;
    tm = first + in % high;
    tn = in / high;
}

typedef __attribute__((address_space(3))) int8_t lds_byte;

// Where the steps' rows come from: the tile and step that are fetched next.
template <typename G>
struct Source {
    const MatmulArgs& g;
    uint32_t tiles, steps, lane, wave;
    uint32_t tile, step = 0;
    __amdgpu_buffer_rsrc_t ra, rb;
    const int8_t *pa, *pb;                // of the tile's first rows
    using offset = std::conditional_t<G::DIRECT, uint32_t, uint64_t>;
    offset oa[G::LA], ob[G::LB];          // a lane's 16 bytes within the tile's rows, of step 0
    v4i va[G::DIRECT ? 1 : G::LA], vb[G::DIRECT ? 1 : G::LB];

    __device__ uint32_t row_of(int j) const { return (j * G::W + wave) * G::ROWS + lane / G::PARTS; }
    __device__ uint32_t part(int j) const { return lane % G::PARTS ^ row_key<G>(row_of(j)); }

    __device__ void aim() {
        uint32_t tm, tn;
        place_tile(tile, g.tiles_m, g.tiles_n, tm, tn);
        const uint64_t m0 = (uint64_t)tm * G::TM, n0 = (uint64_t)tn * G::TN;
        const uint32_t last_a = (uint32_t)(g.m - m0 < G::TM ? g.m - m0 : G::TM) - 1, last_b = (uint32_t)(g.n - n0 < G::TN ? g.n - n0 : G::TN) - 1;
        pa = g.a + m0 * g.lda;
        pb = g.b + n0 * g.ldb;
        // rows past the last one: the last one again (their results are not stored)
#pragma unroll
        for (int j = 0; j < G::LA; ++j) oa[j] = min(row_of(j), last_a) * (offset)g.lda + part(j) * 16;
#pragma unroll
        for (int j = 0; j < G::LB; ++j) ob[j] = min(row_of(j), last_b) * (offset)g.ldb + part(j) * 16;
        if constexpr (G::DIRECT) {
            ra = __builtin_amdgcn_make_buffer_rsrc((void*)pa, 0, last_a * (uint32_t)g.lda + g.k, 0x00020000);
            rb = __builtin_amdgcn_make_buffer_rsrc((void*)pb, 0, last_b * (uint32_t)g.ldb + g.k, 0x00020000);
            if (steps == 1) fold();
        }
    }
    // The last step, if the columns end within it: lanes whose part lies behind the end read the step's first part instead.
    __device__ void fold() {
        const uint32_t left = g.k - (steps - 1) * G::STEP;
        if (left == G::STEP) return;
#pragma unroll
        for (int j = 0; j < G::LA; ++j)
            if (part(j) * 16 >= left) oa[j] -= part(j) * 16;
#pragma unroll
        for (int j = 0; j < G::LB; ++j)
            if (part(j) * 16 >= left) ob[j] -= part(j) * 16;
    }
    // Start the transfer of a step (DIRECT: to LDS; otherwise into registers, for land()).
    __device__ void fetch(int8_t* a, int8_t* b) {
        if constexpr (G::DIRECT) {
#pragma unroll
            for (int j = 0; j < G::LA; ++j)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_byte*)(a + (j * G::W + wave) * 1024), 16, oa[j], step * G::STEP, 0, 0);
#pragma unroll
            for (int j = 0; j < G::LB; ++j)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (lds_byte*)(b + (j * G::W + wave) * 1024), 16, ob[j], step * G::STEP, 0, 0);
        } else {
            const uint32_t c = step * G::STEP;
            if (c + G::STEP <= g.k) {   // one branch for all of a step's loads, which then are on their way together
#pragma unroll
                for (int j = 0; j < G::LA; ++j) __builtin_memcpy(&va[j], pa + oa[j] + c, 16);
#pragma unroll
                for (int j = 0; j < G::LB; ++j) __builtin_memcpy(&vb[j], pb + ob[j] + c, 16);
            } else if (g.k >= 16) {
#pragma unroll
                for (int j = 0; j < G::LA; ++j) __builtin_memcpy(&va[j], pa + (oa[j] - part(j) * 16) + min(c + part(j) * 16, g.k - 16), 16);
#pragma unroll
                for (int j = 0; j < G::LB; ++j) __builtin_memcpy(&vb[j], pb + (ob[j] - part(j) * 16) + min(c + part(j) * 16, g.k - 16), 16);
#pragma unroll
                for (int j = 0; j < G::LA; ++j) va[j] = unseen(va[j], c + part(j) * 16 - min(c + part(j) * 16, g.k - 16));
            } else {
#pragma unroll
                for (int j = 0; j < G::LA; ++j) va[j] = load_few(pa + (oa[j] - part(j) * 16), part(j) * 16, g.k);
#pragma unroll
                for (int j = 0; j < G::LB; ++j) vb[j] = load_few(pb + (ob[j] - part(j) * 16), part(j) * 16, g.k);
            }
        }
    }
    __device__ void land(int8_t* a, int8_t* b) {
        if constexpr (!G::DIRECT) {
#pragma unroll
            for (int j = 0; j < G::LA; ++j) *(v4i*)(a + (j * G::W + wave) * 1024 + lane * 16) = va[j];
#pragma unroll
            for (int j = 0; j < G::LB; ++j) *(v4i*)(b + (j * G::W + wave) * 1024 + lane * 16) = vb[j];
            // lgkmcnt(0): the compiler left the wait out of the barrier at the loop's head, over whose back edge these stores come
            __builtin_amdgcn_s_waitcnt(0xC07F);
        }
    }
    // Before the barrier behind which all waves read a step: what this wave fetched of it is in LDS.  (The compiler put the same wait there by
    // itself; with it written out the instructions are the same.)
    __device__ void arrived() const {
        if constexpr (G::DIRECT) __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
    }
    // After the last tile the fetches repeat its steps, which nobody reads.
    __device__ void advance() {
        if (++step == steps) {
            step = 0;
            if (tile + gridDim.x < tiles) tile += gridDim.x;
            aim();
        } else if (G::DIRECT && step == steps - 1) {
            fold();
        }
    }
    // Before a step is multiplied, where the columns end within it: zeros for the tokens' columns behind the end, by the wave that
    // fetched them (the channels' may hold anything then).
    __device__ void clear_tail(int8_t* a) const {
        const uint32_t left = g.k - (steps - 1) * G::STEP;
        __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0): the transfers to LDS have landed
#pragma unroll
        for (int j = 0; j < G::LA; ++j)
            if (part(j) * 16 + 16 > left) {
                v4i* at = (v4i*)(a + (j * G::W + wave) * 1024 + lane * 16);
                v4i v = {0, 0, 0, 0};
                if constexpr (G::WORDS) {   // (with this 8192^3 takes 443 us instead of 432)
                    v = *at;
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] = part(j) * 16 + i * 4 < left ? v[i] : 0;
                }
                *at = v;
            }
    }
};

// The products of one step.
template <typename G>
__device__ inline void multiply_step(v4i (&acc)[G::FM][G::FQ][4], const int8_t* a, const int8_t* b, uint32_t wm, uint32_t wn, uint32_t lane) {
    constexpr int R = G::FM + G::FQ * 4, M = G::FM * G::FQ * 4, V = G::LA + G::LB, PIECES = G::STEP / 64;
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int kk = 0; kk < PIECES; ++kk) {
        v4i tok[G::FM], ch[G::FQ][4];
#pragma unroll
        for (int f = 0; f < G::FM; ++f) {
            const uint32_t row = wm + f * 16 + lane % 16;
            tok[f] = *(const v4i*)(a + row * G::STEP + ((kk * 4 + lane / 16) ^ row_key<G>(row)) * 16);
        }
#pragma unroll
        for (int q = 0; q < G::FQ; ++q)
#pragma unroll
            for (int f = 0; f < 4; ++f) {
                const uint32_t row = wn + q * 64 + f * 16 + lane % 16;
                ch[q][f] = *(const v4i*)(b + row * G::STEP + ((kk * 4 + lane / 16) ^ row_key<G>(row)) * 16);
            }
#pragma unroll
        for (int fm = 0; fm < G::FM; ++fm)
#pragma unroll
            for (int q = 0; q < G::FQ; ++q)
#pragma unroll
                for (int f = 0; f < 4; ++f) acc[fm][q][f] = mfma(ch[q][f], tok[fm], acc[fm][q][f]);
    }
    if constexpr (G::DIRECT) {
        // Order: the reads of the first 64 columns; products with the next columns' reads between them, and in the first half of
        // the step the next step's transfers (a burst of transfers at the step's start held the products up: 8192^3 486 -> 427 us
        // with this and the rounds over tiles).
        constexpr int N = M < 8 ? M : 8, SPREAD = (PIECES / 2) * N;
        __builtin_amdgcn_sched_group_barrier(0x100, R, 0);
#pragma unroll
        for (int kk = 0; kk < PIECES - 1; ++kk)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, M / N, 0);
                if (kk < PIECES / 2) __builtin_amdgcn_sched_group_barrier(0x020, (V + SPREAD - 1) / SPREAD, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, (R + N - 1) / N, 0);
            }
        __builtin_amdgcn_sched_group_barrier(0x008, M, 0);
    }
    __builtin_amdgcn_s_setprio(0);
}

// LDS written by some lanes of a wave and read by others of it: their order in the code is the order that they are done in.
__device__ inline void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// A wave's results of a tile, scaled, to memory, 16 tokens x 64 channels at a time: through 4 KB of LDS of its own, so that a store's
// lanes write the channels of a token side by side (lines of 128 bytes).  16-byte parts of a token's 256 are permuted by its number.
template <typename T, typename G>
__device__ inline void store_tile(const MatmulArgs& g, v4i (&acc)[G::FM][G::FQ][4], float* turn, uint64_t m0, uint64_t n0, uint32_t lane) {
    constexpr int RUN = 16 / sizeof(T), PARTS = RUN / 4, LANES = 64 / RUN, ROWS = 64 / LANES;   // channels a lane, lanes a token
    static_assert(G::FM * 16 <= 64, "a lane holds the scale of one of the wave's tokens");
    const float own = g.sa[min(m0 + lane % (G::FM * 16), g.m - 1)];   // (read where it was used, it was waited for eight times a tile)
#pragma unroll
    for (int q = 0; q < G::FQ; ++q) {
        const uint64_t channel = n0 + q * 64 + lane % LANES * RUN;
        float sb[RUN], bias[RUN];
#pragma unroll
        for (int i = 0; i < RUN; ++i) {
            const uint64_t c = min(channel + i, g.n - 1);
            sb[i] = g.sb[c];
            bias[i] = g.bias ? g.bias[c] : 0.f;
        }
#pragma unroll
        for (int fm = 0; fm < G::FM; ++fm) {
#pragma unroll
            for (int f = 0; f < 4; ++f) {
                const uint32_t token = lane % 16;
                typedef float v4f __attribute__((ext_vector_type(4)));
                *(v4f*)(turn + token * 64 + ((f * 4 + lane / 16) ^ token) * 4) = __builtin_convertvector(acc[fm][q][f], v4f);
                acc[fm][q][f] = v4i{0, 0, 0, 0};
            }
            wave_sync();
#pragma unroll
            for (int r = 0; r < 16; r += ROWS) {
                const uint32_t row = r + lane / LANES;
                const uint64_t token = m0 + fm * 16 + row;
                const float sa = __shfl(own, fm * 16 + row);
                if (token < g.m) {
                    float y[RUN];
#pragma unroll
                    for (int p = 0; p < PARTS; ++p)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            y[p * 4 + i] = fmaf(turn[row * 64 + ((lane % LANES * PARTS + p) ^ row) * 4 + i], sa * sb[p * 4 + i], bias[p * 4 + i]);
                    T* out = (T*)g.out + token * g.ldo + channel;
                    if (channel + RUN <= g.n) store_run<T, RUN>(out, y);
                    else
#pragma unroll
                        for (int i = 0; i < RUN; ++i)
                            if (channel + i < g.n) out[i] = (T)y[i];
                }
            }
            wave_sync();
        }
    }
}
// A wave's sums of a tile over some of the columns, as they are, 16 bytes a lane (out: rows of whole 64 channels).
template <typename G>
__device__ inline void store_sums(const MatmulArgs& g, v4i (&acc)[G::FM][G::FQ][4], uint64_t m0, uint64_t n0, uint32_t lane) {
#pragma unroll
    for (int fm = 0; fm < G::FM; ++fm) {
        const uint64_t token = m0 + fm * 16 + lane % 16;
#pragma unroll
        for (int q = 0; q < G::FQ; ++q)
#pragma unroll
            for (int f = 0; f < 4; ++f) {
                if (token < g.m) *(v4i*)((int*)g.out + token * g.ldo + n0 + q * 64 + f * 16 + lane / 16 * 4) = acc[fm][q][f];
                acc[fm][q][f] = v4i{0, 0, 0, 0};
            }
    }
}

// A wave's results of a tile as logits of a vocabulary: for each token their largest, and what the softmax needs of them: s = sum e^(l - m),
// t = sum e^(l - m) (l - m).  Lane / 16 has channels 4 (lane / 16) .. + 3 of each fragment, so that a token's are in 4 lanes.
template <typename G>
__device__ inline void sum_tile(const MatmulArgs& g, v4i (&acc)[G::FM][G::FQ][4], uint64_t m0, uint64_t n0, uint32_t lane) {
    static_assert(G::FQ * 64 == HEAD_GROUP, "a wave's channels are one group");
    constexpr float LOG2E = 1.44269504088896340736f, MINUS_INF = -__builtin_huge_valf();
    float sb[G::FQ][4][4], off[G::FQ][4][4];   // off: 0, or -inf behind the last channel
#pragma unroll
    for (int q = 0; q < G::FQ; ++q)
#pragma unroll
        for (int f = 0; f < 4; ++f)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint64_t c = n0 + q * 64 + f * 16 + lane / 16 * 4 + i;
                sb[q][f][i] = g.sb[min(c, g.n - 1)];
                off[q][f][i] = c < g.n ? 0.f : MINUS_INF;
            }
    const float own = g.sa[min(m0 + lane % (G::FM * 16), g.m - 1)];
#pragma unroll
    for (int fm = 0; fm < G::FM; ++fm) {
        const float sa = __shfl(own, fm * 16 + lane % 16);
        float m = MINUS_INF;
#pragma unroll
        for (int q = 0; q < G::FQ; ++q)
#pragma unroll
            for (int f = 0; f < 4; ++f)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float x = fmaf((float)acc[fm][q][f][i], sa * sb[q][f][i], off[q][f][i]);
                    acc[fm][q][f][i] = (int)__float_as_uint(x);
                    m = fmaxf(m, x);
                }
        m = fmaxf(m, __shfl_xor(m, 16));
        m = fmaxf(m, __shfl_xor(m, 32));
        const float base = m == MINUS_INF ? 0.f : m;
        float s = 0.f, t = 0.f;
#pragma unroll
        for (int q = 0; q < G::FQ; ++q)
#pragma unroll
            for (int f = 0; f < 4; ++f) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float d = __uint_as_float((uint32_t)acc[fm][q][f][i]) - base, e = __builtin_amdgcn_exp2f(d * LOG2E);
                    s += e;
                    t = fmaf(e, fmaxf(d, -1000.f), t);
                }
                acc[fm][q][f] = v4i{0, 0, 0, 0};
            }
        s += __shfl_xor(s, 16);
        t += __shfl_xor(t, 16);
        s += __shfl_xor(s, 32);
        t += __shfl_xor(t, 32);
        const uint64_t token = m0 + fm * 16 + lane % 16;
        if (lane < 16 && token < g.m && n0 < g.n) ((float4*)g.out)[token * g.ldo + n0 / HEAD_GROUP] = make_float4(m, s, t, 0.f);
    }
}
#endif

template <typename T, typename G>
__global__ __launch_bounds__(64 * G::W) void scaled_matmul_kernel(MatmulArgs g) {
#if defined(__HIP_DEVICE_COMPILE__)
    __shared__ __align__(16) int8_t a0[G::TM * G::STEP], b0[G::TN * G::STEP], a1[G::TM * G::STEP], b1[G::TN * G::STEP];
    __shared__ __align__(16) float turns[std::is_void_v<T> || std::is_same_v<T, int> ? 1 : G::W][16 * 64];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t wm = wave % G::WM * (G::TM / G::WM), wn = wave / G::WM * (G::TN / G::WN);
    if constexpr (std::is_same_v<T, int>) {   // the workgroup's part of the columns, and where its sums go
        const uint32_t c0 = blockIdx.y * g.part_cols;
        g.a += c0;
        g.b += c0;
        g.k = min(g.k - c0, g.part_cols);
        g.out = (int*)g.out + blockIdx.y * g.m * g.ldo;
    }
    const uint32_t tiles = g.tiles_m * g.tiles_n, steps = (g.k + G::STEP - 1) / G::STEP;
    const bool partial = G::DIRECT && g.k % G::STEP != 0;
    Source<G> src{g, tiles, steps, lane, wave, blockIdx.x};
    src.aim();
    v4i acc[G::FM][G::FQ][4] = {};
    uint32_t tile = blockIdx.x, step = 0;
    src.fetch(a0, b0);
    src.land(a0, b0);
    src.advance();
    for (;;) {
        if (partial && step == steps - 1) src.clear_tail(a0);
        src.arrived();
        __syncthreads();
        src.fetch(a1, b1);
        multiply_step<G>(acc, a0, b0, wm, wn, lane);
        src.land(a1, b1);
        src.advance();
        if (++step == steps) {
            uint32_t tm, tn;
            place_tile(tile, g.tiles_m, g.tiles_n, tm, tn);
            if constexpr (std::is_same_v<T, int>) store_sums<G>(g, acc, (uint64_t)tm * G::TM + wm, (uint64_t)tn * G::TN + wn, lane);
            else if constexpr (std::is_void_v<T>) sum_tile<G>(g, acc, (uint64_t)tm * G::TM + wm, (uint64_t)tn * G::TN + wn, lane);
            else store_tile<T, G>(g, acc, turns[wave], (uint64_t)tm * G::TM + wm, (uint64_t)tn * G::TN + wn, lane);
            step = 0;
            tile += gridDim.x;
            if (tile >= tiles) break;
        }
        if (partial && step == steps - 1) src.clear_tail(a1);
        src.arrived();
        __syncthreads();
        src.fetch(a0, b0);
        multiply_step<G>(acc, a1, b1, wm, wn, lane);
        src.land(a0, b0);
        src.advance();
        if (++step == steps) {
            uint32_t tm, tn;
            place_tile(tile, g.tiles_m, g.tiles_n, tm, tn);
            if constexpr (std::is_same_v<T, int>) store_sums<G>(g, acc, (uint64_t)tm * G::TM + wm, (uint64_t)tn * G::TN + wn, lane);
            else if constexpr (std::is_void_v<T>) sum_tile<G>(g, acc, (uint64_t)tm * G::TM + wm, (uint64_t)tn * G::TN + wn, lane);
            else store_tile<T, G>(g, acc, turns[wave], (uint64_t)tm * G::TM + wm, (uint64_t)tn * G::TN + wn, lane);
            step = 0;
            tile += gridDim.x;
            if (tile >= tiles) break;
        }
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0): nothing arrives in LDS that is no longer this workgroup's
#endif
}

// ---- few tokens -------------------------------------------------------------------------------------------------------------
// Up to 32 tokens: reading b is all there is, so that many waves, each with several loads on their way, matter more than the
// matrix cores' rate.  A wave takes 16 channels and every KS-th 128 columns, straight from memory into the fragments' order (16
// bytes of each of 16 rows); the 8 waves of a workgroup are KS parts of 8 / KS groups of channels and are added up in LDS.
template <typename T, int MT, int KS, bool ALIGNED>
__global__ __launch_bounds__(512) void scaled_matmul_few_kernel(MatmulArgs g) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int GROUPS = 8 / KS, AHEAD = 4;   // 128-column steps loaded before they are multiplied
    __shared__ __align__(16) v4i parts[KS == 1 ? 1 : 8][MT][64];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint64_t n0 = ((uint64_t)blockIdx.x * GROUPS + wave / KS) * 16;
    const int8_t* row_b = g.b + min(n0 + lane % 16, g.n - 1) * g.ldb;
    const int8_t* row_a[MT];
#pragma unroll
    for (int f = 0; f < MT; ++f) row_a[f] = g.a + min((uint64_t)(f * 16 + lane % 16), g.m - 1) * g.lda;
    v4i acc[MT] = {};
    for (uint32_t c0 = wave % KS * LINE; c0 < g.k; c0 += KS * LINE * AHEAD) {
        v4i ch[AHEAD][2], tok[AHEAD][2][MT];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t c = c0 + u * KS * LINE + h * 64 + lane / 16 * 16;
                ch[u][h] = v4i{0, 0, 0, 0};
#pragma unroll
                for (int f = 0; f < MT; ++f) tok[u][h][f] = v4i{0, 0, 0, 0};
                // no loads behind the end, which would cost what others do (1 token x 1024 x 1024 4.5 us with them, 3.1 without)
                if (c < g.k) {
                    if constexpr (ALIGNED) {
                        ch[u][h] = *(const v4i*)(row_b + c);
#pragma unroll
                        for (int f = 0; f < MT; ++f) tok[u][h][f] = *(const v4i*)(row_a[f] + c);
                    } else {   // k >= 16: the launch's rule
                        const uint32_t at = min(c, g.k - 16);
                        __builtin_memcpy(&ch[u][h], row_b + at, 16);
#pragma unroll
                        for (int f = 0; f < MT; ++f) {
                            __builtin_memcpy(&tok[u][h][f], row_a[f] + at, 16);
                            tok[u][h][f] = unseen(tok[u][h][f], c - at);
                        }
                    }
                }
            }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int f = 0; f < MT; ++f) acc[f] = mfma(ch[u][h], tok[u][h][f], acc[f]);
    }
    if constexpr (KS > 1) {
#pragma unroll
        for (int f = 0; f < MT; ++f) parts[wave][f][lane] = acc[f];
        __syncthreads();
        // the group's waves share the fragments to add up
        const uint32_t first = wave / KS * KS;
#pragma unroll
        for (int f = 0; f < MT; ++f) {
            if (f % KS != wave % KS) continue;
            acc[f] = parts[first][f][lane];
            for (int p = 1; p < KS; ++p) acc[f] += parts[first + p][f][lane];
        }
    }
    const uint64_t channel = n0 + lane / 16 * 4;
#pragma unroll
    for (int f = 0; f < MT; ++f) {
        const uint64_t token = f * 16 + lane % 16;
        if (f % KS != wave % KS || token >= g.m) continue;
        const float sa = g.sa[token];
        T* out = (T*)g.out + token * g.ldo + channel;
        float y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint64_t c = min(channel + i, g.n - 1);
            y[i] = fmaf((float)acc[f][i], sa * g.sb[c], g.bias ? g.bias[c] : 0.f);
        }
        if (channel + 4 <= g.n) store_run<T, 4>(out, y);
        else
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (channel + i < g.n) out[i] = (T)y[i];
    }
#endif
}

// As many parts of the columns as give 2048 waves, 8 at most: one token x 32000 x 1024 with 1 / 2 / 4 / 8 parts 10.3 / 8.9 / 13.2 / 21.6 us,
// x 4096 x 4096 20.5 / 11.8 / 7.5 / 6.1, x 8192 x 8192 39 / 22 / 15.4 / 16.0.
template <typename T, int MT, int KS, bool ALIGNED>
hipError_t launch_few_parts(const MatmulArgs& g, hipStream_t stream) {
    hipError_t e = hipSuccess;
    in_launches(g.n, 16 * (8 / KS), 512, [&](uint64_t first, uint64_t n, uint32_t workgroups) {
        MatmulArgs part = g;
        part.b = g.b + first * g.ldb;
        part.sb = g.sb + first;
        if (g.bias) part.bias = g.bias + first;
        part.out = (T*)g.out + first;
        part.n = n;
        scaled_matmul_few_kernel<T, MT, KS, ALIGNED><<<dim3(workgroups), dim3(512), 0, stream>>>(part);
        if (e == hipSuccess) e = hipGetLastError();
    });
    return e;
}

template <typename T, int MT, bool ALIGNED>
hipError_t launch_few(const MatmulArgs& g, hipStream_t stream) {
    const uint64_t groups = (g.n + 15) / 16;
    if (groups >= 2048) return launch_few_parts<T, MT, 1, ALIGNED>(g, stream);
    if (groups >= 1024) return launch_few_parts<T, MT, 2, ALIGNED>(g, stream);
    if (groups >= 512) return launch_few_parts<T, MT, 4, ALIGNED>(g, stream);
    return launch_few_parts<T, MT, 8, ALIGNED>(g, stream);
}

template <typename T, typename G>
hipError_t launch_tile_shape(MatmulArgs g, hipStream_t stream, uint32_t parts = 1) {
    const uint64_t tm = (g.m + G::TM - 1) / G::TM, tn = (g.n + G::TN - 1) / G::TN;
    g.tiles_m = (uint32_t)tm;
    g.tiles_n = (uint32_t)tn;
    // as many workgroups as the 256 CUs, with 160 KB of LDS each, hold at once
    const uint64_t most = 256 * (163840 / (2 * (G::TM + G::TN) * G::STEP + G::W * 4096));
    const uint64_t tiles = tm * tn;
    scaled_matmul_kernel<T, G><<<dim3((uint32_t)(tiles < most ? tiles : most), parts), dim3(64 * G::W), 0, stream>>>(g);
    return hipGetLastError();
}

// The logits of the groups of channels that a row's best entries lie in (head_lists_kernel): a workgroup takes up to 32 entries of
// one group's list and all of its channels, its waves a quarter of the columns each, straight from memory into the fragments' order.  (A
// wave for each part of a list: 4096 rows x 5 of 250 groups x 2048 columns 46 us, this 39.5; neighbouring parts on the same die, whose
// L2 would then serve the channels once: 54.)
__global__ __launch_bounds__(256) void head_groups_kernel(HeadArgs h) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int CH = HEAD_GROUP / 16, TOK = HEAD_LIST_STEP / 16, AHEAD = 2;
    const MatmulArgs& g = h.product;
    const uint32_t lane = threadIdx.x & 63, groups = h.groups;
    const uint32_t wave = threadIdx.x >> 6;
    __shared__ __align__(16) int sums[TOK][CH][4][64];
    // which part of which list: the lists' lengths are known on the device only
    uint32_t item = blockIdx.x, group = groups, count = 0;
    for (uint32_t g0 = 0; g0 < groups; g0 += 64) {
        const uint32_t own = g0 + lane < groups ? h.counts[g0 + lane] : 0, parts = (own + HEAD_LIST_STEP - 1) / HEAD_LIST_STEP;
        uint32_t upto = parts;
#pragma unroll
        for (int o = 1; o < 64; o *= 2) {
            const uint32_t left = __shfl_up(upto, o);
            if (lane >= (uint32_t)o) upto += left;
        }
        const uint64_t past = __ballot(upto > item);
        if (past) {
            const int at = __ffsll((unsigned long long)past) - 1;
            group = g0 + at;
            count = __shfl(own, at);
            item -= __shfl(upto, at) - __shfl(parts, at);
            break;
        }
        item -= __shfl(upto, 63);
    }
    if (group == groups) return;   // the same in all four waves
    for (uint32_t i = threadIdx.x; i < TOK * CH * 64; i += 256) ((v4i*)sums)[i] = v4i{0, 0, 0, 0};
    __syncthreads();
    const uint32_t* list = h.lists + (uint64_t)group * g.m + item * HEAD_LIST_STEP;
    const uint32_t here = min(count - item * HEAD_LIST_STEP, (uint32_t)HEAD_LIST_STEP);
    const uint64_t n0 = (uint64_t)group * HEAD_GROUP;
    uint32_t entry[TOK];
    const int8_t* row_a[TOK];
#pragma unroll
    for (int f = 0; f < TOK; ++f) {
        entry[f] = list[min(f * 16 + lane % 16, here - 1)];
        row_a[f] = g.a + (uint64_t)(entry[f] / h.n_top) * g.lda;
    }
    const int8_t* row_b[CH];
#pragma unroll
    for (int f = 0; f < CH; ++f) row_b[f] = g.b + min(n0 + f * 16 + lane % 16, g.n - 1) * g.ldb;
    v4i acc[TOK][CH] = {};
    for (uint32_t c0 = wave * 64; c0 < g.k; c0 += 4 * 64 * AHEAD) {
        v4i ch[AHEAD][CH], tok[AHEAD][TOK];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const uint32_t c = c0 + u * 4 * 64 + lane / 16 * 16, at = c < g.k ? c : 0;   // behind the columns: any channels' bytes, times zeros
#pragma unroll
            for (int f = 0; f < CH; ++f) ch[u][f] = *(const v4i*)(row_b[f] + at);
#pragma unroll
            for (int f = 0; f < TOK; ++f) {
                const v4i v = *(const v4i*)(row_a[f] + at);
                tok[u][f] = c < g.k ? v : v4i{0, 0, 0, 0};
            }
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
#pragma unroll
            for (int t = 0; t < TOK; ++t)
#pragma unroll
                for (int f = 0; f < CH; ++f) acc[t][f] = mfma(ch[u][f], tok[u][t], acc[t][f]);
    }
#pragma unroll
    for (int t = 0; t < TOK; ++t)
#pragma unroll
        for (int f = 0; f < CH; ++f)
#pragma unroll
            for (int i = 0; i < 4; ++i) atomicAdd(&sums[t][f][i][lane], acc[t][f][i]);
    __syncthreads();
#pragma unroll
    for (int t = 0; t < TOK; ++t) {
        if (t * 16 + lane % 16 >= here) continue;
        const float sa = g.sa[entry[t] / h.n_top];
        float* out = h.logits + (uint64_t)entry[t] * HEAD_GROUP + lane / 16 * 4;
        for (uint32_t f = wave * (CH / 4); f < (wave + 1) * (CH / 4); ++f) {
            float x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {   // as sum_tile has them
                const uint64_t channel = n0 + f * 16 + lane / 16 * 4 + i;
                x[i] = fmaf((float)sums[t][f][i][lane], sa * g.sb[min(channel, g.n - 1)], channel < g.n ? 0.f : -__builtin_huge_valf());
            }
            store_run<float, 4>(out + f * 16, x);
        }
    }
#endif
}

// The parts' sums added, scaled, to memory: 4 channels a thread.
template <typename T>
__global__ __launch_bounds__(256) void join_parts_kernel(MatmulArgs g, const int* sums, uint64_t row, uint32_t parts) {
    const uint64_t quads = (g.n + 3) / 4, at = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= g.m * quads) return;
    const uint64_t token = at / quads, channel = at % quads * 4;
    v4i sum = {0, 0, 0, 0};
    for (uint32_t p = 0; p < parts; ++p) sum += *(const v4i*)(sums + (p * g.m + token) * row + channel);
    const float sa = g.sa[token];
    T* out = (T*)g.out + token * g.ldo + channel;
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint64_t c = min(channel + i, g.n - 1);
        y[i] = fmaf((float)sum[i], sa * g.sb[c], g.bias ? g.bias[c] : 0.f);
    }
    if (channel + 4 <= g.n) store_run<T, 4>(out, y);
    else
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (channel + i < g.n) out[i] = (T)y[i];
}

template <typename T, bool DIRECT>
hipError_t launch_parts(const MatmulArgs& g, uint32_t parts, void* workspace, hipStream_t stream) {
    using G = Tile<64, 64, 4, 1, DIRECT ? 256 : 128, DIRECT>;
    MatmulArgs p = g;
    p.out = workspace;
    p.ldo = (g.n + 63) / 64 * 64;
    p.part_cols = (uint32_t)(((g.k + parts - 1) / parts + G::STEP - 1) / G::STEP * G::STEP);
    parts = (g.k + p.part_cols - 1) / p.part_cols;
    hipError_t e = launch_tile_shape<int, G>(p, stream, parts);
    if (e != hipSuccess) return e;
    const uint64_t threads = g.m * ((g.n + 3) / 4);
    join_parts_kernel<T><<<dim3((uint32_t)((threads + 255) / 256)), dim3(256), 0, stream>>>(g, (const int*)workspace, p.ldo, parts);
    return hipGetLastError();
}

// UNIT: the rows lie at multiples of 16 bytes, of 4, or anywhere.
// 256^2, where 128^2, two workgroups of which a CU holds, would take more than one round (256^2 / 128^2 tiles, us: 2048 x 4096 x 2048 128 / 512 tiles 33.5 /
// 23.4, 128 x 50000 x 1024 196 / 391 tiles 23.5 / 16.7, 3000 x 3000 x 2048 144 / 576 tiles 33.8 / 34.4, 4096 x 4096 x 4096 256 / 1024 tiles 67.8 / 70.8;
// rows at 4 bytes 34.8 / 30.0, 22.9 / 18.9, 36.5 / 40.2, 70.9 / 91.9); through registers they gain nothing (126.3 / 118.8 for 4096^3).
// 128^2 / 64^2: 2048 x 1024 x 1024 128 / 512 tiles 11.1 / 8.1, 1536 x 2048 x 4096 192 / 768 26.1 / 27.6, 2048 x 2048 x 1024 256 / 1024 12.3 / 13.3, 4096 x 4096 x
// 4096 70.8 / 114; through registers 18.0 / 12.2, 56.3 / 45.7, 18.7 / 22.1, 119 / 217.
template <typename T, int UNIT>
hipError_t launch_tiles(const MatmulArgs& g, hipStream_t stream) {
    constexpr bool DIRECT = UNIT >= 4;
    const uint64_t middle = ((g.m + 127) / 128) * ((g.n + 127) / 128);
    if constexpr (DIRECT)
        if (middle > 512) return launch_tile_shape<T, Tile<256, 256, 4, 2, 128, true, UNIT == 4>>(g, stream);
    if (middle >= 192) return launch_tile_shape<T, Tile<128, 128, 2, 2, 128, DIRECT>>(g, stream);
    // Small tiles wait for memory once a step: longer steps where there are columns for them, the longest (a workgroup a CU) where there
    // are no more tiles than CUs.  128 / 256 / 512 columns: 128 x 4096 x 4096 24.8 / 16.6 / 14.3 us, 256 x 8192 x 8192 50.6 / 40.0 / 47.6,
    // 256 x 1024 x 1024 6.8 / 6.1 / 6.5.  Through registers they pay no more: 1111 x 1003 x 1029 15.6 / 17.4.
    if constexpr (DIRECT) {
        const uint64_t small = ((g.m + 63) / 64) * ((g.n + 63) / 64);
        if (g.k >= 2048 && small <= 256) return launch_tile_shape<T, Tile<64, 64, 4, 1, 512, true>>(g, stream);
        if (g.k > 256) return launch_tile_shape<T, Tile<64, 64, 4, 1, 256, true>>(g, stream);
    }
    return launch_tile_shape<T, Tile<64, 64, 4, 1, 128, DIRECT>>(g, stream);
}

template <typename T, int UNIT>
hipError_t launch_type(const MatmulArgs& g, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    if (by_columns(g.m, g.n, g.k, UNIT)) {
        if constexpr (UNIT >= 4)
            if (g.m > 16) return launch_few<T, 2, UNIT == 16>(g, stream);
        return launch_few<T, 1, UNIT == 16>(g, stream);
    }
    uint32_t parts = column_parts(g.m, g.n, g.k, UNIT);
    while (parts > 1 && parts_bytes(g.m, g.n, parts) > workspace_bytes) --parts;
    return parts > 1 ? launch_parts<T, UNIT >= 4>(g, parts, workspace, stream) : launch_tiles<T, UNIT>(g, stream);
}

bool rows_at(const MatmulArgs& g, uint32_t bytes) {
    return (uintptr_t)g.a % bytes == 0 && (uintptr_t)g.b % bytes == 0 && g.lda % bytes == 0 && g.ldb % bytes == 0 && g.k % bytes == 0 &&
           g.lda < (1u << 23) && g.ldb < (1u << 23);   // 32-bit offsets within a tile
}

template <typename T>
hipError_t launch_aligned(const MatmulArgs& g, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    if (rows_at(g, 16)) return launch_type<T, 16>(g, workspace, workspace_bytes, stream);
    if (rows_at(g, 4)) return launch_type<T, 4>(g, workspace, workspace_bytes, stream);
    return launch_type<T, 1>(g, workspace, workspace_bytes, stream);
}

}  // namespace

bool scaled_matmul_aligned(const MatmulArgs& g) { return rows_at(g, 16); }

hipError_t launch_head_sums(const HeadArgs& h, hipStream_t stream) {
    MatmulArgs g = h.product;
    g.out = h.sums;
    g.ldo = h.groups;
    return launch_tile_shape<void, Tile<256, 256, 4, 2, 128, true, false>>(g, stream);
}

hipError_t launch_head_groups(const HeadArgs& h, hipStream_t stream) {
    // at most: every list has a part that is not full
    const uint64_t items = h.groups + h.product.m * h.n_top / HEAD_LIST_STEP;
    head_groups_kernel<<<dim3((uint32_t)items), dim3(256), 0, stream>>>(h);
    return hipGetLastError();
}

hipError_t launch_scaled_matmul(const MatmulArgs& g, uint32_t out_dtype, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    if (g.m == 0 || g.n == 0) return hipSuccess;
    if (out_dtype == TYPE_F16) return launch_aligned<f16_t>(g, workspace, workspace_bytes, stream);
    if (out_dtype == TYPE_BF16) return launch_aligned<bf16_t>(g, workspace, workspace_bytes, stream);
    return launch_aligned<float>(g, workspace, workspace_bytes, stream);
}

}  // namespace dessert
