// int8 x int8 products with a scale for each token (row of a) and each channel (row of b):
//     out[i][j] = T( float(sum_c a[i][c] * b[j][c]) * (sa[i] * sb[j]) + bias[j] )
// The sums are exact in int32 whatever their order, so any split of the columns gives the same bits.  Both operands lie with
// their columns side by side, which is the order that v_mfma_i32_16x16x64_i8 takes: 16 bytes of one row per lane.
#include "kernels.hpp"
#include "number_formats.hpp"

namespace dessert {

namespace {

constexpr int STEP = 128;   // columns (bytes) of a row per round of the tile kernel: one line of 128 bytes

// 16 bytes of a row from column c on; columns from k on read as zero.
__device__ inline v4i load_chunk(const int8_t* row, uint32_t c, uint32_t k) {
    v4i v = {0, 0, 0, 0};
    if (c + 16 <= k) {
        __builtin_memcpy(&v, row + c, 16);
    } else if (c < k) {
        int8_t bytes[16];
#pragma unroll
        for (uint32_t i = 0; i < 16; ++i) bytes[i] = c + i < k ? row[c + i] : (int8_t)0;
        __builtin_memcpy(&v, bytes, 16);
    }
    return v;
}

__device__ inline v4i mfma(v4i x, v4i y, v4i acc) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(x, y, acc, 0, 0, 0); }

template <typename T>
__device__ inline void store_channels(const MatmulArgs& g, uint64_t token, uint64_t channel, const int (&sum)[16]) {
    const float sa = g.sa[token];
    T* out = (T*)g.out + token * g.ldo + channel;
    float y[16];
    if (channel + 16 <= g.n) {
        float sb[16], bias[16];
        load_run<float, 16>(g.sb + channel, sb);
        if (g.bias) load_run<float, 16>(g.bias + channel, bias);
#pragma unroll
        for (int i = 0; i < 16; ++i) y[i] = g.bias ? fmaf((float)sum[i], sa * sb[i], bias[i]) : (float)sum[i] * (sa * sb[i]);
        store_run<T, 16>(out, y);
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (channel + i < g.n) {
                const float s = sa * g.sb[channel + i];
                out[i] = (T)(g.bias ? fmaf((float)sum[i], s, g.bias[channel + i]) : (float)sum[i] * s);
            }
    }
}

// Rows' positions within a 128-byte line of LDS are permuted by a key of the row, so that the 8 lanes that read in one cycle
// meet 8 different quarters of banks.  Tokens: 16 consecutive rows a fragment.  Channels: fragment f of a block of 64 holds
// rows 16 * (i / 4) + 4 * f + i % 4, so that a lane's results over the 4 fragments are 16 consecutive channels.
__device__ inline uint32_t token_key(uint32_t row) { return row & 7; }
__device__ inline uint32_t channel_key(uint32_t row) { return (row & 3) | ((row >> 2) & 4); }

// One workgroup: TM tokens x TN channels, WM x WN waves.
template <typename T, int TM, int TN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void scaled_matmul_tile_kernel(MatmulArgs g) {
    constexpr int W = WM * WN, FM = TM / WM / 16, FQ = TN / WN / 64;
    __shared__ __align__(16) int8_t sa_tile[TM * STEP];
    __shared__ __align__(16) int8_t sb_tile[TN * STEP];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t tile = blockIdx.x;
    const uint64_t m0 = (uint64_t)(tile % g.tiles_m) * TM, n0 = (uint64_t)(tile / g.tiles_m) * TN;
    const uint32_t wm = wave % WM * (TM / WM), wn = wave / WM * (TN / WN);
    v4i acc[FM][FQ][4] = {};
    for (uint32_t c0 = 0; c0 < g.k; c0 += STEP) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < TM / 8 / W; ++j) {
            const uint32_t row = (j * W + wave) * 8 + lane / 8, chunk = (lane & 7) ^ token_key(row);
            const uint64_t r = m0 + row < g.m ? m0 + row : g.m - 1;
            *(v4i*)(sa_tile + row * STEP + (lane & 7) * 16) = load_chunk(g.a + r * g.lda, c0 + chunk * 16, g.k);
        }
#pragma unroll
        for (int j = 0; j < TN / 8 / W; ++j) {
            const uint32_t row = (j * W + wave) * 8 + lane / 8, chunk = (lane & 7) ^ channel_key(row);
            const uint64_t r = n0 + row < g.n ? n0 + row : g.n - 1;
            *(v4i*)(sb_tile + row * STEP + (lane & 7) * 16) = load_chunk(g.b + r * g.ldb, c0 + chunk * 16, g.k);
        }
        __syncthreads();
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            v4i tok[FM], ch[FQ][4];
#pragma unroll
            for (int f = 0; f < FM; ++f) {
                const uint32_t row = wm + f * 16 + lane % 16;
                tok[f] = *(const v4i*)(sa_tile + row * STEP + ((kk * 4 + lane / 16) ^ token_key(row)) * 16);
            }
#pragma unroll
            for (int q = 0; q < FQ; ++q)
#pragma unroll
                for (int f = 0; f < 4; ++f) {
                    const uint32_t i = lane % 16, row = wn + q * 64 + i / 4 * 16 + f * 4 + i % 4;
                    ch[q][f] = *(const v4i*)(sb_tile + row * STEP + ((kk * 4 + lane / 16) ^ channel_key(row)) * 16);
                }
#pragma unroll
            for (int fm = 0; fm < FM; ++fm)
#pragma unroll
                for (int q = 0; q < FQ; ++q)
#pragma unroll
                    for (int f = 0; f < 4; ++f) acc[fm][q][f] = mfma(ch[q][f], tok[fm], acc[fm][q][f]);
        }
    }
#pragma unroll
    for (int fm = 0; fm < FM; ++fm) {
        const uint64_t token = m0 + wm + fm * 16 + lane % 16;
        if (token >= g.m) continue;
#pragma unroll
        for (int q = 0; q < FQ; ++q) {
            int sum[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) sum[i] = acc[fm][q][i / 4][i % 4];
            store_channels<T>(g, token, n0 + wn + q * 64 + lane / 16 * 16, sum);
        }
    }
}

template <typename T>
hipError_t launch_tiles(MatmulArgs g, hipStream_t stream) {
    constexpr int TM = 128, TN = 128;
    g.tiles_m = (uint32_t)((g.m + TM - 1) / TM);
    g.tiles_n = (uint32_t)((g.n + TN - 1) / TN);
    scaled_matmul_tile_kernel<T, TM, TN, 2, 2><<<dim3(g.tiles_m * g.tiles_n), dim3(256), 0, stream>>>(g);
    return hipGetLastError();
}

}  // namespace

size_t scaled_matmul_workspace(uint64_t, uint64_t, uint32_t) { return 0; }

hipError_t launch_scaled_matmul(const MatmulArgs& g, uint32_t out_dtype, void*, hipStream_t stream) {
    if (g.m == 0 || g.n == 0) return hipSuccess;
    if (out_dtype == TYPE_F16) return launch_tiles<f16_t>(g, stream);
    if (out_dtype == TYPE_BF16) return launch_tiles<bf16_t>(g, stream);
    return launch_tiles<float>(g, stream);
}

}  // namespace dessert
