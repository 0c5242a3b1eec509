// Rows of numbers to int8 with one scale a row.
//   largest magnitude: scale = max|x| / 127 in 32 bits, code = x / scale
//   unit norm:         scale = |x| / 127, code = 127 x / |x|, the norm in 64 bits (the codes of a vector are whole numbers: a sum of squares
//                      in 32 bits would move some of them over a half)
// each code the nearest integer to the real quotient, ties to even.  Bound by memory: rows are read once and kept in registers between the
// reduction and the codes.  A row with an infinity or NaN gets codes 0 and scale NaN.
#include "kernels.hpp"
#include "number_formats.hpp"

namespace dessert {

namespace {

// What turns a row's numbers into codes: num / den, also as a 32-bit factor.
struct Quotient {
    double num, den;
    float factor;
    bool zero, fast;   // fast: the factor is good to 2^-23

    __device__ Quotient(float peak, double squares, bool bad, bool unit, float& scale) {
        const double norm = sqrt(squares);
        scale = bad ? __builtin_nanf("") : unit ? (float)(norm / 127.0) : peak / 127.f;
        num = unit ? 127.0 : 1.0;
        den = unit ? norm : (double)scale;
        zero = bad || den == 0.0;
        factor = zero ? 0.f : (float)(num / den);
        fast = factor < 0x1p125f && factor > 0x1p-125f;
    }
    // The factor is off by 2^-24 and the product by as much, of at most 127: less than 2^-15.  Where that could matter, next to a half,
    // the quotient is formed in 64 bits: num * x is exact there, and a quotient of such numbers that is no half is further than its
    // rounding away from one.
    __device__ int code(float x) const {
        if (zero) return 0;
        const float t = x * factor;
        float n = rintf(t);
        if (!fast || fabsf(fabsf(t - n) - 0.5f) < 0x1p-14f) n = (float)rint(num * (double)x / den);
        return (int)fminf(fmaxf(n, -127.f), 127.f);
    }
};

// Over the lanes of a row: G consecutive lanes (a power of two).
template <int G>
__device__ inline void reduce_row(float& peak, double& squares, bool& bad) {
    float b = bad ? 1.f : 0.f;
#pragma unroll
    for (int o = 1; o < (G < 64 ? G : 64); o *= 2) {
        peak = fmaxf(peak, __shfl_xor(peak, o));
        squares += __shfl_xor(squares, o);
        b = fmaxf(b, __shfl_xor(b, o));
    }
    if constexpr (G > 64) {
        __shared__ float s_peak[G / 64], s_bad[G / 64];
        __shared__ double s_squares[G / 64];
        if ((threadIdx.x & 63) == 0) {
            s_peak[threadIdx.x >> 6] = peak;
            s_bad[threadIdx.x >> 6] = b;
            s_squares[threadIdx.x >> 6] = squares;
        }
        __syncthreads();
        peak = b = 0.f;
        squares = 0.0;
#pragma unroll
        for (int w = 0; w < G / 64; ++w) {
            peak = fmaxf(peak, s_peak[w]);
            b = fmaxf(b, s_bad[w]);
            squares += s_squares[w];
        }
    }
    bad = b != 0.f;
}

template <bool UNIT>
__device__ inline void take(float x, float& peak, double& squares, bool& bad) {
    bad = bad || !(fabsf(x) <= 3.402823466e38f);
    if constexpr (UNIT) squares = fma((double)x, (double)x, squares);
    else peak = fmaxf(peak, fabsf(x));
}

// 8 elements of a row from column c on; 0 behind the end.
template <typename T>
__device__ inline void load_eight(const T* row, uint32_t c, uint32_t cols, T (&v)[8]) {
    if (c + 8 <= cols) __builtin_memcpy(v, row + c, sizeof(v));
    else
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = c + i < cols ? row[c + i] : (T)0.f;
}

__device__ inline void store_eight(int8_t* row, uint32_t c, uint32_t cols, const int8_t (&q)[8]) {
    if (c + 8 <= cols) __builtin_memcpy(row + c, q, 8);
    else
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < cols) row[c + i] = q[i];
}

// G lanes a row, RUNS runs of 8 elements a lane (cols <= 8 G RUNS), ROWS rows a group of lanes one after the other, all loaded at once.
template <typename T, int G, int RUNS, int ROWS, bool UNIT>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const T* __restrict__ x, uint64_t rows, uint32_t cols, uint64_t stride,
                                                            int8_t* __restrict__ codes, float* __restrict__ scales) {
    static_assert(G <= 64 || ROWS == 1, "one row a workgroup where its waves share it");
    constexpr int PER = 256 / G;
    const uint32_t at = threadIdx.x % G;
    T v[ROWS][RUNS][8];
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
        const uint64_t r = ((uint64_t)blockIdx.x * ROWS + k) * PER + threadIdx.x / G;
#pragma unroll
        for (int j = 0; j < RUNS; ++j) load_eight(x + min(r, rows - 1) * stride, (j * G + at) * 8, cols, v[k][j]);
    }
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
        const uint64_t r = ((uint64_t)blockIdx.x * ROWS + k) * PER + threadIdx.x / G;
        float peak = 0.f, scale;
        double squares = 0.0;
        bool bad = false;
#pragma unroll
        for (int j = 0; j < RUNS; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) take<UNIT>((float)v[k][j][i], peak, squares, bad);
        reduce_row<G>(peak, squares, bad);
        const Quotient quotient(peak, squares, bad, UNIT, scale);
        if (r >= rows) continue;
        if (at == 0) scales[r] = scale;
#pragma unroll
        for (int j = 0; j < RUNS; ++j) {
            int8_t q[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) q[i] = (int8_t)quotient.code((float)v[k][j][i]);
            store_eight(codes + r * cols, (j * G + at) * 8, cols, q);
        }
    }
}

// Longer rows: a workgroup a row, read twice (the second time from the caches).
template <typename T, bool UNIT>
__global__ __launch_bounds__(256) void quantize_long_rows_kernel(const T* __restrict__ x, uint32_t cols, uint64_t stride,
                                                                 int8_t* __restrict__ codes, float* __restrict__ scales) {
    const uint64_t r = blockIdx.x;
    const T* row = x + r * stride;
    float peak = 0.f, scale;
    double squares = 0.0;
    bool bad = false;
    for (uint32_t c = threadIdx.x * 8; c < cols; c += 2048) {
        T v[8];
        load_eight(row, c, cols, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) take<UNIT>((float)v[i], peak, squares, bad);
    }
    reduce_row<256>(peak, squares, bad);
    const Quotient quotient(peak, squares, bad, UNIT, scale);
    if (threadIdx.x == 0) scales[r] = scale;
    for (uint32_t c = threadIdx.x * 8; c < cols; c += 2048) {
        T v[8];
        load_eight(row, c, cols, v);
        int8_t q[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = (int8_t)quotient.code((float)v[i]);
        store_eight(codes + r * cols, c, cols, q);
    }
}

template <typename T, int G, int RUNS, int ROWS, bool UNIT>
void launch_shape(const T* x, uint64_t rows, uint32_t cols, uint64_t stride, int8_t* codes, float* scales, hipStream_t stream) {
    constexpr uint64_t per = 256 / G * ROWS;
    quantize_rows_kernel<T, G, RUNS, ROWS, UNIT><<<dim3((uint32_t)((rows + per - 1) / per)), dim3(256), 0, stream>>>(x, rows, cols, stride, codes,
                                                                                                                     scales);
}

// As few lanes a row as hold it in 2 to 4 runs; several short rows a lane where there are enough rows to fill the chip anyway.
template <typename T, bool UNIT>
hipError_t launch_type(const void* data, uint64_t rows, uint32_t cols, uint64_t stride, int8_t* codes, float* scales, hipStream_t stream) {
    const T* x = (const T*)data;
    const bool many = rows >= 65536;
    if (cols <= 128 && many) launch_shape<T, 16, 1, 4, UNIT>(x, rows, cols, stride, codes, scales, stream);
    else if (cols <= 128) launch_shape<T, 16, 1, 1, UNIT>(x, rows, cols, stride, codes, scales, stream);
    else if (cols <= 512 && many) launch_shape<T, 64, 1, 4, UNIT>(x, rows, cols, stride, codes, scales, stream);
    else if (cols <= 512) launch_shape<T, 64, 1, 1, UNIT>(x, rows, cols, stride, codes, scales, stream);
    else if (cols <= 1024) launch_shape<T, 64, 2, 1, UNIT>(x, rows, cols, stride, codes, scales, stream);
    else if (cols <= 2048) launch_shape<T, 256, 1, 1, UNIT>(x, rows, cols, stride, codes, scales, stream);
    else if (cols <= 4096) launch_shape<T, 256, 2, 1, UNIT>(x, rows, cols, stride, codes, scales, stream);
    else if (cols <= 8192) launch_shape<T, 256, 4, 1, UNIT>(x, rows, cols, stride, codes, scales, stream);
    else quantize_long_rows_kernel<T, UNIT><<<dim3((uint32_t)rows), dim3(256), 0, stream>>>(x, cols, stride, codes, scales);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize_rows(const void* x, uint32_t dtype, uint64_t rows, uint32_t cols, uint64_t stride, bool unit, int8_t* codes,
                                float* scales, hipStream_t stream) {
    if (rows == 0) return hipSuccess;
    if (dtype == TYPE_F16)
        return unit ? launch_type<f16_t, true>(x, rows, cols, stride, codes, scales, stream)
                    : launch_type<f16_t, false>(x, rows, cols, stride, codes, scales, stream);
    if (dtype == TYPE_BF16)
        return unit ? launch_type<bf16_t, true>(x, rows, cols, stride, codes, scales, stream)
                    : launch_type<bf16_t, false>(x, rows, cols, stride, codes, scales, stream);
    return unit ? launch_type<float, true>(x, rows, cols, stride, codes, scales, stream)
                : launch_type<float, false>(x, rows, cols, stride, codes, scales, stream);
}

}  // namespace dessert
