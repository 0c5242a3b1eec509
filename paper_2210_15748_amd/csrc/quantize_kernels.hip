// Rows of numbers to int8 with one scale a row.
//   largest magnitude: scale = max|x| / 127 in 32 bits, code = x / scale
//   unit norm:         scale = |x| / 127, code = 127 x / |x|
// each code the nearest integer to the real quotient, ties to even.  Quotients are formed in 64 bits from a reciprocal (one
// multiplication an element); one that comes out within 2^-20 of a half is divided for real, which makes exact ties and
// their neighbours come out as the formula says.  A row with an infinity or NaN gets codes 0 and scale NaN.
#include "kernels.hpp"
#include "number_formats.hpp"

namespace dessert {

namespace {

// Nearest integer to num * x / den, ties to even; recip = num / den rounded.
__device__ inline int nearest(double x, double num, double den, double recip) {
    double t = x * recip;
    const double half = fabs(t - floor(t) - 0.5);
    if (half < 0x1p-20) t = num * x / den;   // num * x is exact: x has at most 24 bits, num 7
    return (int)rint(t);
}

// G lanes a row (a power of two; 64 and fewer: part of a wave, else a workgroup of G), runs of 8 elements a lane.
template <typename T, int G>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const T* __restrict__ x, uint64_t rows, uint32_t cols, uint64_t stride,
                                                            bool unit, int8_t* __restrict__ codes, float* __restrict__ scales) {
    constexpr int PER = 256 / G;
    const uint32_t at = threadIdx.x % G;
    const uint64_t r = (uint64_t)blockIdx.x * PER + threadIdx.x / G;
    const bool live = r < rows;
    const T* row = x + (live ? r : 0) * stride;
    float peak = 0.f;
    double sq = 0.0;
    bool finite = true;
    for (uint32_t c = at * 8; c < cols && live; c += G * 8) {
        float v[8];
        if (c + 8 <= cols) load_run<T, 8>(row + c, v);
        else
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = c + i < cols ? (float)row[c + i] : 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            finite = finite && fabsf(v[i]) <= 3.402823466e38f;
            peak = fmaxf(peak, fabsf(v[i]));
            sq += (double)v[i] * (double)v[i];
        }
    }
    // over the row's lanes
    float bad = finite ? 0.f : 1.f;
    for (int o = 1; o < (G < 64 ? G : 64); o *= 2) {
        peak = fmaxf(peak, __shfl_xor(peak, o));
        sq += __shfl_xor(sq, o);
        bad = fmaxf(bad, __shfl_xor(bad, o));
    }
    if constexpr (G > 64) {
        __shared__ float s_peak[4], s_bad[4];
        __shared__ double s_sq[4];
        if ((threadIdx.x & 63) == 0) {
            s_peak[threadIdx.x >> 6] = peak;
            s_bad[threadIdx.x >> 6] = bad;
            s_sq[threadIdx.x >> 6] = sq;
        }
        __syncthreads();
        peak = fmaxf(fmaxf(s_peak[0], s_peak[1]), fmaxf(s_peak[2], s_peak[3]));
        bad = fmaxf(fmaxf(s_bad[0], s_bad[1]), fmaxf(s_bad[2], s_bad[3]));
        sq = s_sq[0] + s_sq[1] + s_sq[2] + s_sq[3];
    }
    if (!live) return;
    const double norm = sqrt(sq);
    const float scale = bad != 0.f ? __builtin_nanf("") : unit ? (float)(norm / 127.0) : peak / 127.f;
    const double num = unit ? 127.0 : 1.0, den = unit ? norm : (double)scale;
    const bool zero = bad != 0.f || den == 0.0;
    const double recip = zero ? 0.0 : num / den;
    if (at == 0) scales[r] = scale;
    int8_t* out = codes + r * cols;
    for (uint32_t c = at * 8; c < cols; c += G * 8) {
        int8_t q[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float v = c + i < cols && !zero ? (float)row[c + i] : 0.f;
            const int n = zero ? 0 : nearest(v, num, den, recip);
            q[i] = (int8_t)(n > 127 ? 127 : n < -127 ? -127 : n);
        }
        if (c + 8 <= cols) __builtin_memcpy(out + c, q, 8);
        else
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c + i < cols) out[c + i] = q[i];
    }
}

template <typename T>
hipError_t launch_type(const void* x, uint64_t rows, uint32_t cols, uint64_t stride, bool unit, int8_t* codes, float* scales,
                       hipStream_t stream) {
    if (cols <= 128) {
        quantize_rows_kernel<T, 16><<<dim3((uint32_t)((rows + 15) / 16)), dim3(256), 0, stream>>>(
            (const T*)x, rows, cols, stride, unit, codes, scales);
    } else if (cols <= 1024) {
        quantize_rows_kernel<T, 64><<<dim3((uint32_t)((rows + 3) / 4)), dim3(256), 0, stream>>>(
            (const T*)x, rows, cols, stride, unit, codes, scales);
    } else {
        quantize_rows_kernel<T, 256><<<dim3((uint32_t)rows), dim3(256), 0, stream>>>(
            (const T*)x, rows, cols, stride, unit, codes, scales);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize_rows(const void* x, uint32_t dtype, uint64_t rows, uint32_t cols, uint64_t stride, bool unit, int8_t* codes,
                                float* scales, hipStream_t stream) {
    if (rows == 0) return hipSuccess;
    if (dtype == TYPE_F16) return launch_type<f16_t>(x, rows, cols, stride, unit, codes, scales, stream);
    if (dtype == TYPE_BF16) return launch_type<bf16_t>(x, rows, cols, stride, unit, codes, scales, stream);
    return launch_type<float>(x, rows, cols, stride, unit, codes, scales, stream);
}

}  // namespace dessert
