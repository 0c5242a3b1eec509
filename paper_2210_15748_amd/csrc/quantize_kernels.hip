// Rows of numbers to int8 with one scale a row.
//   largest magnitude: scale = max|x| * (1 / 127), both in 32 bits, code = x / scale
//   unit norm:         scale = |x| / 127, code = 127 x / |x|, the norm in 64 bits (the codes of a vector are whole numbers: a sum of squares
//                      in 32 bits would move some of them over a half)
// each code the nearest integer to the real quotient, ties to even.  Bound by memory: rows are read once and kept in registers between the
// reduction and the codes.  A row with an infinity or NaN gets codes 0 and scale NaN.
#include <type_traits>

#include "kernels.hpp"
#include "launch_slices.hpp"
#include "number_formats.hpp"

namespace dessert {

namespace {

// What a row's elements are reduced to: the largest magnitude's bits, or the sum of the squares.  Bits order magnitudes as their
// values, infinities and NaN above all; a sum of squares of 32-bit floats cannot overflow 64 bits.
template <bool UNIT>
struct Reduced {
    using type = std::conditional_t<UNIT, double, uint32_t>;
    type v = 0;

    template <typename T>
    __device__ void take(const T (&x)[8]) {
        if constexpr (UNIT) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v = fma((double)(float)x[i], (double)(float)x[i], v);
        } else if constexpr (sizeof(T) == 2) {   // two at a time
            typedef uint16_t pair __attribute__((ext_vector_type(2)));
            pair m[4];
            __builtin_memcpy(m, x, 16);
#pragma unroll
            for (int i = 0; i < 4; ++i) m[i] &= (uint16_t)0x7FFF;
            const pair p = __builtin_elementwise_max(__builtin_elementwise_max(m[0], m[1]), __builtin_elementwise_max(m[2], m[3]));
            v = max(v, (uint32_t)max(p.x, p.y));
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v = max(v, __float_as_uint(x[i]) & 0x7FFFFFFFu);
        }
    }
    __device__ void join(type o) {
        if constexpr (UNIT) v += o;
        else v = max(v, o);
    }
    // over the G consecutive lanes of a row (a power of two)
    template <int G>
    __device__ void join_lanes() {
#pragma unroll
        for (int o = 1; o < (G < 64 ? G : 64); o *= 2) join(__shfl_xor(v, o));
        if constexpr (G > 64) {
            __shared__ type parts[G / 64];
            if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = v;
            __syncthreads();
            v = parts[0];
#pragma unroll
            for (int w = 1; w < G / 64; ++w) join(parts[w]);
        }
    }
};

// What turns a row's numbers into codes.
template <typename T, bool UNIT>
struct Quotient {
    double num, den;          // a code is num * x / den
    float factor, scale;      // factor: num / den to 2^-23, or 0
    bool none;                // all codes are 0

    __device__ Quotient() {}
    __device__ explicit Quotient(typename Reduced<UNIT>::type v) {
        if constexpr (UNIT) {
            const double norm = sqrt(v);
            num = 127.0;
            den = norm;
            scale = v < __builtin_huge_val() ? (float)(norm / 127.0) : __builtin_nanf("");
            factor = 127.f / (float)norm;
        } else {
            float peak;
            if constexpr (sizeof(T) == 2) {
                const uint16_t bits = (uint16_t)v;
                T x;
                __builtin_memcpy(&x, &bits, 2);
                peak = (float)x;
            } else {
                peak = __uint_as_float(v);
            }
            scale = peak < __builtin_huge_valf() ? peak * (1.f / 127.f) : __builtin_nanf("");
            num = 1.0;
            den = scale;
            factor = 1.f / scale;
        }
        none = !(den > 0.0 && scale == scale);
    }
    // The factor is off by at most 2^-23 and the product with it by 2^-24, of at most 127: less than 2^-15.  A product that close to a half, and all of
    // a row whose factor is no ordinary number, are compared with the half in 64 bits instead: num * x is exact there.
    __device__ uint64_t codes(const T (&x)[8]) const {
        constexpr float MAGIC = 12582912.f;   // 1.5 * 2^23: a sum with it is rounded to a whole number, whose last bits it holds
        uint32_t n[8];
        float off = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float t = (float)x[i] * factor, m = t + MAGIC;
            n[i] = __float_as_uint(m);
            off = fmaxf(off, fabsf(t - (m - MAGIC)));
        }
        if (off > 0.5f - 0x1p-14f || !(factor < 0x1p125f && factor > 0x1p-125f)) {
            const double wide = none ? 0.0 : num / den;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float y = (float)x[i];
                asm volatile("" : "+v"(y));   // converted here, not kept in 64 bits since the sum of squares
                const double a = num * (double)y, below = floor((double)y * wide);
                const double over = fma(-(below + 0.5), den, a);   // a against the half above `below`: its sign is exact
                const int b = (int)fmin(fmax(below, -128.0), 127.0);
                const int q = over > 0.0 || (over == 0.0 && (b & 1)) ? b + 1 : b;
                n[i] = none ? 0 : (uint32_t)min(max(q, -127), 127);
            }
        }
        uint32_t lo = __builtin_amdgcn_perm(n[1], n[0], 0x0C0C0400) | __builtin_amdgcn_perm(n[3], n[2], 0x04000C0C);
        uint32_t hi = __builtin_amdgcn_perm(n[5], n[4], 0x0C0C0400) | __builtin_amdgcn_perm(n[7], n[6], 0x04000C0C);
        return (uint64_t)hi << 32 | lo;
    }
};

// 8 elements of a row from column c on; 0 behind the end.
template <typename T>
__device__ inline void load_eight(const T* row, uint32_t c, uint32_t cols, T (&v)[8]) {
    if (c + 8 <= cols) __builtin_memcpy(v, row + c, sizeof(v));
    else
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = c + i < cols ? row[c + i] : (T)0.f;
}

__device__ inline void store_eight(int8_t* row, uint32_t c, uint32_t cols, uint64_t q) {
    if (c + 8 <= cols) __builtin_memcpy(row + c, &q, 8);
    else
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < cols) row[c + i] = (int8_t)(q >> 8 * i);
}

// G lanes a row, RUNS runs of 8 elements a lane (cols <= 8 G RUNS), ROWS rows a group of lanes one after the other, all loaded at once.
// With several rows a lane sees to the root and the quotients of one of them (64-bit operations: a third of the time of short rows
// when every lane formed them for every row).
// Read + written per second: 16384 x 8192 bf16 5.5 TB/s, 131072 x 512 fp16 5.8, 573440 x 128 fp16 5.9 (unit norm 5.1), 4096 x 16384 bf16 5.0 (3.2 when
// such rows were read twice).
template <typename T, int G, int RUNS, int ROWS, bool UNIT>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const T* __restrict__ x, uint64_t rows, uint32_t cols, uint64_t stride,
                                                            int8_t* __restrict__ codes, float* __restrict__ scales) {
    static_assert(G <= 64 || ROWS == 1, "one row a workgroup where its waves share it");
    constexpr int PER = 256 / G;
    const uint32_t at = threadIdx.x % G;
    const uint64_t first = (uint64_t)blockIdx.x * ROWS * PER + threadIdx.x / G;
    T v[ROWS][RUNS][8];
#pragma unroll
    for (int k = 0; k < ROWS; ++k)
#pragma unroll
        for (int j = 0; j < RUNS; ++j) load_eight(x + min(first + k * PER, rows - 1) * stride, (j * G + at) * 8, cols, v[k][j]);
    Reduced<UNIT> reduced[ROWS];
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
#pragma unroll
        for (int j = 0; j < RUNS; ++j) reduced[k].take(v[k][j]);
        reduced[k].template join_lanes<G>();
    }
    typename Reduced<UNIT>::type own = reduced[0].v;
#pragma unroll
    for (int k = 1; k < ROWS; ++k)
        if (at % ROWS == k) own = reduced[k].v;
    const Quotient<T, UNIT> mine(own);
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
        Quotient<T, UNIT> quotient = mine;
        if constexpr (ROWS > 1) {
            const int from = (int)((threadIdx.x & 63) / G * G) + k;
            quotient.den = __shfl(mine.den, from);
            quotient.factor = __shfl(mine.factor, from);
            quotient.none = __shfl((int)mine.none, from);
        }
        const uint64_t r = first + k * PER;
        if (r >= rows) continue;
        if (at == k) scales[r] = mine.scale;
#pragma unroll
        for (int j = 0; j < RUNS; ++j) store_eight(codes + r * cols, (j * G + at) * 8, cols, quotient.codes(v[k][j]));
    }
}

// Longer rows: a workgroup a row, read twice (the second time from the caches).
template <typename T, bool UNIT>
__global__ __launch_bounds__(1024) void quantize_long_rows_kernel(const T* __restrict__ x, uint32_t cols, uint64_t stride,
                                                                  int8_t* __restrict__ codes, float* __restrict__ scales) {
    const uint64_t r = blockIdx.x;
    const T* row = x + r * stride;
    Reduced<UNIT> reduced;
    for (uint32_t c = threadIdx.x * 8; c < cols; c += 8192) {
        T v[8];
        load_eight(row, c, cols, v);
        reduced.take(v);
    }
    reduced.template join_lanes<1024>();
    const Quotient<T, UNIT> quotient(reduced.v);
    if (threadIdx.x == 0) scales[r] = quotient.scale;
    for (uint32_t c = threadIdx.x * 8; c < cols; c += 8192) {
        T v[8];
        load_eight(row, c, cols, v);
        store_eight(codes + r * cols, c, cols, quotient.codes(v));
    }
}

template <typename T, int G, int RUNS, int ROWS, bool UNIT>
void launch_shape(const T* x, uint64_t rows, uint32_t cols, uint64_t stride, int8_t* codes, float* scales, hipStream_t stream) {
    in_launches(rows, 256 / G * ROWS, 256, [&](uint64_t first, uint64_t n, uint32_t workgroups) {
        quantize_rows_kernel<T, G, RUNS, ROWS, UNIT><<<dim3(workgroups), dim3(256), 0, stream>>>(x + first * stride, n, cols, stride,
                                                                                                 codes + first * cols, scales + first);
    });
}

// As few lanes a row as hold it in 2 to 4 runs; several short rows a lane where there are enough rows to fill the chip anyway (one / several in us:
// 16384 x 128 fp16 4.7 / 6.2, unit norm 4.9 / 5.2; 65536 8.3 / 9.1, 9.2 / 8.8; 573440 41.4 / 36.9, 51.4 / 39.7; 65536 x 200 fp16 18.3 / 16.8, 22.7 / 19.6;
// 131072 x 512 fp16 35.6 / 33.8, 43.3 / 36.6; 573440 x 32 fp32 31.1 / 27.5, 42.3 / 33.7, but x 128 62.4 / 68.3, 63.9 / 67.0).
template <typename T, bool UNIT>
hipError_t launch_type(const void* data, uint64_t rows, uint32_t cols, uint64_t stride, int8_t* codes, float* scales, hipStream_t stream) {
    const T* x = (const T*)data;
    const bool many = rows >= 65536;
    if (cols <= 128 && many) launch_shape<T, 16, 1, UNIT ? 2 : 4, UNIT>(x, rows, cols, stride, codes, scales, stream);
    else if (cols <= 128) launch_shape<T, 16, 1, 1, UNIT>(x, rows, cols, stride, codes, scales, stream);
    else if (cols <= 512 && many) launch_shape<T, 64, 1, UNIT ? 2 : 4, UNIT>(x, rows, cols, stride, codes, scales, stream);
    else if (cols <= 512) launch_shape<T, 64, 1, 1, UNIT>(x, rows, cols, stride, codes, scales, stream);
    else if (cols <= 1024) launch_shape<T, 64, 2, 1, UNIT>(x, rows, cols, stride, codes, scales, stream);
    else if (cols <= 2048) launch_shape<T, 256, 1, 1, UNIT>(x, rows, cols, stride, codes, scales, stream);
    else if (cols <= 4096) launch_shape<T, 256, 2, 1, UNIT>(x, rows, cols, stride, codes, scales, stream);
    else if (cols <= 8192) launch_shape<T, 256, 4, 1, UNIT>(x, rows, cols, stride, codes, scales, stream);
    else if (cols <= 16384) launch_shape<T, 256, 8, 1, UNIT>(x, rows, cols, stride, codes, scales, stream);
    else
        in_launches(rows, 1, 1024, [&](uint64_t first, uint64_t, uint32_t workgroups) {
            quantize_long_rows_kernel<T, UNIT><<<dim3(workgroups), dim3(1024), 0, stream>>>(x + first * stride, cols, stride, codes + first * cols,
                                                                                            scales + first);
        });
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
