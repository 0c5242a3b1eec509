// Element types of the row operators (dtype codes as in dessert.h) and their conversion from 32-bit floats.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dessert {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef _Float16 f16_t;
typedef __bf16 bf16_t;

constexpr uint32_t TYPE_F16 = 1, TYPE_BF16 = 2, TYPE_F32 = 3;

// N elements to any element's address (16-byte accesses need no alignment on this hardware)
template <typename T, int N>
__device__ inline void store_run(T* p, const float (&x)[N]) {
    T v[N];
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = (T)x[i];   // round to nearest, ties to even
    __builtin_memcpy(p, v, sizeof(v));
}

}  // namespace dessert
