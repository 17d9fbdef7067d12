// Matrices with a row stride whose rows may begin at any element, and the loads
// and stores of the kernels that read and write them.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "round_kernels.hpp"

namespace autoloco {

struct MatrixView {
    const void* data;
    int64_t rows, cols, stride;   // in elements
};
struct MatrixOut {
    void* data;
    int64_t rows, cols, stride;
};

// 16 bytes at an address that is a multiple of 2 or 4 only: the memory unit takes
// them in one access.
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));

template <bool BF16>
__device__ __forceinline__ float load_one(const void* p, int64_t i) {
    if constexpr (BF16)
        return __uint_as_float((uint32_t)static_cast<const uint16_t*>(p)[i] << 16);
    else
        return static_cast<const float*>(p)[i];
}
template <bool BF16>
__device__ __forceinline__ void store_one(void* p, int64_t i, float v) {
    if constexpr (BF16)
        static_cast<uint16_t*>(p)[i] = (uint16_t)bf16_rne(v);
    else
        static_cast<float*>(p)[i] = v;
}

// Elements i..i+7 of a row of n (those past n: fill).
template <bool BF16>
__device__ __forceinline__ void load8(float (&x)[8], const void* row, int64_t i, int64_t n, float fill = 0.f) {
    if (i + 8 <= n) {
        if constexpr (BF16) {
            const u32x4_any w = *reinterpret_cast<const u32x4_any*>(static_cast<const uint16_t*>(row) + i);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x[2 * j] = bf16_lo(w[j]);
                x[2 * j + 1] = bf16_hi(w[j]);
            }
        } else {
            const u32x4_any* p = reinterpret_cast<const u32x4_any*>(static_cast<const float*>(row) + i);
            const u32x4_any a = p[0], b = p[1];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x[j] = __uint_as_float(a[j]);
                x[4 + j] = __uint_as_float(b[j]);
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = i + j < n ? load_one<BF16>(row, i + j) : fill;
    }
}
template <bool BF16>
__device__ __forceinline__ void store8(void* row, int64_t i, int64_t n, const float (&x)[8]) {
    if (i + 8 <= n) {
        if constexpr (BF16) {
            u32x4_any w;
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = bf16_pack(x[2 * j], x[2 * j + 1]);
            *reinterpret_cast<u32x4_any*>(static_cast<uint16_t*>(row) + i) = w;
        } else {
            u32x4_any* p = reinterpret_cast<u32x4_any*>(static_cast<float*>(row) + i);
            u32x4_any a, b;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                a[j] = __float_as_uint(x[j]);
                b[j] = __float_as_uint(x[4 + j]);
            }
            p[0] = a;
            p[1] = b;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (i + j < n) store_one<BF16>(row, i + j, x[j]);
    }
}

}  // namespace autoloco
