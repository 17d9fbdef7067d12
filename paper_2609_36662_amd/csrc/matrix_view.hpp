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

}  // namespace autoloco
