// Global gradient norms over many tensors and clipping, on gfx950.
//
//   norm_k = sqrt(sum of g^2 over all tensors of worker k)
//   c_k = min(1, max_norm / (norm_k + 1e-6)),  g <- c_k g
//
// The tensors are cut into chunks of at most kChunk elements, listed worker by
// worker in a table in device memory.  Two streaming passes over the chunks, one
// grid row a worker: the squares (fp32 per 8 values, fp64 beyond, the reductions of
// reduce.hpp), then the scaling, in which every workgroup adds its worker's sums up
// again as the AdamW step does, so that no kernel stands between the passes.  Bound
// by HBM: the gradients are read twice and written once.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "adamw_kernels.hpp"
#include "matrix_view.hpp"

namespace autoloco {

constexpr int kChunk = 16384;

// One chunk of a gradient tensor: n elements at grad, to packed (or grad itself).
struct GradChunk {
    void* grad;
    float* packed;
    int32_t n;
    int32_t bf16;
    int64_t unused;
};

struct ClipArgs {
    const GradChunk* chunks;
    int64_t first[kMaxK + 1];   // each worker's first chunk
    double* partials;           // [workers][gridDim.x]
    double max_norm;
    double* sums;               // [workers] squared norms
    double* host_sums;          // the same in coherent host memory, or null
    float* norms;               // [workers], or null
};

template <bool BF16>
__device__ __forceinline__ double chunk_squares(const GradChunk& c) {
    double t = 0.0;
    for (int i = threadIdx.x * 8; i < c.n; i += kBlock * 8) {
        float v[8];
        load8<BF16>(v, c.grad, i, c.n);
        float s = v[0] * v[0];
#pragma unroll
        for (int j = 1; j < 8; ++j) s = __builtin_fmaf(v[j], v[j], s);
        t += (double)s;
    }
    return t;
}

[[maybe_unused]] static __global__ void __launch_bounds__(kBlock) tensor_norm_kernel(ClipArgs a) {
    const int k = blockIdx.y;
    double acc[1] = {0.0};
    for (int64_t i = a.first[k] + blockIdx.x; i < a.first[k + 1]; i += gridDim.x) {
        const GradChunk c = a.chunks[i];
        acc[0] += c.bf16 ? chunk_squares<true>(c) : chunk_squares<false>(c);
    }
    const double part = block_reduce<1, kBlock>(acc);
    if (threadIdx.x == 0) a.partials[(int64_t)k * gridDim.x + blockIdx.x] = part;
}

template <bool BF16>
__device__ __forceinline__ void chunk_scale(const GradChunk& c, float coef) {
    for (int i = threadIdx.x * 8; i < c.n; i += kBlock * 8) {
        float v[8];
        load8<BF16>(v, c.grad, i, c.n);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= coef;
        if (c.packed != nullptr)
            store8<false>(c.packed, i, c.n, v);
        else
            store8<BF16>(c.grad, i, c.n, v);
    }
}

[[maybe_unused]] static __global__ void __launch_bounds__(kBlock) tensor_clip_kernel(ClipArgs a) {
    __shared__ double total;
    const int k = blockIdx.y;
    double t[1] = {0.0};
    for (int b = threadIdx.x; b < (int)gridDim.x; b += kBlock) t[0] += a.partials[(int64_t)k * gridDim.x + b];
    const double sum = block_reduce<1, kBlock>(t);
    if (threadIdx.x == 0) {
        total = sum;
        if (blockIdx.x == 0) {
            a.sums[k] = sum;
            if (a.host_sums != nullptr) a.host_sums[k] = sum;
            if (a.norms != nullptr) a.norms[k] = (float)sqrt(sum);
        }
    }
    __syncthreads();
    const float coef = a.max_norm > 0.0 ? clip_coef(total, a.max_norm) : 1.0f;
    for (int64_t i = a.first[k] + blockIdx.x; i < a.first[k + 1]; i += gridDim.x) {
        const GradChunk c = a.chunks[i];
        if (c.packed == nullptr && coef == 1.0f) return;   // nothing to change in place
        if (c.bf16)
            chunk_scale<true>(c, coef);
        else
            chunk_scale<false>(c, coef);
    }
}

hipError_t launch_tensor_norm(int workers, int blocks, const ClipArgs& a, hipStream_t s);
hipError_t launch_tensor_clip(int workers, int blocks, const ClipArgs& a, hipStream_t s);

}  // namespace autoloco
