// Global gradient norms over many tensors and clipping, on gfx950.
//
//   norm_k = sqrt(sum of g^2 over all tensors of worker k)
//   c_k = min(1, max_norm / (norm_k + 1e-6)),  g <- c_k g
//
// The tensors are cut into chunks of at most kChunk elements, listed worker by
// worker in a table in device memory.  Two streaming passes over the chunks, one
// grid row a worker: the squares (in fp64, which costs nothing beside the reading, the reductions of
// reduce.hpp), then the scaling, in which every workgroup adds its worker's sums up
// again as the AdamW step does, so that no kernel stands between the passes.  Bound by
// HBM: the gradients are read twice and written once.  Two workers' 1.1B bf16 gradients
// packed to fp32: 3.2 ms for 17.6 GB (5.5 TB/s; the first pass 6.2, the second, which
// writes twice what it reads, 5.2).  Chunks of 4,096 to 32,768 elements are alike.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "adamw_kernels.hpp"
#include "matrix_view.hpp"

namespace autoloco {

// Elements of a chunk; of a small list, whose chunks are no more than the chip's
// workgroups, fewer.
constexpr int kChunk = 16384, kSmallChunk = 4096;
constexpr int64_t kSmallList = int64_t(16) << 20;

// One chunk of a gradient tensor: n elements at grad, to packed (or grad itself).
struct GradChunk {
    void* grad;
    float* packed;
    int32_t n;
    int32_t bf16;
    int64_t reserved;   // 32 bytes a chunk
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

// Chunks begin at any element: a head of single elements up to the boundary at which
// vectors of V may begin, the vectors (four of a thread's in flight, the last ones too),
// and a tail.  four(whole, head, i, n): vectors i, i + kBlock, i + 2 kBlock, i + 3 kBlock, all there if
// whole (a constant), else those below n; single(j): element j.
template <int V, typename Four, typename Single>
__device__ __forceinline__ void over_chunk(const void* boundary, int element, int n, Four four, Single single) {
    const int off = (int)(reinterpret_cast<uintptr_t>(boundary) / element % V);
    const int head = off == 0 ? 0 : V - off < n ? V - off : n;
    const int vectors = (n - head) / V;
    int i = threadIdx.x;
    for (; i + 3 * kBlock < vectors; i += 4 * kBlock) four(std::true_type{}, head, i, vectors);
    if (i < vectors) four(std::false_type{}, head, i, vectors);
    if (threadIdx.x < 2 * V) {
        const int j = (int)threadIdx.x < head ? (int)threadIdx.x : (int)threadIdx.x + vectors * V;
        if (j < n) single(j);
    }
}

template <bool BF16>
__device__ __forceinline__ double chunk_squares(const GradChunk& c) {
    constexpr int V = BF16 ? 8 : 4;
    double t = 0.0;
    auto add = [&](float g) { t = __builtin_fma((double)g, (double)g, t); };
    over_chunk<V>(
        c.grad, 16 / V, c.n,
        [&](auto whole, int head, int i, int vectors) {
            constexpr int U = 4;
            const u32x4* p = reinterpret_cast<const u32x4*>(static_cast<const char*>(c.grad) + head * (16 / V)) + i;
            u32x4 w[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                w[u] = u32x4{0, 0, 0, 0};
                if (decltype(whole)::value || i + u * kBlock < vectors) w[u] = p[u * kBlock];
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int u = 0; u < U; ++u) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if constexpr (BF16) {
                        add(bf16_lo(w[u][j]));
                        add(bf16_hi(w[u][j]));
                    } else {
                        add(__uint_as_float(w[u][j]));
                    }
                }
            }
        },
        [&](int j) { add(load_one<BF16>(c.grad, j)); });
    return t;
}

[[maybe_unused]] static __global__ void __launch_bounds__(kBlock) tensor_norm_kernel(ClipArgs a) {
    const int k = blockIdx.y;
    double acc[1] = {0.0};
    const int64_t end = a.first[k + 1];
    int64_t i = a.first[k] + blockIdx.x;
    if (i < end) {
        GradChunk c = a.chunks[i];
        for (;;) {
            i += gridDim.x;
            const GradChunk next = a.chunks[i < end ? i : end - 1];   // on its way while this one is worked on
            acc[0] += c.bf16 ? chunk_squares<true>(c) : chunk_squares<false>(c);
            if (i >= end) break;
            c = next;
        }
    }
    const double part = block_reduce<1, kBlock>(acc);
    if (threadIdx.x == 0) a.partials[(int64_t)k * gridDim.x + blockIdx.x] = part;
}

// Four elements a vector, so that neighbouring lanes write neighbouring 16 bytes.
// Nothing is kept in the caches: the gradients pass here for the last time.
template <bool BF16, bool PACK>
__device__ __forceinline__ void chunk_scale(const GradChunk& c, float coef) {
    constexpr int E = BF16 ? 2 : 4, D = PACK ? 4 : E;   // bytes of an element read, written
    void* to = PACK ? static_cast<void*>(c.packed) : c.grad;
    over_chunk<4>(
        to, D, c.n,
        [&](auto whole, int head, int i, int vectors) {
            constexpr int U = 4;
            typedef std::conditional_t<BF16, u32x2_any, u32x4_any> Raw;
            typedef std::conditional_t<D == 2, u32x2r, u32x4> Out;
            const Raw* p = reinterpret_cast<const Raw*>(static_cast<const char*>(c.grad) + head * E) + i;
            Out* o = reinterpret_cast<Out*>(static_cast<char*>(to) + head * D) + i;
            Raw w[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                w[u] = Raw{};
                if (decltype(whole)::value || i + u * kBlock < vectors) w[u] = __builtin_nontemporal_load(p + u * kBlock);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float v[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if constexpr (BF16)
                        v[j] = coef * (j % 2 == 0 ? bf16_lo(w[u][j / 2]) : bf16_hi(w[u][j / 2]));
                    else
                        v[j] = coef * __uint_as_float(w[u][j]);
                }
                Out x;
                if constexpr (D == 2) {
                    x[0] = bf16_pack(v[0], v[1]);
                    x[1] = bf16_pack(v[2], v[3]);
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[j] = __float_as_uint(v[j]);
                }
                if (decltype(whole)::value || i + u * kBlock < vectors) __builtin_nontemporal_store(x, o + u * kBlock);
            }
        },
        [&](int j) { store_one<D == 2>(to, j, coef * load_one<BF16>(c.grad, j)); });
}

// The same for a coefficient that fp32 might not hold, so that huge gradients clipped to a
// tiny norm do not become 0: a power of two that takes half of its exponent first, then the
// rest.  Below 2^-60 only, element by element (two factors in the loop above cost every
// call: two workers' 1.1B gradients 3.20 -> 3.23 ms, 18M 33.8 -> 34.6 us).
__device__ __forceinline__ void chunk_scale_far(const GradChunk& c, double coef) {
    const int half = -ilogb(coef) / 2;
    const float first = (float)ldexp(1.0, -half), second = (float)ldexp(coef, half);
    for (int j = threadIdx.x; j < c.n; j += kBlock) {
        const float v = second * (first * (c.bf16 ? load_one<true>(c.grad, j) : load_one<false>(c.grad, j)));
        if (c.packed != nullptr)
            c.packed[j] = v;
        else if (c.bf16)
            store_one<true>(c.grad, j, v);
        else
            store_one<false>(c.grad, j, v);
    }
}

[[maybe_unused]] static __global__ void __launch_bounds__(kBlock) tensor_clip_kernel(ClipArgs a) {
    __shared__ double total;
    const int k = blockIdx.y;
    // From the last chunk down: what the caches still hold of the first pass comes first.
    const int64_t begin = a.first[k];
    int64_t i = a.first[k + 1] - 1 - blockIdx.x;
    GradChunk c{};
    if (i >= begin) c = a.chunks[i];   // on its way while the sums are added up
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
    const double ratio = a.max_norm > 0.0 ? clip_ratio(total, a.max_norm) : 1.0;
    const float coef = (float)ratio;
    const bool far = ratio > 0.0 && ratio < 0x1p-60;
    if (i < begin) return;
    if (c.packed == nullptr && coef == 1.0f) return;   // nothing to change in place
    for (;;) {
        i -= gridDim.x;
        const GradChunk next = a.chunks[i >= begin ? i : begin];
        if (far) {
            chunk_scale_far(c, ratio);
        } else if (c.packed != nullptr) {
            if (c.bf16)
                chunk_scale<true, true>(c, coef);
            else
                chunk_scale<false, true>(c, coef);
        } else {
            if (c.bf16)
                chunk_scale<true, false>(c, coef);
            else
                chunk_scale<false, false>(c, coef);
        }
        if (i < begin) break;
        c = next;
    }
}

hipError_t launch_tensor_norm(int workers, int blocks, const ClipArgs& a, hipStream_t s);
hipError_t launch_tensor_clip(int workers, int blocks, const ClipArgs& a, hipStream_t s);

}  // namespace autoloco
