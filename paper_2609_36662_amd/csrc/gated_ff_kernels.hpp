// The gated feed-forward block on gfx950, in bf16.
//
//   g = x Wg^T,  u = x Wu^T,  h = act(g) u,  y = h Wd^T
//   dh = dy Wd,  dg = dh u act'(g),  du = dh act(g)
//   dx = dg Wg + du Wu,  dWg = dg^T x,  dWu = du^T x,  dWd = dy^T h
//
// Both projections are one product, whose tiles take as many columns of g as of u, so
// that the activation and the product are done on the sums in fp32.  dh exists only as
// the sums of a product whose epilogue reads g and u and writes dg and du.  dx adds both
// its terms up in one sum.  h, and of training g and u, dg and du, are rounded to bf16,
// since they are the next products' operands; everything else is fp32 up to the outputs' rounding.
// (y and dWd are 0.235 % of their norm off by it, where their own rounding alone is 0.166; dx, dWg
// and dWu 0.30 %.)
//
// Bound by the matrix cores for many rows and by rounds of tiles that are not full.  Among
// other calls (medians; cards and runs lie up to 5 % to either side): 2,048 rows of 4,096 with
// 11,008 between, both projections 355 us (1.04 PFLOP/s, cores busy 60 %) and the last product 181
// (1.02); 4,096 rows of 2,048 with 5,632 between, g, u and h kept 204 us (0.93), y 92 us (1.03), dh
// 136 us (0.69; g and u read, dg and du written), dx 183 us (1.03), each weights' gradient 107 us
// (0.88: 176 tiles of 256 on 256 units; in a loop over the same operands 89 us, in fp32, whose
// words are stored one by one, 116).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "product_tiles.hpp"

namespace autoloco {

constexpr int kSilu = 0, kGelu = 1;

// act(g) and its derivative.
template <int ACT>
__device__ __forceinline__ void activate(float g, float& a, float& slope) {
    if constexpr (ACT == kSilu) {
        const float s = 1.f / (1.f + __expf(-g));
        a = g * s;
        slope = s * (1.f + g * (1.f - s));
    } else {
        const float cdf = 0.5f * erfcf(g * -0.70710678f);   // as exact far below zero as above
        a = g * cdf;
        slope = cdf + g * __expf(-0.5f * g * g) * 0.39894228f;
    }
}

// h = act(g) u, and g and u themselves if they are kept.
template <int ACT>
struct GateEpilogue {
    MatrixOut h, gate, up;   // gate, up: data null, or both kept
    typedef Nothing Read;
    __device__ __forceinline__ Read load(int64_t, int64_t, int) const { return {}; }
    __device__ __forceinline__ void operator()(int64_t m, int64_t n, const float (&g)[8], const float (&u)[8], int count, Read) const {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float a, slope;
            activate<ACT>(g[i], a, slope);
            v[i] = a * u[i];
        }
        store_piece(static_cast<uint16_t*>(h.data) + m * h.stride + n, pack8(v), count);
        if (gate.data != nullptr) {
            store_piece(static_cast<uint16_t*>(gate.data) + m * gate.stride + n, pack8(g), count);
            store_piece(static_cast<uint16_t*>(up.data) + m * up.stride + n, pack8(u), count);
        }
    }
};

// dg = dh u act'(g) and du = dh act(g); they may lie where g and u do: whoever writes an
// element is who read it.
template <int ACT>
struct GateGradEpilogue {
    MatrixView gate, up;
    MatrixOut dgate, dup;
    struct Read {
        u32x4 gate, up;
    };
    __device__ __forceinline__ Read load(int64_t m, int64_t n, int count) const {
        return {load_piece(static_cast<const uint16_t*>(gate.data) + m * gate.stride + n, count),
                load_piece(static_cast<const uint16_t*>(up.data) + m * up.stride + n, count)};
    }
    __device__ __forceinline__ void operator()(int64_t m, int64_t n, const float (&dh)[8], int count, const Read& x) const {
        float g[8], u[8];
        unpack8(g, x.gate);
        unpack8(u, x.up);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float a, slope;
            activate<ACT>(g[i], a, slope);
            g[i] = dh[i] * u[i] * slope;
            u[i] = dh[i] * a;
        }
        store_piece(static_cast<uint16_t*>(dgate.data) + m * dgate.stride + n, pack8(g), count);
        store_piece(static_cast<uint16_t*>(dup.data) + m * dup.stride + n, pack8(u), count);
    }
};

template <bool BF16>
struct StoreEpilogue {
    MatrixOut out;
    typedef Nothing Read;
    __device__ __forceinline__ Read load(int64_t, int64_t, int) const { return {}; }
    __device__ __forceinline__ void operator()(int64_t m, int64_t n, const float (&v)[8], int count, Read) const {
        if constexpr (BF16) {
            store_piece(static_cast<uint16_t*>(out.data) + m * out.stride + n, pack8(v), count);
        } else {
            float* to = static_cast<float*>(out.data) + m * out.stride + n;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < count) to[i] = v[i];
        }
    }
};

// (Both operands across take more registers than two workgroups of tiles of 128 have.)
template <typename E, bool AT, bool BT, int T, bool PAIR, typename Epi>
__global__ void __launch_bounds__(256, BT && T == 2 ? 1 : 2) product_kernel(Terms terms, int64_t rows, int64_t cols, Tiles grid, uint32_t first, Epi epi) {
    uint32_t ti, tj;
    tile_at(first + blockIdx.x, grid, ti, tj);
    product_tile<E, AT, BT, T, PAIR>(terms, ti, tj, [&](const f32x16 (&acc)[T][T], uint8_t* strip, int64_t m0, int64_t n0, uint32_t lane) {
        finish<PAIR>(acc, strip, m0, n0, rows, cols, lane, epi);
    });
}
template <typename E, bool AT, bool BT, int TM, int TN, int ST, bool PAIR, typename Epi>
__global__ void __launch_bounds__(256, tile_groups(TM, TN, ST)) direct_kernel(Terms terms, int64_t rows, int64_t cols, Tiles grid,
                                                                             uint32_t first, Epi epi) {
    uint32_t ti, tj;
    tile_at(first + blockIdx.x, grid, ti, tj);
    direct_tile<E, AT, BT, TM, TN, ST, PAIR>(terms, ti, tj, [&](const auto& acc, uint8_t* strip, int64_t m0, int64_t n0, uint32_t lane) {
        finish<PAIR>(acc, strip, m0, n0, rows, cols, lane, epi);
    });
}

// ------------------------------------------------------------ single tokens --
// Up to 16 rows: a workgroup takes 16 columns of the result (PAIR: of both projections),
// its NW waves the summed axis in turn, joined in LDS in wave order.  A lane takes its
// column's weight and its row of x straight from memory, 8 elements of each, as the 16x16x32
// instruction wants them.  Bound by the weights' way from memory: 13 rows of 4,096 with 11,008
// between 38 and 22 us (4.7 and 4.1 TB/s).  1 row of 2,048 with 5,632 between 14.6 and 8.5 us (3.2 and
// 2.7 TB/s): the first launch's waves make four rounds of loads, each waiting for the one before, and
// the second has 128 workgroups for 256 units.  Whole lines are read at a time; by halves, past the
// caches, the two calls took 26.6 and 80 us for 21.6 and 68.
template <int NW, int U, bool PAIR, typename Epi>
__global__ void __launch_bounds__(NW * 64) tokens_kernel(MatrixView x, Operand w, const uint16_t* w2, uint32_t first, Epi epi) {
    constexpr int R = PAIR ? 2 : 1;
    typedef __bf16 v8 __attribute__((ext_vector_type(8)));
    __shared__ __align__(16) float part[NW][R * 256];
    static_assert(__alignof__(part) >= 16, "stored four at a time");
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int r = lane & 15, q = lane >> 4;
    const int64_t n0 = ((int64_t)first + blockIdx.x) * 16;
    const int64_t wr = n0 + r < w.n ? n0 + r : w.n - 1;
    const uint16_t* from[2] = {w.p + wr * w.stride, PAIR ? w2 + wr * w.stride : nullptr};
    const uint16_t* xr = static_cast<const uint16_t*>(x.data) + (r < x.rows ? r : x.rows - 1) * x.stride;
    f32x4 acc[R] = {};
    // U pieces of 32 on their way at a time
    const int64_t whole = x.cols / (NW * U * 32) * (NW * U * 32);
    auto multiply = [&](u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8, b), __builtin_bit_cast(v8, a), c, 0, 0, 0);
    };
    for (int64_t k = (int64_t)wave * U * 32 + q * 8; k < whole; k += NW * U * 32) {
        u32x4 b[R][U], a[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < R; ++i)
                b[i][u] = __builtin_bit_cast(u32x4, *reinterpret_cast<const u32x4_any*>(from[i] + k + u * 32));
#pragma unroll
        for (int u = 0; u < U; ++u) a[u] = __builtin_bit_cast(u32x4, *reinterpret_cast<const u32x4_any*>(xr + k + u * 32));
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < R; ++i) acc[i] = multiply(a[u], b[i][u], acc[i]);
    }
    for (int64_t k = whole + wave * 32 + q * 8; k - q * 8 < x.cols; k += NW * 32) {
        const u32x4 a = load_piece(xr + k, x.cols - k);
#pragma unroll
        for (int i = 0; i < R; ++i) acc[i] = multiply(a, load_piece(from[i] + k, x.cols - k), acc[i]);
    }
    // a lane has row lane % 16 and the columns 4 (lane / 16) to 4 (lane / 16) + 3
#pragma unroll
    for (int i = 0; i < R; ++i) *reinterpret_cast<f32x4*>(&part[wave][i * 256 + r * 16 + q * 4]) = acc[i];
    __syncthreads();
    for (int t = threadIdx.x; t < (int)x.rows * 2; t += NW * 64) {
        const int m = t >> 1, c = (t & 1) * 8;
        const int64_t left = w.n - n0 - c;
        if (left <= 0) continue;
        float v[R][8];
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[i][e] = part[0][i * 256 + m * 16 + c + e];
#pragma unroll
                for (int k = 1; k < NW; ++k) v[i][e] += part[k][i * 256 + m * 16 + c + e];
            }
        const int count = left < 8 ? (int)left : 8;
        if constexpr (PAIR)
            epi(m, n0 + c, v[0], v[R - 1], count, {});
        else
            epi(m, n0 + c, v[0], count, {});
    }
}

// The block of a call, and its gradients'.
struct GatedFf {
    MatrixView x, w_gate, w_up, w_down;
    MatrixOut y, h, gate, up;
    int activation;
};
struct GatedFfGrad {
    MatrixView x, w_gate, w_up, w_down, h, gate, up, dy;
    MatrixOut dgate, dup, dx, dw_gate, dw_up, dw_down;   // dx, dw_*: data null where not wanted
    bool dw_bf16;
    int activation;
};
hipError_t launch_gated_ff(const GatedFf& f, bool tokens, hipStream_t s);
hipError_t launch_gated_ff_grad(const GatedFfGrad& f, hipStream_t s);

}  // namespace autoloco
