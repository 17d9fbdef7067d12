// The orthogonalised inner step of a list of matrices, on gfx950.
//
//   M <- mu M + G,  U = G + mu M or M,  X = U / (|U| + eps)
//   then some times  A = X X^T,  B = b A + c A A,  X <- a X + B X
//   W <- (1 - lr wd) W - lr s X
//
// Every matrix is worked on lying down (X is m x n with m <= n; a tall one is turned as it
// is read and turned back as W is written), so that A is the smaller of the two products.
// Matrices of all shapes go through one launch a product: a tile table, made with the list,
// says which tile of which matrix a workgroup takes.
//
// The products' operands are fp16, each scaled by a power of two so that its values lie in
// the type's normal range (X by about sqrt(n), A and B by 2^11; X's singular values stay below
// 1.21, A's entries below 1.5, B's below 12): sums are fp32.  bf16 would round eight times as
// coarsely, and what is lost of X in one iteration is multiplied by up to 3.4 in each of the
// next.  So X is carried in two parts, hi + lo, of which the products read hi: the sum a X
// keeps 22 bits.  (Relative error of X after five iterations, a decaying spectrum and one
// with 15 of 16 directions a thousandth of the others: 1e-3 and 6e-4; without lo 4e-3 and 4e-2,
// in bf16 2e-2 and 3e-1.)
//
// Bound by the matrix cores for large matrices, by the tiles' first loads and epilogues for
// sums of few steps.  One layer of 4,096 and 11,008 (tiles of 256; us, cores busy; cards lie
// up to 3 % to either side): A 800, 60 %; B 530, 50 %; X 1,730, 51 %; the last X with W 2,170, 38 %; M 406
// (4.7 TB/s) and U 418.  Two times four layers of 768 and 2,048 (tiles of 128): 100, 22 %; 78, 16 %;
// 193, 21 %; 290, 14 %.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "product_tiles.hpp"

namespace autoloco {

constexpr float kNsA = 3.4445f, kNsB = -4.7750f, kNsC = 2.0315f;
constexpr float kScaleA = 2048.f;
constexpr int kMuonParts = 256;    // partial sums of a matrix's norm at most
// A smaller eps counts as this one: beside the norm of anything but zeros (2^-149 at least) neither
// does, and of zeros the scale over it is finite.
constexpr double kMuonLeastEps = 1e-300;

// What a step needs of one matrix, in device memory.
struct MuonMatrix {
    float* param;
    float* momentum;
    const void* grad;
    uint16_t* model;                  // or null
    int64_t param_stride, momentum_stride, grad_stride, model_stride;
    int32_t rows, cols;               // of the tensors
    int32_t m, n, ld, lda;            // X: m x n with rows of ld; A and B: m x m with rows of lda
    int32_t tall, grad_bf16;
    float scale;                      // of X
    float update;                     // s for AUTOLOCO_MUON_RMS, and
    float update_spectral;            // for AUTOLOCO_MUON_SPECTRAL
    int32_t parts;                    // partial sums of the norm
    double* norm;                     // their places
    uint16_t* hi[2];                  // X's first part, read and written in turn
    uint16_t* lo;
    uint16_t* a;
    uint16_t* b;
};
// Every size of tile gives the same bits, so that a matrix's step does not go by what else is
// in its list: multiply-adds are written out, and what is rounded to fp16 is rounded to fp32
// first (here), where the compiler would join a multiply-add and the conversion in some places.
__device__ __forceinline__ float in_fp32(float v) {
    asm("" : "+v"(v));
    return v;
}
// A tile of a matrix, or a piece of its norm, for one workgroup.
struct MuonTile {
    int32_t matrix;
    uint16_t i, j;
};
struct MuonStep {
    const MuonMatrix* matrices;
    const MuonTile* tiles;
    double eps;                       // above zero: at least kMuonLeastEps
    float momentum, decay, lr;        // decay: 1 - lr weight_decay
    int32_t nesterov, spectral, from; // from: which of hi a product reads
};

__device__ __forceinline__ float half_lo(uint32_t w) { return (float)__builtin_bit_cast(_Float16, (uint16_t)w); }
__device__ __forceinline__ float half_hi(uint32_t w) { return (float)__builtin_bit_cast(_Float16, (uint16_t)(w >> 16)); }
__device__ __forceinline__ uint32_t half_bits(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }
__device__ __forceinline__ void unpack8h(float (&x)[8], u32x4 w) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        x[2 * j] = half_lo(w[j]);
        x[2 * j + 1] = half_hi(w[j]);
    }
}
__device__ __forceinline__ u32x4 pack8h(const float (&v)[8]) {
    u32x4 w;
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = half_bits(v[2 * j]) | half_bits(v[2 * j + 1]) << 16;
    return w;
}

// The gradient's eight neighbours at element i, and U of them.
__device__ __forceinline__ void load_grad(float (&g)[8], const MuonMatrix& x, int64_t i, int64_t left) {
    if (x.grad_bf16)
        load8<true>(g, x.grad, i, left);
    else
        load8<false>(g, x.grad, i, left);
}

// M <- mu M + G and a part of |U|^2, in fp64, eight neighbours of a row at a time.
[[maybe_unused]] static __global__ void __launch_bounds__(256) muon_momentum_kernel(MuonStep s) {
    __shared__ double part[4];
    const MuonTile t = s.tiles[blockIdx.x];
    const MuonMatrix x = s.matrices[t.matrix];
    const uint32_t runs = (uint32_t)(x.cols + 7) / 8, n = (uint32_t)x.rows * runs;
    const uint32_t per = (n + x.parts - 1) / x.parts, at = t.i * per, end = at + per < n ? at + per : n;
    double sum = 0.0;
    constexpr uint32_t U = 4;
    for (uint32_t e0 = at + threadIdx.x; e0 < end; e0 += U * 256) {
        float g[U][8], m[U][8];
        int64_t row[U];
        int32_t c[U];
#pragma unroll
        for (uint32_t i = 0; i < U; ++i) {
            const uint32_t e = e0 + i * 256;
            if (e >= end) continue;
            row[i] = e / runs;
            c[i] = (int32_t)(e % runs) * 8;
            load_grad(g[i], x, row[i] * x.grad_stride + c[i], x.cols - c[i]);
            load8<false>(m[i], x.momentum, row[i] * x.momentum_stride + c[i], x.cols - c[i]);
        }
#pragma unroll
        for (uint32_t i = 0; i < U; ++i) {
            if (e0 + i * 256 >= end) continue;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                m[i][k] = __builtin_fmaf(s.momentum, m[i][k], g[i][k]);
                const double u = s.nesterov ? __builtin_fmaf(s.momentum, m[i][k], g[i][k]) : m[i][k];
                sum += u * u;   // nothing beyond the row: its values are zeros
            }
            store8<false>(x.momentum, row[i] * x.momentum_stride + c[i], m[i], x.cols - c[i]);
        }
    }
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) sum += __shfl_xor(sum, k);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) x.norm[t.i] = part[0] + part[1] + part[2] + part[3];
}

// X = U / (|U| + eps), scaled, in two parts; zeros up to whole steps of the products.  A
// workgroup takes 64 x 64 of X, eight neighbours of the tensor's rows a lane; of a tall
// matrix they are turned in LDS.
[[maybe_unused]] static __global__ void __launch_bounds__(256) muon_start_kernel(MuonStep s) {
    __shared__ double part[4];
    __shared__ float turn[64][65];
    const MuonTile t = s.tiles[blockIdx.x];
    const MuonMatrix x = s.matrices[t.matrix];
    double sum = (int)threadIdx.x < x.parts ? x.norm[threadIdx.x] : 0.0;
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) sum += __shfl_xor(sum, k);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
    const int64_t i0 = (int64_t)t.i * 64, j0 = (int64_t)t.j * 64;
    const int a = threadIdx.x >> 3, b = (threadIdx.x & 7) * 8;   // of 32 rows, of 64 columns
    const int64_t c = (x.tall ? i0 : j0) + b;
    float u[2][8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int64_t r = (x.tall ? j0 : i0) + h * 32 + a, left = r < x.rows ? x.cols - c : 0;
        float g[8];
        load8<false>(u[h], x.momentum, r * x.momentum_stride + c, left);
        if (s.nesterov) {
            load_grad(g, x, r * x.grad_stride + c, left);
#pragma unroll
            for (int k = 0; k < 8; ++k) u[h][k] = __builtin_fmaf(s.momentum, u[h][k], g[k]);
        }
    }
    __syncthreads();
    // in fp64: norms beyond the range of fp32's reciprocals are fine.  An infinite one leaves no
    // direction: all of X is NaN, not only what was infinite.
    const double norm = sqrt(part[0] + part[1] + part[2] + part[3]);
    const double factor = __builtin_isinf(norm) ? (double)__builtin_nanf("") : (double)x.scale / (norm + s.eps);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            u[h][k] = (float)((double)u[h][k] * factor);
            if (x.tall) turn[b + k][h * 32 + a] = u[h][k];
        }
    if (x.tall) __syncthreads();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        if (x.tall)
#pragma unroll
            for (int k = 0; k < 8; ++k) u[h][k] = turn[h * 32 + a][b + k];
        const u32x4 hi = pack8h(u[h]);
        float v[8];
        unpack8h(v, hi);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = u[h][k] - v[k];
        const int64_t to = (i0 + h * 32 + a) * x.ld + j0 + b;
        *reinterpret_cast<u32x4*>(x.hi[0] + to) = hi;
        *reinterpret_cast<u32x4*>(x.lo + to) = pack8h(v);
    }
}

// A and B are symmetric: only the tiles on and below the diagonal are computed, and what lies
// below it is stored on both sides, so that they are symmetric to the last bit whatever the
// tiles.  (The padding's sums are zeros.)
struct Symmetric {
    uint16_t* to;
    int64_t ld;
    // Elements first..last of eight.
    __device__ __forceinline__ void store(int64_t at, const float (&v)[8], int64_t first, int64_t last) const {
        const u32x4 w = pack8h(v);
        if (first <= 0 && last >= 7) {
            *reinterpret_cast<u32x4*>(to + at) = w;
            return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i >= first && i <= last) to[at + i] = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
    }
    typedef Nothing ColumnRead;
    __device__ __forceinline__ ColumnRead load_column(int64_t, int64_t, int) const { return {}; }
    template <typename Read>
    __device__ __forceinline__ void by_row(int64_t m, int64_t n, const float (&v)[8], int, const Read&) const {
        store(m * ld + n, v, 0, m - n);
    }
    __device__ __forceinline__ void by_column(int64_t n, int64_t m, const float (&v)[8], int, Nothing) const {
        store(n * ld + m, v, n + 1 - m, 7);
    }
};
// A, scaled, from X X^T.
struct GramEpilogue : Symmetric {
    float factor;
    typedef Nothing Read;
    __device__ __forceinline__ Read load_row(int64_t, int64_t, int, bool) const { return {}; }
    __device__ __forceinline__ void along(int64_t, int64_t, float (&v)[8], Read) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = in_fp32(v[i] * factor);
    }
};
// B = b A + c A A.
struct PolynomialEpilogue : Symmetric {
    const uint16_t* a;
    typedef u32x4 Read;
    __device__ __forceinline__ Read load_row(int64_t m, int64_t n, int, bool) const { return *reinterpret_cast<const u32x4*>(a + m * ld + n); }
    __device__ __forceinline__ void along(int64_t, int64_t, float (&v)[8], const Read& x) const {
        float w[8];
        unpack8h(w, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = in_fp32(__builtin_fmaf(kNsB, w[i], kNsC / kScaleA * v[i]));
    }
};
// X <- a X + B X, with both parts of X as they were.
struct XParts {
    u32x4 hi, lo;
};
__device__ __forceinline__ XParts load_x(const uint16_t* hi, const uint16_t* lo, int64_t at) {
    return {*reinterpret_cast<const u32x4*>(hi + at), *reinterpret_cast<const u32x4*>(lo + at)};
}
__device__ __forceinline__ void next_x(float (&w)[8], const XParts& x, const float (&v)[8]) {
    float l[8];
    unpack8h(w, x.hi);
    unpack8h(l, x.lo);
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = in_fp32(__builtin_fmaf(kNsA, w[i] + l[i], v[i] * (1.f / kScaleA)));
}
struct UpdateEpilogue {
    const uint16_t* from;
    uint16_t* to;
    uint16_t* lo;
    int64_t ld;
    typedef XParts Read;
    __device__ __forceinline__ Read load(int64_t m, int64_t n, int) const { return load_x(from, lo, m * ld + n); }
    __device__ __forceinline__ void operator()(int64_t m, int64_t n, const float (&v)[8], int, const Read& x) const {
        float w[8], h[8];
        next_x(w, x, v);
        const u32x4 hi = pack8h(w);
        unpack8h(h, hi);
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] -= h[i];
        *reinterpret_cast<u32x4*>(to + m * ld + n) = hi;
        *reinterpret_cast<u32x4*>(lo + m * ld + n) = pack8h(w);
    }
};

// W <- decay W - step X in `count` elements of row r from column c, with W as it was.
struct Weights {
    float w[8];
};
__device__ __forceinline__ Weights load_weights(const MuonMatrix& x, int64_t r, int64_t c, int count) {
    Weights p;
    load8<false>(p.w, x.param, r * x.param_stride + c, count);
    return p;
}
__device__ __forceinline__ void step_param(const MuonMatrix& x, float decay, float step, int64_t r, int64_t c, const float (&v)[8], int count,
                                           const Weights& p) {
    float w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = __builtin_fmaf(-step, v[i], decay * p.w[i]);
    store8<false>(x.param, r * x.param_stride + c, w, count);
    if (x.model != nullptr) store8<true>(x.model, r * x.model_stride + c, w, count);
}
__device__ __forceinline__ float step_of(const MuonStep& s, const MuonMatrix& x) {
    return s.lr * (s.spectral ? x.update_spectral : x.update) / x.scale;
}
// The last X goes straight into W.
struct FinalEpilogue {
    const MuonMatrix& x;
    const uint16_t* from;
    float decay, step;
    struct Read {
        XParts x;
        Weights w;
    };
    typedef Weights ColumnRead;
    __device__ __forceinline__ Read load_row(int64_t m, int64_t n, int count, bool by_rows) const {
        Read read;
        read.x = load_x(from, x.lo, m * x.ld + n);
        if (by_rows) read.w = load_weights(x, m, n, count);
        return read;
    }
    __device__ __forceinline__ ColumnRead load_column(int64_t r, int64_t c, int count) const { return load_weights(x, r, c, count); }
    __device__ __forceinline__ void along(int64_t, int64_t, float (&v)[8], const Read& read) const {
        float w[8];
        next_x(w, read.x, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = w[i];
    }
    __device__ __forceinline__ void by_row(int64_t r, int64_t c, const float (&v)[8], int count, const Read& read) const {
        step_param(x, decay, step, r, c, v, count, read.w);
    }
    __device__ __forceinline__ void by_column(int64_t r, int64_t c, const float (&v)[8], int count, const Weights& w) const {
        step_param(x, decay, step, r, c, v, count, w);
    }
};

enum MuonPhase { MUON_GRAM, MUON_POLYNOMIAL, MUON_UPDATE, MUON_FINAL };

template <MuonPhase PHASE, int TM, int TN, int ST>
__global__ void __launch_bounds__(256, tile_groups(TM, TN, ST)) muon_product_kernel(MuonStep s) {
    const MuonTile t = s.tiles[blockIdx.x];
    const MuonMatrix& x = s.matrices[t.matrix];
    const uint16_t* hi = x.hi[s.from];
    const int64_t mp = x.lda;   // whole steps of 64: zeros beyond m
    if constexpr (PHASE == MUON_GRAM || PHASE == MUON_POLYNOMIAL) {
        const Operand a = PHASE == MUON_GRAM ? Operand{hi, x.ld, mp} : Operand{x.a, mp, mp};
        const Terms terms{{{a, a, nullptr, a.stride}, {}}, 1};
        direct_tile<Fp16, false, false, TM, TN, ST, false>(
            terms, t.i, t.j, [&](const auto& acc, uint8_t* strip, int64_t m0, int64_t n0, uint32_t lane) {
                if constexpr (PHASE == MUON_GRAM)
                    finish_turned(acc, strip, m0, n0, mp, mp, lane, true, true, GramEpilogue{{x.a, mp}, kScaleA / (x.scale * x.scale)});
                else
                    finish_turned(acc, strip, m0, n0, mp, mp, lane, true, true, PolynomialEpilogue{{x.b, mp}, x.a});
            });
    } else {
        const Terms terms{{{Operand{x.b, mp, mp}, Operand{hi, x.ld, x.ld}, nullptr, mp}, {}}, 1};
        direct_tile<Fp16, false, true, TM, TN, ST, false>(
            terms, t.i, t.j, [&](const auto& acc, uint8_t* strip, int64_t m0, int64_t n0, uint32_t lane) {
                if constexpr (PHASE == MUON_UPDATE)
                    finish<false>(acc, strip, m0, n0, mp, x.ld, lane, UpdateEpilogue{hi, x.hi[s.from ^ 1], x.lo, x.ld});
                else
                    finish_turned(acc, strip, m0, n0, x.m, x.n, lane, x.tall == 0, x.tall != 0, FinalEpilogue{x, hi, s.decay, step_of(s, x)});
            });
    }
}

// W from X where there are no iterations.
[[maybe_unused]] static __global__ void __launch_bounds__(256) muon_apply_kernel(MuonStep s) {
    const MuonTile t = s.tiles[blockIdx.x];
    const MuonMatrix& x = s.matrices[t.matrix];
    const int64_t i0 = (int64_t)t.i * 64, j0 = (int64_t)t.j * 64;
    for (int e = threadIdx.x; e < 64 * 64; e += 256) {
        const int64_t r = (x.tall ? j0 : i0) + (e >> 6), c = (x.tall ? i0 : j0) + (e & 63);
        if (r >= x.rows || c >= x.cols) continue;
        const int64_t at = (x.tall ? c : r) * x.ld + (x.tall ? r : c);
        float v[8] = {half_lo(x.hi[0][at]) + half_lo(x.lo[at])};
        step_param(x, s.decay, step_of(s, x), r, c, v, 1, load_weights(x, r, c, 1));
    }
}

hipError_t launch_muon_momentum(const MuonStep& s, int64_t blocks, hipStream_t stream);
hipError_t launch_muon_start(const MuonStep& s, int64_t blocks, hipStream_t stream);
hipError_t launch_muon_product(MuonPhase phase, TileSize size, const MuonStep& s, int64_t blocks, hipStream_t stream);
hipError_t launch_muon_apply(const MuonStep& s, int64_t blocks, hipStream_t stream);

}  // namespace autoloco
