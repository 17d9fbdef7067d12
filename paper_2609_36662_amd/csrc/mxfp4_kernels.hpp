// Microscaled 4-bit floating point on gfx950: quantisation along the rows and the
// columns of a matrix, the values back, and products.
//
// A block of 32 values x shares the scale 2^e, e = floor(log2 max|x|) - 2: the
// largest magnitude lands in [4, 8) of the representable {0, .5, 1, 1.5, 2, 3, 4, 6}.
// The exponent field of max|x| gives e + 129 directly.  The conversion instructions
// divide by the scale, round to nearest even and saturate at 6.  The matrix
// instructions take the codes and scales as they are stored, 32 values a lane, and
// add the products up in fp32.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "matrix_view.hpp"

namespace autoloco {

struct Mx4 {
    uint8_t* codes;
    uint8_t* scales;
    int64_t rows;
    int64_t row_bytes;   // 64 * groups
    int32_t groups;      // ceil(cols / 128)
};

typedef int32_t i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr uint32_t kScaleOne = 127, kScaleNan = 255;

// The scale byte of a block from the bits of its largest magnitude (an infinity or
// a NaN has the largest bits of all).
__device__ __forceinline__ uint32_t mx_scale(uint32_t amax_bits) {
    const uint32_t e = amax_bits >> 23;
    return amax_bits == 0 ? kScaleOne : e == 255 ? kScaleNan : e > 2 ? e - 2 : 0;
}

// Codes of 8 values under scale byte s, the first in the lowest bits.
__device__ __forceinline__ uint32_t mx_codes8(const float (&x)[8], uint32_t s) {
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = x[i];
    if (s < 32) {   // scales below the normal range of the instruction's fp32 operand
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] *= 0x1p32f;
        s += 32;
    }
    if (s == kScaleNan) {
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = 0.f;
        s = kScaleOne;
    }
    const float scale = __uint_as_float(s << 23);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[0], y[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[2], y[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[4], y[5], scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[6], y[7], scale, 3);
    return w;
}

// Values as they lie in memory: 8 of them are 4 words of bf16 pairs or 8 of fp32.
template <bool BF16>
constexpr int kWords8 = BF16 ? 4 : 8;

__device__ __forceinline__ uint32_t pk_max_u16(uint32_t a, uint32_t b) {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}

// Largest magnitude's bits (fp32) among N words.
template <bool BF16, int N>
__device__ __forceinline__ uint32_t mx_amax(const uint32_t (&w)[N]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if constexpr (BF16)
            m = pk_max_u16(m, w[i] & 0x7FFF7FFFu);
        else
            m = m > (w[i] & 0x7FFFFFFFu) ? m : w[i] & 0x7FFFFFFFu;
    }
    if constexpr (BF16) {
        const uint32_t hi = m & 0xFFFF0000u, lo = m << 16;
        m = hi > lo ? hi : lo;
    }
    return m;
}

// Codes of 8 values: bf16 pairs are converted as they are, unless the scale is one
// that mx_codes8 treats apart.
template <bool BF16>
__device__ __forceinline__ uint32_t mx_codes8_raw(const uint32_t* w, uint32_t s) {
    if constexpr (BF16) {
        if (s >= 32 && s != kScaleNan) {
            typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
            const float scale = __uint_as_float(s << 23);
            uint32_t c = 0;
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[0]), scale, 0);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[1]), scale, 1);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[2]), scale, 2);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[3]), scale, 3);
            return c;
        }
    }
    float v[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (BF16) {
            v[2 * i] = bf16_lo(w[i]);
            v[2 * i + 1] = bf16_hi(w[i]);
        } else {
            v[2 * i] = __uint_as_float(w[2 * i]);
            v[2 * i + 1] = __uint_as_float(w[2 * i + 1]);
        }
    }
    return mx_codes8(v, s);
}

// N words of a row from column i on (N * 2 or N values; those past n: 0).
template <bool BF16, int N>
__device__ __forceinline__ void load_raw(uint32_t (&w)[N], const char* row, int64_t i, int64_t n) {
    constexpr int E = BF16 ? 2 : 1;
    const char* p = row + i * (BF16 ? 2 : 4);
    if (i + N * E <= n) {
#pragma unroll
        for (int j = 0; j < N / 4; ++j) {
            const u32x4_any v = reinterpret_cast<const u32x4_any*>(p)[j];
            w[4 * j] = v[0];
            w[4 * j + 1] = v[1];
            w[4 * j + 2] = v[2];
            w[4 * j + 3] = v[3];
        }
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            w[j] = 0;
            if constexpr (BF16) {
                if (i + 2 * j < n) w[j] = reinterpret_cast<const uint16_t*>(p)[2 * j];
                if (i + 2 * j + 1 < n) w[j] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[2 * j + 1] << 16;
            } else {
                if (i + j < n) w[j] = reinterpret_cast<const uint32_t*>(p)[j];
            }
        }
    }
}

// The values of 8 codes under scale byte s.
__device__ __forceinline__ void mx_values8(float (&x)[8], uint32_t w, uint32_t s) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t c = w >> (4 * i) & 15u, m = c & 7u;
        // magnitude: subnormal 0 and 0.5, else (1 + bit / 2) 2^(exponent - 1)
        const float a = m < 2 ? 0.5f * (float)m : __uint_as_float(((m >> 1) + 126u) << 23 | (m & 1u) << 22);
        const float v = __builtin_ldexpf(a, (int)s - 127);
        x[i] = s == kScaleNan ? __uint_as_float(0x7FC00000u) : c & 8u ? -v : v;
    }
}

// 16 bytes of values as they lie in memory, from 8 (bf16) or 4 codes.  The conversion
// instruction where the values are in the normal range.
template <bool BF16>
__device__ __forceinline__ u32x4 mx_values_raw(uint32_t w, uint32_t s) {
    u32x4 v;
    if (s >= 32 && s < 250) {
        const float scale = __uint_as_float(s << 23);
        if constexpr (BF16) {
            v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
            v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
            v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
            v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
        } else {
            const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1);
            v = u32x4{__float_as_uint(a[0]), __float_as_uint(a[1]), __float_as_uint(b[0]), __float_as_uint(b[1])};
        }
    } else {
        float x[8];
        mx_values8(x, w, s);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = BF16 ? bf16_pack(x[2 * i], x[2 * i + 1]) : __float_as_uint(x[i]);
    }
    return v;
}

template <int CTRL>
__device__ __forceinline__ uint32_t max_dpp(uint32_t v) {
    const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, false);
    return o > v ? o : v;
}

// ---------------------------------------------------------------- quantise --
// Along the rows: a lane takes 8 columns of each of U neighbouring groups, four lanes a
// block; a workgroup 16 rows (nt workgroups across; first: the launch's first one, since a
// grid has fewer than 2^32 threads).  Bound by reading x and, with bf16, still by the
// instructions: two groups an address, where one for each, found by dividing a thread's
// number, took 22.8 us for 20,000 x 2,048 bf16 against 19.2 (5.4 TB/s) and 15.5 against 14.6
// for 4,096 x 4,096 fp32; four groups 20.4 and 16.0.
constexpr int kRowsGroups = 2;
template <bool BF16>
__global__ void __launch_bounds__(kBlock) mx_rows_kernel(MatrixView x, Mx4 q, uint32_t nt, uint32_t first) {
    constexpr int U = kRowsGroups;
    const uint32_t b = first + blockIdx.x, rt = b / nt;
    const int g0 = (int)(b % nt) * U;
    const int piece = threadIdx.x & 15;
    const int64_t row = (int64_t)rt * 16 + (threadIdx.x >> 4);
    const bool there = row < q.rows;
    const char* from = static_cast<const char*>(x.data) + (there ? row : q.rows - 1) * x.stride * (BF16 ? 2 : 4);
    const int64_t c0 = (int64_t)g0 * 128 + piece * 8;
    uint32_t v[U][kWords8<BF16>];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if ((int64_t)(g0 + u + 1) * 128 <= x.cols)   // the same in every lane
            load_raw<BF16>(v[u], from + c0 * (BF16 ? 2 : 4), u * 128, u * 128 + 8);
        else
            load_raw<BF16>(v[u], from, c0 + u * 128, x.cols);
    }
    __builtin_amdgcn_sched_barrier(0);
    uint8_t* codes = q.codes + row * q.row_bytes + g0 * 64 + piece * 4;
    uint8_t* scales = q.scales + ((int64_t)g0 * q.rows + row) * 4 + (piece >> 2);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        uint32_t m = mx_amax<BF16>(v[u]);
        m = max_dpp<0xB1>(m);   // lanes ^ 1, then ^ 2: the block's four
        m = max_dpp<0x4E>(m);
        const uint32_t s = mx_scale(m);
        const uint32_t w = mx_codes8_raw<BF16>(v[u], s);
        if (there && g0 + u < q.groups) {
            *reinterpret_cast<uint32_t*>(codes + u * 64) = w;
            if ((piece & 3) == 0) scales[u * q.rows * 4] = (uint8_t)s;
        }
    }
}

// Along the columns (and the rows): a workgroup takes 128 rows of 256 bytes, all loads
// in flight together, into LDS, where a lane then reads 32 rows of one word: one fp32
// column or two bf16 ones.  2,048 x 5,632 bf16 in both directions: 23 MB read and 12
// written.
template <bool BF16, bool ROWS>
__global__ void __launch_bounds__(kBlock) mx_cols_kernel(MatrixView x, Mx4 q, Mx4 qt, uint32_t tiles, uint32_t first) {
    constexpr int E = BF16 ? 2 : 1;          // elements a word
    constexpr int W = 64 * E;                // columns of a tile
    __shared__ uint32_t tile[128 * 64];
    const uint32_t b = first + blockIdx.x, rt = b / tiles, ct = b % tiles;
    const int64_t r0 = (int64_t)rt * 128, c0 = (int64_t)ct * W;
    const int lane16 = threadIdx.x & 15, line = threadIdx.x >> 4;
    const int64_t c = c0 + lane16 * 4 * E;
    uint32_t w[8][4];
#pragma unroll
    for (int p = 0; p < 8; ++p) {
        const int64_t row = r0 + p * 16 + line;
        load_raw<BF16>(w[p], static_cast<const char*>(x.data) + row * x.stride * (BF16 ? 2 : 4), c, row < x.rows ? x.cols : 0);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int p = 0; p < 8; ++p) {
        const int r = p * 16 + line;
        const int64_t row = r0 + r;
        *reinterpret_cast<u32x4*>(&tile[r * 64 + lane16 * 4]) = u32x4{w[p][0], w[p][1], w[p][2], w[p][3]};
        if constexpr (ROWS) {
            uint32_t m = mx_amax<BF16>(w[p]);
            m = max_dpp<0xB1>(m);
            m = max_dpp<0x4E>(m);
            if constexpr (!BF16) m = max_dpp<0x141>(m);   // 7 - lane inside each 8: the other four of the block
            const uint32_t s = mx_scale(m);
            uint32_t code;
            if constexpr (BF16) {
                code = mx_codes8_raw<true>(w[p], s);
            } else {
                const uint32_t v[8] = {w[p][0], w[p][1], w[p][2], w[p][3], 0, 0, 0, 0};
                code = mx_codes8_raw<false>(v, s);
            }
            if (row < x.rows) {
                uint8_t* d = q.codes + row * q.row_bytes + c / 2;
                if constexpr (BF16)
                    *reinterpret_cast<uint32_t*>(d) = code;
                else
                    *reinterpret_cast<uint16_t*>(d) = (uint16_t)code;
                if ((lane16 & (BF16 ? 3 : 7)) == 0) q.scales[(c0 / 128 * q.rows + row) * 4 + (c % 128) / 32] = (uint8_t)s;
            }
        }
    }
    __syncthreads();
    const int word = threadIdx.x & 63, blk = threadIdx.x >> 6;
    uint32_t v[32];
#pragma unroll
    for (int r = 0; r < 32; ++r) v[r] = tile[(blk * 32 + r) * 64 + word];
    __syncthreads();
    // codes of the tile's columns through LDS: [W][4] pieces of 16 bytes
    auto column = [&](int h, uint32_t amax, auto words8) {   // words8(j): rows 8 j on as they would lie in memory
        const uint32_t s = mx_scale(amax);
        u32x4 code;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t u[kWords8<BF16>];
            words8(j, u);
            code[j] = mx_codes8_raw<BF16>(u, s);
        }
        const int col = word * E + h;
        *reinterpret_cast<u32x4*>(&tile[col * 16 + blk * 4]) = code;
        if (c0 + col < x.cols) qt.scales[((int64_t)rt * qt.rows + c0 + col) * 4 + blk] = (uint8_t)s;
    };
    if constexpr (BF16) {
        uint32_t m = 0;
#pragma unroll
        for (int r = 0; r < 32; ++r) m = pk_max_u16(m, v[r] & 0x7FFF7FFFu);
        column(0, m << 16, [&](int j, uint32_t* u) {
#pragma unroll
            for (int i = 0; i < 4; ++i) u[i] = __builtin_amdgcn_perm(v[8 * j + 2 * i + 1], v[8 * j + 2 * i], 0x05040100u);
        });
        column(1, m & 0xFFFF0000u, [&](int j, uint32_t* u) {
#pragma unroll
            for (int i = 0; i < 4; ++i) u[i] = __builtin_amdgcn_perm(v[8 * j + 2 * i + 1], v[8 * j + 2 * i], 0x07060302u);
        });
    } else {
        column(0, mx_amax<false>(v), [&](int j, uint32_t* u) {
#pragma unroll
            for (int i = 0; i < 8; ++i) u[i] = v[8 * j + i];
        });
    }
    __syncthreads();
#pragma unroll
    for (int p = 0; p < E; ++p) {
        const int i = p * kBlock + threadIdx.x, col = i >> 2;
        if (c0 + col < x.cols)
            *reinterpret_cast<u32x4*>(qt.codes + (c0 + col) * qt.row_bytes + (int64_t)rt * 64 + (i & 3) * 16) =
                *reinterpret_cast<const u32x4*>(&tile[i * 4]);
    }
}

// -------------------------------------------------------------- dequantise --
// A lane writes 16 bytes of each of two neighbouring groups, so that neighbouring lanes
// write neighbouring ones; a workgroup 16 rows (bf16) or 8, nt workgroups across.  Bound by
// writing: 50,257 x 768 fp32 34 us (5.1 TB/s) one call after another (with 32 bytes a lane and
// values put together from bits 47).  After another kernel it ends sooner and leaves the
// caches full: in turn with mx_rows_kernel of that size 27 us, and that one 42 instead of
// its 32, 70 us for both.  Stores past the caches take 27 us in any case, but whoever reads the
// values next pays for it: 8,192 x 4,096 fp32 with its 4-bit form taken again 50 and 53 us,
// multiplied in place 76 against 71; 4,096 x 4,096 26.8 against 25.7 and 35.4 against 33.5.
template <bool BF16>
constexpr int kValueRows = BF16 ? 16 : 8;
template <bool BF16>
__global__ void __launch_bounds__(kBlock) mx_values_kernel(Mx4 q, MatrixOut out, uint32_t nt, uint32_t first) {
    constexpr int V = BF16 ? 8 : 4, L = 128 / V, U = kRowsGroups;
    const uint32_t b = first + blockIdx.x, rt = b / nt;
    const int g0 = (int)(b % nt) * U;
    const int piece = threadIdx.x % L;
    const int64_t row = (int64_t)rt * kValueRows<BF16> + threadIdx.x / L;
    if (row >= q.rows) return;
    const uint8_t* codes = q.codes + row * q.row_bytes + g0 * 64 + piece * (V / 2);
    const uint8_t* scales = q.scales + ((int64_t)g0 * q.rows + row) * 4 + piece / (32 / V);
    char* to = static_cast<char*>(out.data) + row * out.stride * (BF16 ? 2 : 4);
    uint32_t w[U], s[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        w[u] = 0;
        s[u] = 0;
        if (g0 + u < q.groups) {   // the same in every lane
            if constexpr (BF16)
                w[u] = *reinterpret_cast<const uint32_t*>(codes + u * 64);
            else
                w[u] = *reinterpret_cast<const uint16_t*>(codes + u * 64);
            s[u] = scales[u * q.rows * 4];
        }
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t c = (int64_t)(g0 + u) * 128 + piece * V;
        const u32x4 v = mx_values_raw<BF16>(w[u], s[u]);
        if (c + V <= out.cols) {
            *reinterpret_cast<u32x4_any*>(to + c * (BF16 ? 2 : 4)) = v;
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (c + e < out.cols) {
                    if constexpr (BF16)
                        reinterpret_cast<uint16_t*>(to)[c + e] = (uint16_t)(v[e / 2] >> (16 * (e & 1)));
                    else
                        reinterpret_cast<uint32_t*>(to)[c + e] = v[e];
                }
        }
    }
}

// ----------------------------------------------------------------- product --
__device__ __forceinline__ i32x8 operand(u32x4 w) { return i32x8{(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0}; }

// Up to 16 rows of x, quantised as they are read.  A workgroup takes 16 R rows of the
// weight (first: the launch's first one); its NW waves take groups of 128 columns in turn and are joined in LDS in wave
// order.  A wave reads x in whole rows, 8 columns a lane and four rows at a time,
// quantises them as mx_rows_kernel does, and passes the codes through its own piece of
// LDS into the order of the 16x16x128 instruction: row lane % 16, columns 32 (lane / 16)
// on.  (A lane that reads its own 32 columns needs no exchange, but its neighbours are 64
// bytes apart, and the address unit takes a cycle for every lane: 13 x 4,096 x 11,008
// rows 10.2 us against 9.6, 16 x 11,008 x 4,096 rows 17.6 against 13.1.)  Bound by the
// latency of the weight's and x's loads, then by the quantisation (one row of x 7.4 us
// where thirteen take 9.6): 24 MB of weight at 2.5 TB/s, launch included.
template <bool BF16, int R, int NW>
__global__ void __launch_bounds__(NW * 64) mx_tokens_kernel(MatrixView x, Mx4 w, MatrixOut y, uint32_t first) {
    constexpr int W = kWords8<BF16>;
    constexpr int kRow = 80;                       // bytes of a row of codes: 16 rows' pieces in 64 banks
    __shared__ __align__(16) uint8_t xlds[NW][16 * kRow + 64];
    __shared__ float part[NW][R * 256];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, j = lane >> 4;
    const int64_t n0 = ((int64_t)first + blockIdx.x) * (16 * R);
    const uint8_t* wc[R];
    const uint8_t* ws[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int64_t wn = n0 + 16 * i + r < w.rows ? n0 + 16 * i + r : w.rows - 1;
        wc[i] = w.codes + wn * w.row_bytes + j * 16;
        ws[i] = w.scales + wn * 4 + j;
    }
    const int quads = ((int)x.rows + 3) / 4;
    uint8_t* mine = xlds[wave];
    f32x4 acc[R] = {};
    for (int g = wave; g < w.groups; g += NW) {
        u32x4 c[R];
        uint32_t s[R], v[4][W];
        // x first: it is nearer, and is worked on while the weight is still on its way
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int64_t row = 4 * q + j < x.rows ? 4 * q + j : x.rows - 1;
            if (q < quads)
                load_raw<BF16>(v[q], static_cast<const char*>(x.data) + row * x.stride * (BF16 ? 2 : 4),
                               (int64_t)g * 128 + r * 8, x.cols);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < R; ++i) {
            c[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(wc[i] + (int64_t)g * 64));
            s[i] = ws[i][(int64_t)g * w.rows * 4];
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (q < quads) {
                uint32_t m = mx_amax<BF16>(v[q]);
                m = max_dpp<0xB1>(m);
                m = max_dpp<0x4E>(m);
                const uint32_t xs = mx_scale(m);
                *reinterpret_cast<uint32_t*>(mine + (4 * q + j) * kRow + r * 4) = mx_codes8_raw<BF16>(v[q], xs);
                if ((r & 3) == 0) mine[16 * kRow + (4 * q + j) * 4 + r / 4] = (uint8_t)xs;
            }
        // the wave's own stores before its loads: LDS keeps their order, the compiler has to
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        const u32x4 xc = *reinterpret_cast<const u32x4*>(mine + r * kRow + j * 16);
        const uint32_t xs = mine[16 * kRow + r * 4 + j];
#pragma unroll
        for (int i = 0; i < R; ++i)
            acc[i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(c[i]), operand(xc), acc[i], 4, 4, 0, (int)s[i],
                                                                      0, (int)xs);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
#pragma unroll
    for (int i = 0; i < R; ++i) *reinterpret_cast<f32x4*>(&part[wave][i * 256 + lane * 4]) = acc[i];
    __syncthreads();
    // value t: token t / (16 R), row t % (16 R) of the workgroup's
    for (int t = threadIdx.x; t < (int)x.rows * 16 * R; t += NW * 64) {
        const int m = t / (16 * R), n = t % (16 * R);
        const int at = (n >> 4) * 256 + ((n >> 2 & 3) * 16 + m) * 4 + (n & 3);
        float sum = part[0][at];
#pragma unroll
        for (int k = 1; k < NW; ++k) sum += part[k][at];
        if (n0 + n < y.cols) store_one<BF16>(y.data, m * y.stride + n0 + n, sum);
    }
}

// Zeros where there is nothing to add up.
template <bool BF16>
__global__ void __launch_bounds__(kBlock) zero_matrix_kernel(MatrixOut out) {
    const int64_t n = out.rows * out.cols;
    for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i < n; i += (int64_t)gridDim.x * kBlock)
        store_one<BF16>(out.data, i / out.cols * out.stride + i % out.cols, 0.f);
}

hipError_t launch_mx_quantize(bool bf16, const MatrixView& x, const Mx4* q, const Mx4* qt, hipStream_t s);
hipError_t launch_mx_values(bool bf16, const Mx4& q, const MatrixOut& out, hipStream_t s);
hipError_t launch_mx_matmul(bool bf16, const Mx4& a, const Mx4& b, const MatrixOut& out, hipStream_t s);
hipError_t launch_mx_tokens(bool bf16, const MatrixView& x, const Mx4& w, const MatrixOut& y, hipStream_t s);

}  // namespace autoloco
