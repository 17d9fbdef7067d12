// Products of 16-bit matrices in tiles of the result, on gfx950.
//
//   out[m][n] = sum over the terms, over k, of a[m][k] b[n][k]
//
// An operand lies along the summed axis (its row r is p[r stride + k]) or across it
// (p[k stride + r], TR): a linear layer's forward pass has both along it, the gradient
// by its input the weight across, the gradient by its weight both.  Operands across are
// stored in LDS as they lie and turned by the transposing LDS reads, so no matrix is ever
// written out transposed.
//
// A workgroup of four waves (2 x 2) takes 64 T x 64 T of the result, a wave 32 T x 32 T, in
// steps of 64 summed elements.  What lies beyond a matrix counts as zero.  Sums are fp32.
// The result goes through LDS, so that a lane has eight neighbours of a row for the
// epilogue, which rounds, combines with other matrices and stores.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "matrix_view.hpp"

namespace autoloco {

typedef float f32x16 __attribute__((ext_vector_type(16)));

// f(integral_constant j) for j from FROM up to TO.
template <int FROM, int TO, typename F>
__device__ __forceinline__ void each(F&& f) {
    if constexpr (FROM < TO) {
        f(std::integral_constant<int, FROM>{});
        each<FROM + 1, TO>(f);
    }
}

// One operand of a product: n rows in the result's dimension.
struct Operand {
    const uint16_t* p;
    int64_t stride, n;
};
// a b^T over k elements; b2: the second matrix of a pair (PAIR), of b's shape and stride.
struct Term {
    Operand a, b;
    const uint16_t* b2;
    int64_t k;
};
struct Terms {
    Term t[2];
    int count;
};

struct Bf16 {
    static __device__ __forceinline__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c) {
        typedef __bf16 v8 __attribute__((ext_vector_type(8)));
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
};
struct Fp16 {
    static __device__ __forceinline__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c) {
        typedef _Float16 v8 __attribute__((ext_vector_type(8)));
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
};

// Up to 8 16-bit elements at p, zeros for the rest.
__device__ __forceinline__ u32x4 load_piece(const uint16_t* p, int left) {
    if (left >= 8) return __builtin_bit_cast(u32x4, *reinterpret_cast<const u32x4_any*>(p));
    u32x4 v = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < left) v[i / 2] |= (uint32_t)p[i] << (16 * (i & 1));
    return v;
}
// The first `count` of 8 elements to p.
__device__ __forceinline__ void store_piece(uint16_t* p, u32x4 v, int count) {
    if (count >= 8) {
        *reinterpret_cast<u32x4_any*>(p) = v;
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < count) p[i] = (uint16_t)(v[i / 2] >> (16 * (i & 1)));
}
__device__ __forceinline__ u32x4 pack8(const float (&v)[8]) {
    return {bf16_pack(v[0], v[1]), bf16_pack(v[2], v[3]), bf16_pack(v[4], v[5]), bf16_pack(v[6], v[7])};
}
__device__ __forceinline__ void unpack8(float (&x)[8], u32x4 w) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        x[2 * j] = __uint_as_float(w[j] << 16);
        x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
    }
}

// Where an operand's piece of 16 bytes lies in its tile of B rows in LDS.  Along: a row
// takes 128 bytes, piece q at q ^ (row / 2 % 8), so that 16 neighbouring rows' pieces of one
// column range lie in 64 different banks.  Across: a k takes 2 B bytes, and its runs of 64
// bytes (32 rows, what a matrix instruction takes of it) are exchanged by k, so that the
// four k that a transposing read joins lie in different banks.
template <int B>
__device__ __forceinline__ uint32_t exchange(uint32_t k) {
    return B >= 128 ? k & 3 : (k >> 1) & 1;
}
template <bool TR, int B>
__device__ __forceinline__ uint32_t place(uint32_t idx) {
    if constexpr (TR) {
        const uint32_t k = idx / (B / 8), q = idx % (B / 8);
        return k * (2 * B) + (((q >> 2) ^ exchange<B>(k)) << 6) + (q & 3) * 16;
    } else {
        const uint32_t row = idx >> 3, q = idx & 7;
        return row * 128 + ((q ^ (row >> 1 & 7)) << 4);
    }
}
// A lane's pieces of an operand's tile, N of them, step after step.  PAIR: the tile's rows are
// 32 of b, 32 of b2, the next 32 of b and so on.  What is taken for rows that the operand has
// not goes into results that it has not: rows beyond the last are the last again, and a piece
// across may reach beyond its rows where another line of them follows.
template <bool TR, int B, int N, bool PAIR>
struct Pieces {
    const uint16_t* p[N];
    int64_t advance;
    // Whether whole pieces may be taken, in every step but one that reaches the end.
    static __device__ __forceinline__ bool regular(const Operand& o) { return !TR || o.stride >= 8; }
    __device__ __forceinline__ void begin(const Operand& o, const uint16_t* second, int64_t r0, uint32_t thread) {
        advance = TR ? 64 * o.stride : 64;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const uint32_t idx = thread + 256 * j;
            if constexpr (TR) {
                int64_t r = r0 + idx % (B / 8) * 8;
                if (r >= o.n) r = o.n < 8 ? 0 : o.n - 8;
                p[j] = o.p + (int64_t)(idx / (B / 8)) * o.stride + r;
            } else {
                const uint32_t row = idx >> 3;
                const int64_t r = r0 + (PAIR ? (row >> 6) * 32 + (row & 31) : row);
                p[j] = (PAIR && (row >> 5 & 1) ? second : o.p) + (r < o.n ? r : o.n - 1) * o.stride + (idx & 7) * 8;
            }
        }
    }
    // The next step's, whole.  (No branch: loads that may not have been issued are waited for at once.)
    __device__ __forceinline__ void get(u32x4 (&to)[N]) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            to[j] = __builtin_bit_cast(u32x4, *reinterpret_cast<const u32x4_any*>(p[j]));
            p[j] += advance;
        }
    }
};
// One piece of an operand's tile, with zeros for what the operand has not.
template <bool TR, int B, bool PAIR>
__device__ __forceinline__ u32x4 fetch(const Operand& o, const uint16_t* second, int64_t r0, int64_t k0, int64_t K, uint32_t idx) {
    if constexpr (TR) {
        const int64_t k = k0 + idx / (B / 8), r = r0 + idx % (B / 8) * 8, left = o.n - r;
        return load_piece(o.p + k * o.stride + r, k < K ? (left < 8 ? (int)left : 8) : 0);
    } else {
        const uint32_t row = idx >> 3;
        const int64_t r = r0 + (PAIR ? (row >> 6) * 32 + (row & 31) : row), k = k0 + (idx & 7) * 8, left = K - k;
        return load_piece((PAIR && (row >> 5 & 1) ? second : o.p) + r * o.stride + k, r < o.n ? (left < 8 ? (int)left : 8) : 0);
    }
}
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4* LdsPiece;
// A transposing read.  (The restricted pointer says that it is no other access's business:
// without it the compiler waits, before the first of them, for all loads on their way into LDS.)
__device__ __forceinline__ u32x2r turned_read(const LdsPiece __restrict__ p) {
    return __builtin_bit_cast(u32x2r, __builtin_amdgcn_ds_read_tr16_b64_v4i16(p));
}
// Half of a wave's operand across: 32 rows from row, four of each lane's eight summed elements.
template <int B>
__device__ __forceinline__ u32x2r turned_half(const uint8_t* tile, uint32_t row, uint32_t s, uint32_t lane, uint32_t upper) {
    const uint32_t k = 16 * s + 8 * (lane >> 5) + ((lane & 15) >> 2);
    const uint8_t* p = tile + k * (2 * B) + (((row >> 5) ^ exchange<B>(k)) << 6) + (lane >> 4 & 1) * 32 + (lane & 3) * 8;
    // four summed elements on, the exchange is the same
    return turned_read((LdsPiece)(void*)(p + upper * 4 * 2 * B));
}
// Waits until at most N of a wave's loads are outstanding and its LDS reads are done,
// then meets the other waves.
template <int N>
__device__ __forceinline__ void arrived() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// A wave's operand of 32 rows (of the tile, from row) and 16 summed elements (part s of the step's four).
template <bool TR, int B>
__device__ __forceinline__ u32x4 operand_of(const uint8_t* tile, uint32_t row, uint32_t s, uint32_t lane) {
    if constexpr (TR) {
        const u32x2r lo = turned_half<B>(tile, row, s, lane, 0), hi = turned_half<B>(tile, row, s, lane, 1);
        return u32x4{lo[0], lo[1], hi[0], hi[1]};
    } else {
        const uint32_t r = row + (lane & 31), q = 2 * s + (lane >> 5);
        return *reinterpret_cast<const u32x4*>(tile + r * 128 + ((q ^ (r >> 1 & 7)) << 4));
    }
}

// Tiles of the result by rows and columns, and how workgroups go through them.
struct Tiles {
    uint32_t mt, nt;
};
// The tile of workgroup b: workgroups go round the eight dies (each with a cache of
// its own), so each die gets a run of neighbouring tiles, eight rows of tiles wide.
__device__ __forceinline__ void tile_at(uint32_t b, const Tiles& g, uint32_t& m, uint32_t& n) {
    const uint32_t total = g.mt * g.nt, per = total / 8, extra = total % 8;
    const uint32_t die = b % 8, i = b / 8;
    const uint32_t t = die * per + (die < extra ? die : extra) + i;
    const uint32_t band = t / (8 * g.nt), first = band * 8;
    const uint32_t height = g.mt - first < 8 ? g.mt - first : 8;
    const uint32_t in = t - band * 8 * g.nt;
    m = first + in % height;
    n = in / height;
}

// A wave's own LDS stores before its loads: LDS keeps their order, the compiler has to.
__device__ __forceinline__ void own_lds() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}
// 32 rows of a wave's sums into its strip: a lane has row lane % 32 and of each 32 columns
// 8 (i / 4) + 4 (lane / 32) + i % 4.
template <int T>
__device__ __forceinline__ void spill_sums(const f32x16 (&acc)[T], float* s, uint32_t lane) {
    constexpr int kPitch = 32 * T + 4;
#pragma unroll
    for (int u = 0; u < T; ++u)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            *reinterpret_cast<f32x4*>(s + (lane & 31) * kPitch + u * 32 + 8 * q + 4 * (lane >> 5)) =
                f32x4{acc[u][4 * q], acc[u][4 * q + 1], acc[u][4 * q + 2], acc[u][4 * q + 3]};
    own_lds();
}

// What an epilogue that reads nothing has read.
struct Nothing {};

// The accumulators of a wave through its strip of LDS to the epilogue, 32 rows at a time:
// epi(m, n, v, count, read) gets eight neighbouring columns of row m, `count` of them inside; of
// a pair epi(m, n, v, w, count, read), the same columns of both.  read is what epi.load(m, n,
// count) gave: the next 32 rows' loads are on their way while these are finished.
template <bool PAIR, int TM, int T, typename Epi>
__device__ __forceinline__ void finish(const f32x16 (&acc)[TM][T], uint8_t* strip, int64_t m0, int64_t n0, int64_t rows, int64_t cols,
                                       uint32_t lane, const Epi& epi) {
    constexpr int kPitch = 32 * T + 4;           // floats
    constexpr int P = (PAIR ? 2 : 4) * T;        // runs of eight columns in a row
    constexpr int S = 64 / P, R = 32 / S;        // rows that the lanes take together, and a lane's of 32
    float* s = reinterpret_cast<float*>(strip);
    const uint32_t col = lane % P * 8;
    const int64_t n = n0 + col;
    const int64_t left = cols - n;
    const int count = left < 8 ? (int)left : 8;
    // the strip's rows, a few of each lane's at a time: more would not fit the registers
    constexpr int C = R < 4 ? R : 4, H = R / C;
    typename Epi::Read read[2][C];
    auto row_of = [&](int step, int r) { return m0 + step / H * 32 + (step % H * C + r) * S + lane / P; };
    auto fetch = [&](int step) {
#pragma unroll
        for (int r = 0; r < C; ++r) {
            const int64_t m = row_of(step, r);
            if (m < rows && count > 0) read[step & 1][r] = epi.load(m, n, count);
        }
    };
    fetch(0);
    each<0, TM * H>([&](auto which) {   // (left to the compiler, a long loop may stay one, and the sums go to memory)
        constexpr int step = decltype(which)::value;
        if constexpr (step % H == 0) spill_sums<T>(acc[step / H], s, lane);
        if constexpr (step + 1 < TM * H) fetch(step + 1);
        float v[C][8], w[PAIR ? C : 1][8];
#pragma unroll
        for (int r = 0; r < C; ++r) {
            const float* from = s + ((step % H * C + r) * S + lane / P) * kPitch + (PAIR ? col / 32 * 64 + col % 32 : col);
#pragma unroll
            for (int i = 0; i < 8; i += 4) {
                *reinterpret_cast<f32x4*>(v[r] + i) = *reinterpret_cast<const f32x4*>(from + i);
                if constexpr (PAIR) *reinterpret_cast<f32x4*>(w[r] + i) = *reinterpret_cast<const f32x4*>(from + 32 + i);
            }
        }
        if (step % H == H - 1) own_lds();
        if (count > 0) {
#pragma unroll
            for (int r = 0; r < C; ++r) {
                const int64_t m = row_of(step, r);
                if (m >= rows) continue;
                if constexpr (PAIR)
                    epi(m, n, v[r], w[r], count, read[step & 1][r]);
                else
                    epi(m, n, v[r], count, read[step & 1][r]);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    });
}

// The same, where the epilogue wants the result's rows, its columns (the result turned) or
// both: epi.along(m, n, v, read) finishes eight neighbouring columns of row m, then epi.by_row(m,
// n, v, count, read) gets them and epi.by_column(n, m, v, count, read) eight neighbours of
// column n from row m on, with what epi.load_row and epi.load_column gave.
template <int TM, int T, typename Epi>
__device__ __forceinline__ void finish_turned(const f32x16 (&acc)[TM][T], uint8_t* strip, int64_t m0, int64_t n0, int64_t rows, int64_t cols,
                                              uint32_t lane, bool by_rows, bool by_columns, const Epi& epi) {
    constexpr int kPitch = 32 * T + 4, P = 4 * T, S = 64 / P, R = 32 / S, C = R < 4 ? R : 4;
    float* s = reinterpret_cast<float*>(strip);
    const uint32_t col = lane % P * 8;
    const int64_t left = cols - n0 - col;
    const int count = left < 8 ? (int)left : 8;
    each<0, TM>([&](auto which) {
        constexpr int t = decltype(which)::value;
        const int64_t mt = m0 + t * 32;
#pragma unroll
        for (int h = 0; h < R; h += C) {
            const int64_t m = mt + h * S + lane / P;
            float* at = s + (h * S + lane / P) * kPitch + col;
            typename Epi::Read read[C];
#pragma unroll
            for (int r = 0; r < C; ++r)
                if (m + r * S < rows && count > 0) read[r] = epi.load_row(m + r * S, n0 + col, count, by_rows);
            if (h == 0) spill_sums<T>(acc[t], s, lane);
            float v[C][8];
#pragma unroll
            for (int r = 0; r < C; ++r)
#pragma unroll
                for (int i = 0; i < 8; i += 4)
                    *reinterpret_cast<f32x4*>(v[r] + i) = *reinterpret_cast<const f32x4*>(at + r * S * kPitch + i);
#pragma unroll
            for (int r = 0; r < C; ++r) {
                if (m + r * S >= rows || count <= 0) continue;
                epi.along(m + r * S, n0 + col, v[r], read[r]);
                if (by_columns)
#pragma unroll
                    for (int i = 0; i < 8; i += 4)
                        *reinterpret_cast<f32x4*>(at + r * S * kPitch + i) = f32x4{v[r][i], v[r][i + 1], v[r][i + 2], v[r][i + 3]};
                if (by_rows) epi.by_row(m + r * S, n0 + col, v[r], count, read[r]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        own_lds();
        if (!by_columns) return;
        // four lanes take a column's 32 rows, four columns a lane at a time
        constexpr int U = T < 2 ? 2 : 4;
        const uint32_t first = lane % 4 * 8;
        const int64_t down = rows - mt - first;
        const int below = down < 8 ? (int)down : 8;
#pragma unroll
        for (int c0 = 0; c0 < 2 * T; c0 += U) {
            typename Epi::ColumnRead across[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t n = n0 + (c0 + u) * 16 + lane / 4;
                if (n < cols && below > 0) across[u] = epi.load_column(n, mt + first, below);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint32_t c = (c0 + u) * 16 + lane / 4;
                float x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = s[(first + i) * kPitch + c];
                if (n0 + c < cols && below > 0) epi.by_column(n0 + c, mt + first, x, below, across[u]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        own_lds();
    });
}

// A tile whose operands come through registers, piece by piece, whatever their strides,
// sizes and addresses: the pieces of the next Q steps are on their way while one is multiplied.
// Bound by the loads' latency and the turn through registers: 4,095 rows of 2,047 with 5,631
// between take 488 us forward (0.58 PFLOP/s), 482 for dg, du and dx, 643 for the three weights'
// gradients (0.44); 300 rows of 771 with 1,030 between some 28, 11, 18, 19 and three times 7 us.  No
// branch stands between a step's loads: with them the compiler waits for all of a step before the
// next (134 us for both directions of the last, 86 without).
template <typename E, bool AT, bool BT, int T, bool PAIR, typename Finish>
__device__ __forceinline__ void product_tile(const Terms& terms, uint32_t ti, uint32_t tj, const Finish& fin) {
    constexpr int B = 64 * T, kTile = B * 128, N = B * 8 / 256, Q = T == 1 ? 4 : 2;   // N: a thread's pieces of an operand
    constexpr int kStrip = 32 * (32 * T + 4) * 4;
    static_assert(kStrip <= kTile, "the strips fit");
    __shared__ __align__(1024) uint8_t lds[4 * kTile];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave >> 1, wn = wave & 1;
    const int64_t m0 = (int64_t)ti * B, n0 = (int64_t)tj * (PAIR ? B / 2 : B);
    f32x16 acc[T][T] = {};
    // Multiplies a step's pieces; `then` asks for others once they are in LDS.  Steps take the two
    // tiles in turn.
    auto products = [&](const uint8_t* tile) {
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            u32x4 fa[T], fb[T];
#pragma unroll
            for (int t = 0; t < T; ++t) {
                fa[t] = operand_of<AT, B>(tile, (wm * T + t) * 32, s, lane);
                fb[t] = operand_of<BT, B>(tile + kTile, (wn * T + t) * 32, s, lane);
            }
#pragma unroll
            for (int t = 0; t < T; ++t)
#pragma unroll
                for (int u = 0; u < T; ++u) acc[t][u] = E::mfma(fb[u], fa[t], acc[t][u]);
        }
    };
    auto multiply = [&](auto turn, const u32x4 (&ra)[N], const u32x4 (&rb)[N], auto then) {
        uint8_t* tile = lds + (decltype(turn)::value & 1) * 2 * kTile;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            *reinterpret_cast<u32x4*>(tile + place<AT, B>(threadIdx.x + 256 * j)) = ra[j];
            *reinterpret_cast<u32x4*>(tile + kTile + place<BT, B>(threadIdx.x + 256 * j)) = rb[j];
        }
        then();
        // one barrier a step: whoever is past it has read the tile before last
        __syncthreads();
        products(tile);
    };
    for (int term = 0; term < terms.count; ++term) {
        const Term& t = terms.t[term];
        Pieces<AT, B, N, false> a;
        Pieces<BT, B, N, PAIR> b;
        a.begin(t.a, nullptr, m0, threadIdx.x);
        b.begin(t.b, t.b2, n0, threadIdx.x);
        const int64_t steps = (t.k + 63) / 64, whole = a.regular(t.a) && b.regular(t.b) && t.k > 0 ? (t.k - 1) / 64 : 0;
        u32x4 ra[Q][N], rb[Q][N];
        auto get = [&](auto which) {
            a.get(ra[decltype(which)::value]);
            b.get(rb[decltype(which)::value]);
        };
        auto nothing = [] {};
        if (term > 0) __syncthreads();
        int64_t i = 0;
        if (whole >= Q) {
            each<0, Q>(get);
            for (; i + 2 * Q <= whole; i += Q)
                each<0, Q>([&](auto q) { multiply(q, ra[decltype(q)::value], rb[decltype(q)::value], [&] { get(q); }); });
            each<0, Q>([&](auto q) { multiply(q, ra[decltype(q)::value], rb[decltype(q)::value], nothing); });
            i += Q;
        }
        each<0, Q - 1>([&](auto q) {
            if (i + decltype(q)::value < whole) get(q);
        });
        each<0, Q - 1>([&](auto q) {
            if (i + decltype(q)::value < whole) multiply(q, ra[decltype(q)::value], rb[decltype(q)::value], nothing);
        });
        // the steps that reach an end, piece by piece
        for (i = whole; i < steps; ++i) {
            __syncthreads();
#pragma unroll 1
            for (uint32_t idx = threadIdx.x; idx < N * 256; idx += 256) {
                *reinterpret_cast<u32x4*>(lds + place<AT, B>(idx)) = fetch<AT, B, false>(t.a, nullptr, m0, i * 64, t.k, idx);
                *reinterpret_cast<u32x4*>(lds + kTile + place<BT, B>(idx)) = fetch<BT, B, PAIR>(t.b, t.b2, n0, i * 64, t.k, idx);
            }
            __syncthreads();
            products(lds);
        }
    }
    __syncthreads();
    fin(acc, lds + wave * kStrip, m0 + wm * 32 * T, n0 + wn * (PAIR ? 16 : 32) * T, lane);
}

// ------------------------------------------------------- straight into LDS --
// Whether an operand's pieces of 16 bytes lie on 16-byte boundaries and are whole: then they
// can go straight into LDS.  (Offsets within a tile and a step have to fit 32 bits.)
inline bool whole_pieces(const Operand& o, int64_t k, bool across) {
    return reinterpret_cast<uintptr_t>(o.p) % 16 == 0 && o.stride % 8 == 0 && (across ? o.n : k) % 8 == 0 && o.stride < (int64_t(1) << 22);
}

// Which tile a product takes, by the microseconds of its rounds over the chip's 256 compute
// units for s steps of 64 summed elements.  256 x 256 and, with three stages, 256 x 128: one
// workgroup a unit, the fewer bytes read for a product the larger; 128 x 128: two, or one
// with four stages on the way where there are no more tiles than units; 64 x 64 with four
// stages: two.  Measured (256, 256 x 128, 128, 128 with four stages, 64; both operands along,
// microseconds): 8,192^3 774, 949, 999, 1,104 and 1,537 (1.42 PFLOP/s at best); 4,096^3 109, 122,
// 123, 141 and 199; 2,048 x 4,096 x 11,008 216, 157 and 164; 4,096 x 5,632 x 2,048 106, 95, 92,
// 112 and 145; 2,048 x 2,048 x 5,632 106, 72, 64, 49 and 73; 2,048^3 44, 29, 27, 22 and 29; 1,024 x
// 2,048 x 2,048 42, -, 24, 19 and 15; 1,024 x 1,024 x 4,096 74, -, 42, 31 and 19.  Operands across
// take the same within 5 %.  These are products that store one matrix; the rule knows nothing of what
// an epilogue reads and writes beyond that, and says 97 us for dh of 4,096 x 5,632 x 2,048 (136 measured
// among other calls), 160 for the projections of that size with g, u and h kept (204), 288 for 2,048 x 11,008
// x 4,096 with h alone (355).  Whether another tile would suit dh better was not measured.
enum TileSize { TILE_256, TILE_256_128, TILE_128, TILE_128_DEEP, TILE_64, TILE_SIZES };
inline double tile_us(TileSize size, int64_t tiles, double s) {
    const int64_t slots = size == TILE_128 || size == TILE_64 ? 512 : 256;
    const double full = static_cast<double>(tiles / slots), rest = static_cast<double>(tiles % slots);
    switch (size) {
        case TILE_256: return full * (1.36 * s + 12.0) + (rest > 0 ? (1.1 + 0.001 * rest) * s + 8.0 : 0.0);
        case TILE_256_128: return full * (0.9 * s + 4.0) + (rest > 0 ? (0.74 + 0.0006 * rest) * s + 5.0 : 0.0);
        case TILE_128: return full * (0.95 * s + 2.0) + (rest > 256 ? 0.95 * s + 2.0 : rest > 0 ? 0.7 * s + 3.8 : 0.0);
        case TILE_128_DEEP: return tiles > 256 ? 1e30 : 0.53 * s + 4.0;
        default: return full * (0.39 * s + 2.5) + (rest > 256 ? 0.39 * s + 2.5 : rest > 0 ? 0.25 * s + 3.3 : 0.0);
    }
}
constexpr int64_t tile_rows(TileSize size) { return size == TILE_256 || size == TILE_256_128 ? 256 : size == TILE_64 ? 64 : 128; }
constexpr int64_t tile_cols(TileSize size) { return size == TILE_256 ? 256 : size == TILE_64 ? 64 : 128; }
// The tiles of a result.  A pair's take half as many columns of each of its matrices, and 32 at least.
inline Tiles grid_of_product(TileSize size, int64_t rows, int64_t cols, bool pair) {
    const int64_t height = tile_rows(size), width = pair ? tile_cols(size) / 2 : tile_cols(size);
    return Tiles{(uint32_t)((rows + height - 1) / height), (uint32_t)((cols + width - 1) / width)};
}
// The size with the least time for rows x cols of k summed elements.
inline TileSize tile_of_product(int64_t rows, int64_t cols, int64_t k, bool pair) {
    TileSize best = TILE_128;
    double least = 1e300;
    for (int i = 0; i < TILE_SIZES; ++i) {
        const TileSize size = static_cast<TileSize>(i);
        if (pair && size == TILE_64) continue;
        const Tiles g = grid_of_product(size, rows, cols, pair);
        const double us = tile_us(size, (int64_t)g.mt * g.nt, static_cast<double>(k) / 64);
        if (us < least) {
            least = us;
            best = size;
        }
    }
    return best;
}
// f(integral_constants: a wave's 32 rows and 32 columns, stages) of a size.
template <typename F>
auto with_tile(TileSize size, F f) {
    using std::integral_constant;
    constexpr integral_constant<int, 1> one{};
    constexpr integral_constant<int, 2> two{};
    constexpr integral_constant<int, 3> three{};
    constexpr integral_constant<int, 4> four{};
    switch (size) {
        case TILE_256: return f(four, four, two);
        case TILE_256_128: return f(four, two, three);
        case TILE_128: return f(two, two, two);
        case TILE_128_DEEP: return f(two, two, four);
        default: return f(one, one, four);
    }
}
// Workgroups of such a tile a compute unit holds.
constexpr int tile_groups(int TM, int TN, int ST) { return (TM + TN) * ST > 8 ? 1 : 2; }

// A tile whose operands go straight from memory into LDS, no registers between, ST stages of
// 64 summed elements deep: while the matrix instructions work on one, the next arrive.
// Operands of the next 16 summed elements are read from LDS while the present ones are
// multiplied.  A load is one address register and one instruction: the operands' places move
// on by a step at a time, and the offsets of a lane's pieces are the same in every step, but for
// a last one that is not whole: there they are moved back inside, and what lies beyond the end
// is taken out of the operands before they are multiplied.  Of two terms the first is whole
// steps, and the second has its strides.
template <typename E, bool AT, bool BT, int TM, int TN, int ST, bool PAIR, typename Finish>
__device__ __forceinline__ void direct_tile(const Terms& terms, uint32_t ti, uint32_t tj, const Finish& fin) {
    constexpr int KS = 64, BA = 64 * TM, BB = 64 * TN, kTile = BA * 128, kStage = (BA + BB) * 128;
    constexpr int LA = 2 * TM, NL = LA + 2 * TN;       // a wave's loads for a stage: a's, all
    constexpr int kStrip = 32 * (32 * TN + 4) * 4;
    constexpr int RA = AT ? 2 * TM : TM, RB = BT ? 2 * TN : TN, NR = RA + RB;   // reads of LDS for 16 summed elements
    __shared__ __align__(1024) uint8_t lds[ST * kStage];
    static_assert(4 * kStrip <= ST * kStage, "the strips fit the stages");
    const uint32_t lane = threadIdx.x & 63;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t wm = wave >> 1, wn = wave & 1;
    const int64_t m0 = (int64_t)ti * BA, n0 = (int64_t)tj * (PAIR ? BB / 2 : BB);
    const Term& t0 = terms.t[0];
    const int64_t k_end = terms.t[terms.count - 1].k;
    const uint32_t last_steps = (uint32_t)((k_end + KS - 1) / KS);
    const uint32_t first = terms.count > 1 ? (uint32_t)(t0.k / KS) : ~0u;
    const uint32_t steps = terms.count > 1 ? first + last_steps : last_steps;
    const uint32_t rem = (uint32_t)(k_end - (int64_t)(last_steps - 1) * KS);   // of the last step: 1..KS

    // What this lane loads: segment wave + 4 j of an operand's kilobytes, 16 bytes a lane.
    // Along: 8 rows, the piece stored at lane % 8; across: K1 summed elements, the
    // piece stored at lane % (B / 8).  Rows beyond the last are the last again.
    const uint32_t along = (lane & 7) ^ ((wave & 1) << 2 | lane >> 4);
    const uint32_t sa = (uint32_t)t0.a.stride * 2, sb = (uint32_t)t0.b.stride * 2;
    uint32_t off[NL];
    each<0, NL>([&](auto which) {
        constexpr int j = decltype(which)::value;
        constexpr bool a = j < LA, tr = a ? AT : BT;
        constexpr int B = a ? BA : BB, K1 = 512 / B;
        const uint32_t seg = wave + 4 * (a ? j : j - LA), kk = lane / (B / 8);
        const Operand& o = a ? t0.a : t0.b;
        const int64_t at = a ? m0 : n0;
        if constexpr (tr) {
            const int64_t r = at + ((lane % (B / 8) >> 2) ^ exchange<B>(seg * K1 + kk)) * 32 + (lane & 3) * 8;
            off[j] = (seg * K1 + kk) * (a ? sa : sb) + (uint32_t)((r < o.n ? r : o.n - 8) - at) * 2;
        } else {
            const uint32_t row = 8 * seg + (lane >> 3), in = PAIR && !a ? (row >> 6) * 32 + (row & 31) : row;
            const int64_t r = at + in < o.n ? in : o.n - 1 - at;
            off[j] = (uint32_t)r * (a ? sa : sb) + along * 16;
        }
    });
    // Back inside the last step's `rem` summed elements.
    auto shorten = [&]() {
        each<0, NL>([&](auto which) {
            constexpr int j = decltype(which)::value;
            constexpr bool a = j < LA, tr = a ? AT : BT;
            constexpr int B = a ? BA : BB, K1 = 512 / B;
            const uint32_t k = tr ? (wave + 4 * (a ? j : j - LA)) * K1 + lane / (B / 8) : along * 8;
            if (k >= rem) off[j] -= tr ? (k - (rem - 1)) * (a ? sa : sb) : (k + 8 - rem) * 2;
        });
    };
    // The next stage to load: its operands' places and its place in LDS.
    auto begin = [](const Operand& o, const uint16_t* p, bool tr, int64_t at) {
        return reinterpret_cast<const char*>(p + (tr ? at : at * o.stride));
    };
    const char* pa = begin(t0.a, t0.a.p, AT, m0);
    const char* pb = begin(t0.b, t0.b.p, BT, n0);
    const char* pb2 = PAIR ? begin(t0.b, t0.b2, BT, n0) : pb;
    const int64_t da = AT ? (int64_t)KS * sa : KS * 2, db = BT ? (int64_t)KS * sb : KS * 2;
    uint32_t next = 0, into = 0;
    auto issue = [&](auto which) {
        typedef const void __attribute__((address_space(1)))* From;
        typedef void __attribute__((address_space(3)))* To;
        constexpr int j = decltype(which)::value;
        constexpr bool a = j < LA;
        const uint32_t seg = wave + 4 * (a ? j : j - LA);
        // of a pair's rows, 32 are of b and the next 32 of b2
        const char* base = a ? pa : PAIR && (seg >> 2 & 1) ? pb2 : pb;
        __builtin_amdgcn_global_load_lds((From)(const void*)(base + off[j]), (To)(lds + into + (a ? 0 : kTile) + seg * 1024), 16, 0, 0);
    };
    auto advance = [&]() {
        pa += da;
        pb += db;
        if constexpr (PAIR) pb2 += db;
        into = into + kStage == ST * kStage ? 0 : into + kStage;
        ++next;
        if (next == first) {
            pa = begin(terms.t[1].a, terms.t[1].a.p, AT, m0);
            pb = begin(terms.t[1].b, terms.t[1].b.p, BT, n0);
        }
        if (next + 1 == steps && rem < KS) shorten();
    };

    struct Frags {
        u32x4 a[TM], b[TN];
    };
    uint32_t now = 0, then = ST > 1 ? kStage : 0;   // the present stage and the next one
    // One of the NR reads of part s of a stage.
    auto read = [&](Frags& f, uint32_t stage, auto part, auto which) {
        constexpr int j = decltype(which)::value, s = decltype(part)::value;
        constexpr bool a = j < RA, tr = a ? AT : BT;
        constexpr int jj = a ? j : j - RA, t = tr ? jj / 2 : jj;
        const uint8_t* tile = lds + stage + (a ? 0 : kTile);
        constexpr int B = a ? BA : BB;
        const uint32_t row = ((a ? wm * TM : wn * TN) + t) * 32;
        u32x4& to = [&]() -> u32x4& {
            if constexpr (a)
                return f.a[t];
            else
                return f.b[t];
        }();
        if constexpr (tr) {
            const u32x2r v = turned_half<B>(tile, row, s, lane, jj & 1);
            to[2 * (jj & 1)] = v[0];
            to[2 * (jj & 1) + 1] = v[1];
        } else {
            to = operand_of<false, B>(tile, row, s, lane);
        }
    };
    f32x16 acc[TM][TN] = {};

    // Phases of 16 summed elements, TM * TN matrix instructions each.  Between them, in this
    // order (the scheduling barriers keep it): the reads of a later phase's operands in the
    // first half, loads of a later stage from the second quarter on.
    constexpr int NQ = TM * TN, QR = NQ > 1 ? NQ / 2 : 1;
    auto phase = [&](const Frags& f, auto reads, auto read_op, auto extras, auto extra_op) {
        constexpr int R = decltype(reads)::value, X = decltype(extras)::value;
        constexpr int QX = R == 0 || NQ == 1 ? 0 : NQ / 4;
        each<0, NQ>([&](auto slot) {
            constexpr int q = decltype(slot)::value, t = q / TN, u = q % TN;
            acc[t][u] = E::mfma(f.b[u], f.a[t], acc[t][u]);
            if constexpr (q < QR) each<R * q / QR, R * (q + 1) / QR>(read_op);
            if constexpr (q >= QX) each<X * (q - QX) / (NQ - QX), X * (q - QX + 1) / (NQ - QX)>(extra_op);
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    using std::integral_constant;
    auto nothing = [](auto) {};
    constexpr integral_constant<int, 0> none{}, c0{};
    constexpr integral_constant<int, 1> c1{};
    constexpr integral_constant<int, 2> c2{};
    constexpr integral_constant<int, 3> c3{};
    constexpr integral_constant<int, NR> operands{};
    constexpr int H = NL / 2;
    constexpr integral_constant<int, H> half{};
    constexpr integral_constant<int, NL - H> rest{};
    constexpr std::true_type yes{};
    constexpr std::false_type no{};
    constexpr int D = TM * TN == 16 ? 1 : 2;   // phases that operands are read ahead
    Frags f[2 * D];
    auto reading = [&](uint32_t stage, auto phase_of) {
        typedef decltype(phase_of) Part;   // the lambda outlives the parameter, whose type is all it needs
        return [&, stage](auto j) { read(f[Part::value % (2 * D)], stage, Part{}, j); };
    };
    auto run = [&](auto phase_of, auto more, auto x, auto x_op) {
        constexpr int s = decltype(phase_of)::value, to = (s + D) % 4;
        constexpr integral_constant<int, to> target{};
        if constexpr (s + D >= 4 && !decltype(more)::value)
            phase(f[s % (2 * D)], none, nothing, x, x_op);
        else
            phase(f[s % (2 * D)], operands, reading(s + D >= 4 ? then : now, target), x, x_op);
    };
    auto first_half = [&](auto j) { issue(j); };
    auto second_half = [&](auto j) { issue(integral_constant<int, H + decltype(j)::value>{}); };
    // A step.  At its barrier this stage is read and the next has arrived, those of the
    // ST - 2 stages after that may be on their way; another goes where this one was, half its
    // loads in each of the two phases after the barrier.  L: 2 all loads, 1 only those left of
    // a stage (D = 1: the second phase after the barrier is the next step's first), 0 none.
    auto step = [&](auto kind) {
        constexpr int L = decltype(kind)::value;
        if constexpr (D == 1) {
            if constexpr (L >= 1) {
                run(c0, yes, rest, second_half);
                advance();
            } else {
                run(c0, yes, none, nothing);
            }
            run(c1, yes, none, nothing);
            run(c2, yes, none, nothing);
        } else {
            run(c0, yes, none, nothing);
            run(c1, yes, none, nothing);
        }
        arrived<L == 2 ? (ST - 2) * NL : 0>();
        if constexpr (D == 2) {
            if constexpr (L == 2)
                run(c2, yes, half, first_half);
            else
                run(c2, yes, none, nothing);
        }
        if constexpr (D == 1 && L == 2) {
            run(c3, yes, half, first_half);
        } else if constexpr (D == 2 && L == 2) {
            run(c3, yes, rest, second_half);
            advance();
        } else {
            run(c3, yes, none, nothing);
        }
        now = then;
        then = then + kStage == ST * kStage ? 0 : then + kStage;
    };
    // Part s of the last stage, without what lies beyond its end.
    auto ending = [&](auto phase_of) {
        constexpr int s = decltype(phase_of)::value;
        if (rem < KS) {
            const int left = (int)rem - 16 * s - 8 * (int)(lane >> 5);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const uint32_t keep = left >= 2 * w + 2 ? ~0u : left == 2 * w + 1 ? 0xffffu : 0u;
#pragma unroll
                for (int t = 0; t < TM; ++t) f[s % (2 * D)].a[t][w] &= keep;
#pragma unroll
                for (int t = 0; t < TN; ++t) f[s % (2 * D)].b[t][w] &= keep;
            }
        }
        run(phase_of, no, none, nothing);
    };
    if (steps > 0) {
        if (steps == 1 && rem < KS) shorten();
        each<0, (D == 1 ? ST - 1 : ST)>([&](auto k) {
            if (decltype(k)::value < steps) {
                each<0, NL>(issue);
                advance();
            }
        });
        if (steps >= ST) {
            if constexpr (D == 1) each<0, H>(issue);
            arrived<D == 1 ? (ST - 2) * NL + H : (ST - 1) * NL>();
        } else {
            arrived<0>();
        }
        each<0, NR>(reading(0, c0));
        if constexpr (D == 2) each<0, NR>(reading(0, c1));
        uint32_t i = 0;
        for (; i + ST < steps; ++i) step(c2);
        if (D == 1 && i + ST == steps) {
            step(c1);
            ++i;
        }
        for (; i + 1 < steps; ++i) step(c0);
        ending(c0);
        ending(c1);
        ending(c2);
        ending(c3);
    }
    arrived<0>();
    fin(acc, lds + wave * kStrip, m0 + wm * 32 * TM, n0 + wn * (PAIR ? 16 : 32) * TN, lane);
}

}  // namespace autoloco
