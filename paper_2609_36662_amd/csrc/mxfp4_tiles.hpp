// Products of 4-bit matrices in tiles of the result, on gfx950.
//
// A workgroup of four waves (2 x 2) takes 64 T x 64 T of the result, a wave 32 T x 32 T,
// in steps of 256 columns.  Both operands' codes go straight from memory into LDS (16
// bytes a lane, no registers), two stages deep: while the matrix instructions work on
// one, the next arrives.  A row takes 128 bytes of a stage; its eight pieces of 16 bytes
// are stored at place piece ^ (row / 2 % 8), so that 16 neighbouring rows' pieces of one
// column range lie in 64 different banks.  The scales, a word for 128 columns of a row,
// go to registers.  Operands of the next 64 columns are read from LDS while the present
// ones are multiplied.
//
// Bound by power at large sizes: 8,192 x 8,192 x 8,192 takes 263 us (4.2 PFLOP/s) with
// random codes and 185 us (5.9) with zeros, at the same instructions; a bf16 product of
// that size by the vendor's library takes 0.80 ms.  Beyond a few rounds of tiles the
// fixed cost of a tile counts (9 us at 256 x 256: filling two stages, the result's way out).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "mxfp4_kernels.hpp"

namespace autoloco {

// f(integral_constant j) for j from FROM up to TO.
template <int FROM, int TO, typename F>
__device__ __forceinline__ void unrolled(F&& f) {
    if constexpr (FROM < TO) {
        f(std::integral_constant<int, FROM>{});
        unrolled<FROM + 1, TO>(f);
    }
}
template <int N, typename F>
__device__ __forceinline__ void unrolled(F&& f) {
    unrolled<0, N>(f);
}

// Tiles of the result by rows and columns, and how workgroups go through them.
struct TileGrid {
    uint32_t mt, nt;
};

// The tile of workgroup b: workgroups go round the eight dies (each with a cache of
// its own), so each die gets a run of neighbouring tiles, eight rows of tiles wide.
__device__ __forceinline__ void tile_of(uint32_t b, const TileGrid& g, uint32_t& m, uint32_t& n) {
    const uint32_t total = g.mt * g.nt, per = total / 8, extra = total % 8;
    const uint32_t die = b % 8, i = b / 8;
    const uint32_t t = die * per + (die < extra ? die : extra) + i;
    const uint32_t band = t / (8 * g.nt), first = band * 8;
    const uint32_t height = g.mt - first < 8 ? g.mt - first : 8;
    const uint32_t in = t - band * 8 * g.nt;
    m = first + in % height;
    n = in / height;
}

template <int T, bool BF16>
__global__ void __launch_bounds__(256, T == 4 ? 1 : 2) mx_tile_kernel(Mx4 a, Mx4 b, MatrixOut out, TileGrid grid) {
    constexpr int TM = T, TN = T;
    constexpr int BM = 64 * TM, BN = 64 * TN;
    constexpr int kStage = (BM + BN) * 128;
    constexpr int LA = BM / 32, LB = BN / 32;   // loads of a wave for a stage
    __shared__ __align__(1024) uint8_t lds[2 * kStage];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave >> 1, wn = wave & 1;
    uint32_t ti, tj;
    tile_of(blockIdx.x, grid, ti, tj);
    const int64_t m0 = (int64_t)ti * BM, n0 = (int64_t)tj * BN;
    const int groups = a.groups, steps = (groups + 1) / 2;

    // what this lane loads: row 8 p + lane / 8 of segment p = wave + 4 j, the piece stored at lane % 8
    const int piece = (lane & 7) ^ (((wave & 1) << 2) | (lane >> 4));
    uint32_t ao[LA], bo[LB];
    const uint8_t* abase = a.codes + m0 * a.row_bytes;
    const uint8_t* bbase = b.codes + n0 * b.row_bytes;
    auto row_offset = [&](int64_t r0, int j, const Mx4& x) {
        int64_t r = 8 * (wave + 4 * j) + (lane >> 3);
        if (r0 + r >= x.rows) r = x.rows - 1 - r0;
        return (uint32_t)(r * x.row_bytes);
    };
#pragma unroll
    for (int j = 0; j < LA; ++j) ao[j] = row_offset(m0, j, a) + piece * 16;
#pragma unroll
    for (int j = 0; j < LB; ++j) bo[j] = row_offset(n0, j, b) + piece * 16;
    // One of a wave's LA + LB loads for stage i.  In a last step of 128 columns the upper
    // pieces are not there: the lower ones are taken again.
    const uint32_t lower = (uint32_t)(((piece & 3) - piece) * 16);
    auto issue = [&](int i, auto which) {
        constexpr int j = decltype(which)::value;
        const uint32_t at = 2 * i + 1 < groups ? 0u : lower;
        const uint8_t* src;
        if constexpr (j < LA)
            src = abase + (int64_t)i * 128 + (uint32_t)(ao[j] + at);
        else
            src = bbase + (int64_t)i * 128 + (uint32_t)(bo[j - LA] + at);
        __builtin_amdgcn_global_load_lds((const void __attribute__((address_space(1)))*)(const void*)src,
                                         (void __attribute__((address_space(3)))*)(lds + (i & 1) * kStage + wave * 1024 + j * 4096),
                                         16, 0, 0);
    };

    // what this lane multiplies: rows lane % 32 of each 32, columns 32 (lane / 32) on of each 64
    const int r = lane & 31, h = lane >> 5;
    uint32_t as[TM], bs[TN];   // byte offsets of the rows' scale words
#pragma unroll
    for (int t = 0; t < TM; ++t) {
        const int64_t m = m0 + wm * 32 * TM + t * 32 + r;
        as[t] = (uint32_t)((m < a.rows ? m : a.rows - 1) - m0) * 4;
    }
#pragma unroll
    for (int t = 0; t < TN; ++t) {
        const int64_t n = n0 + wn * 32 * TN + t * 32 + r;
        bs[t] = (uint32_t)((n < b.rows ? n : b.rows - 1) - n0) * 4;
    }
    struct Scales {
        uint32_t a[2][TM], b[2][TN];
    };
    constexpr int NS = 2 * (TM + TN);
    auto load_scale = [&](Scales& s, int i, auto which) {   // one of the NS words of step i
        constexpr int g = decltype(which)::value & 1, t = decltype(which)::value >> 1;
        const int64_t q = 2 * i + g < groups ? 2 * i + g : groups - 1;
        if constexpr (t < TM)
            s.a[g][t] = *reinterpret_cast<const uint32_t*>(a.scales + (q * a.rows + m0) * 4 + as[t]);
        else
            s.b[g][t - TM] = *reinterpret_cast<const uint32_t*>(b.scales + (q * b.rows + n0) * 4 + bs[t - TM]);
    };
    struct Frags {
        u32x4 a[TM], b[TN];
    };
    constexpr int NR = TM + TN;
    auto read = [&](Frags& f, int i, int s, auto which) {   // one of the NR operands of phase s of stage i
        constexpr int t = decltype(which)::value;
        const uint8_t* p = lds + (i & 1) * kStage + r * 128 + (((2 * s + h) ^ (r >> 1 & 7)) << 4);
        if constexpr (t < TM)
            f.a[t] = *reinterpret_cast<const u32x4*>(p + (wm * TM + t) * 4096);
        else
            f.b[t - TM] = *reinterpret_cast<const u32x4*>(p + BM * 128 + (wn * TN + t - TM) * 4096);
    };
    f32x16 acc[TM][TN] = {};

    // Phases of 64 columns, TM TN matrix instructions each.  Between them, in this order
    // (the scheduling barriers keep it): the reads of the next phase's operands, then
    // other loads.  Left alone, all reads of a step go first and all products wait for
    // them; a stage's loads in one run keep the matrix cores waiting while the four waves
    // queue at the address unit.
    constexpr int NQ = TM * TN, QR = NQ > 1 ? NQ / 2 : 1;   // slots; those that read operands
    auto phase = [&](const Frags& f, const Scales& sc, auto sub, auto reads, auto read_op, auto extras, auto extra_op) {
        constexpr int S = decltype(sub)::value, R = decltype(reads)::value, X = decltype(extras)::value;
        constexpr int QX = R == 0 || NQ == 1 ? 0 : QR;      // the first slot with other loads
        unrolled<NQ>([&](auto slot) {
            constexpr int q = decltype(slot)::value, t = q / TN, u = q % TN;
            acc[t][u] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
                operand(f.b[u]), operand(f.a[t]), acc[t][u], 4, 4, 2 * (S & 1), (int)(sc.b[S >> 1][u] >> (8 * h)),
                2 * (S & 1), (int)(sc.a[S >> 1][t] >> (8 * h)));
            if constexpr (q < QR) unrolled<R * q / QR, R * (q + 1) / QR>(read_op);
            if constexpr (q >= QX) unrolled<X * (q - QX) / (NQ - QX), X * (q - QX + 1) / (NQ - QX)>(extra_op);
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    using std::integral_constant;
    constexpr int NL = LA + LB;
    auto nothing = [](auto) {};
    constexpr integral_constant<int, 0> none{};
    constexpr integral_constant<int, NL / 2> loads{};
    constexpr integral_constant<int, NR> reads{};
    constexpr integral_constant<int, NS> words{};
    auto reading = [&](Frags& f, int i, int s) { return [&f, &read, i, s](auto j) { read(f, i, s, j); }; };
    Scales sc, next;
    Frags f0, f1;
    unrolled<NL>([&](auto j) { issue(0, j); });
    unrolled<NS>([&](auto j) { load_scale(sc, 0, j); });
    __syncthreads();
    if (steps > 1) unrolled<NL / 2>([&](auto j) { issue(1, j); });
    unrolled<NR>(reading(f0, 0, 0));
    int i = 0;
    auto step = [&](auto more) {
        phase(f0, sc, integral_constant<int, 0>{}, reads, reading(f1, i, 1), loads,
              [&](auto j) { issue(i + 1, integral_constant<int, NL / 2 + decltype(j)::value>{}); });
        phase(f1, sc, integral_constant<int, 1>{}, reads, reading(f0, i, 2), words, [&](auto j) { load_scale(next, i + 1, j); });
        phase(f0, sc, integral_constant<int, 2>{}, reads, reading(f1, i, 3), none, nothing);
        // this stage is read, the next has arrived; the one after it goes where this one was
        __syncthreads();
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (decltype(more)::value)
            phase(f1, sc, integral_constant<int, 3>{}, reads, reading(f0, i + 1, 0), loads, [&](auto j) { issue(i + 2, j); });
        else
            phase(f1, sc, integral_constant<int, 3>{}, reads, reading(f0, i + 1, 0), none, nothing);
        sc = next;
    };
    for (; i + 2 < steps; ++i) step(std::true_type{});
    if (i + 1 < steps) {
        step(std::false_type{});
        ++i;
    }
    phase(f0, sc, integral_constant<int, 0>{}, reads, reading(f1, i, 1), none, nothing);
    if (2 * i + 1 < groups) {
        phase(f1, sc, integral_constant<int, 1>{}, reads, reading(f0, i, 2), none, nothing);
        phase(f0, sc, integral_constant<int, 2>{}, reads, reading(f1, i, 3), none, nothing);
        phase(f1, sc, integral_constant<int, 3>{}, none, nothing, none, nothing);
    } else {
        phase(f1, sc, integral_constant<int, 1>{}, none, nothing, none, nothing);
    }
    // b's rows come first, so a lane has row lane % 32 of a 32 x 32 piece and its columns
    // 8 (i / 4) + 4 (lane / 32) + i % 4: four neighbours at a time.  They go through LDS,
    // 32 rows of the wave's own at a time, and out in whole rows.  (Written straight from
    // the registers, an unrolled store per value is 30 KB of code that runs once.)
    __syncthreads();
    constexpr int E = BF16 ? 2 : 4;
    constexpr int kPitch = 32 * TN * E + 16;
    uint8_t* strip = lds + wave * 32 * kPitch;
    static_assert(4 * 32 * kPitch <= 2 * kStage, "the strips fit the stages");
#pragma unroll
    for (int t = 0; t < TM; ++t) {
#pragma unroll
        for (int u = 0; u < TN; ++u)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f32x4 v = {acc[t][u][4 * q], acc[t][u][4 * q + 1], acc[t][u][4 * q + 2], acc[t][u][4 * q + 3]};
                uint8_t* to = strip + r * kPitch + (u * 32 + 8 * q + 4 * h) * E;
                if constexpr (BF16)
                    *reinterpret_cast<u32x2r*>(to) = u32x2r{bf16_pack(v[0], v[1]), bf16_pack(v[2], v[3])};
                else
                    *reinterpret_cast<f32x4*>(to) = v;
            }
        __builtin_amdgcn_wave_barrier();
        constexpr int P = 32 * TN * E / 16;   // pieces of 16 bytes in a row
        const int64_t n = n0 + wn * 32 * TN + (lane % P) * (16 / E);
        const int64_t m = m0 + (wm * TM + t) * 32;
        uint8_t* row = static_cast<uint8_t*>(out.data) + n * E;
#pragma unroll 1
        for (int k = lane / P; k < 32 && m + k < out.rows; k += 64 / P) {
            const u32x4 v = *reinterpret_cast<const u32x4*>(strip + k * kPitch + (lane % P) * 16);
            uint8_t* to = row + (m + k) * out.stride * E;
            if (n + 16 / E <= out.cols) {
                *reinterpret_cast<u32x4_any*>(to) = v;
            } else {
#pragma unroll
                for (int e = 0; e < 16 / E; ++e)
                    if (n + e < out.cols) {
                        if constexpr (BF16)
                            reinterpret_cast<uint16_t*>(to)[e] = (uint16_t)(v[e / 2] >> (16 * (e & 1)));
                        else
                            reinterpret_cast<uint32_t*>(to)[e] = v[e];
                    }
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

}  // namespace autoloco
