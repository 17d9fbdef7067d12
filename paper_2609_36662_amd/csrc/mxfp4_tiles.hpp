// Products of 4-bit matrices in tiles of the result, on gfx950.
//
// A workgroup of four waves (2 x 2) takes 64 T x 64 T of the result, a wave 32 T x 32 T,
// in steps of 256 columns.  Both operands' codes (16 bytes a lane) and scales (a word for
// 128 columns of a row) go straight from memory into LDS, no registers between, ST
// stages deep: while the matrix instructions work on one, the next arrive.  A row takes
// 128 bytes of a stage; its eight pieces of 16 bytes are stored at place
// piece ^ (row / 2 % 8), so that 16 neighbouring rows' pieces of one column range lie in 64
// different banks.  Operands of later columns are read from LDS while the present ones
// are multiplied.
//
// 8,192 x 8,192 x 8,192 takes 257 us (4.3 PFLOP/s; a bf16 product of that size by the
// vendor's library 0.79 ms) with random codes and 203 with zeros, 4,096 x 11,008 x 4,096 105
// and 92 (each with its counters; in a loop of calls 247 and 195, 96 and 85).  The difference is
// the clock, which power brings down (2.4 GHz with zeros, 1.90 and 2.10 with random
// codes).  The matrix cores are busy 54 % and 40 % of the cycles with either: the rest is a
// loop that waits and the fixed cost of a tile (9 us at 256 x 256: filling the stages, the
// result's way out).
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

// Waits until at most N of a wave's loads are outstanding and its LDS reads are done,
// then meets the other waves.
template <int N>
__device__ __forceinline__ void wait_and_meet() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

template <int T, int ST, bool BF16>
__global__ void __launch_bounds__(256, T == 1 || (T == 2 && ST == 2) ? 2 : 1) mx_tile_kernel(Mx4 a, Mx4 b, MatrixOut out, TileGrid grid) {
    constexpr int B = 64 * T;                   // rows of either operand
    constexpr int kCodes = 2 * B * 128, kStage = kCodes + 2 * B * 8;
    constexpr int LA = 2 * T, NL = 4 * T, NV = NL + T;   // a wave's loads for a stage: a's codes, all codes, and scales
    __shared__ __align__(1024) uint8_t lds[ST * kStage];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave >> 1, wn = wave & 1;
    uint32_t ti, tj;
    tile_of(blockIdx.x, grid, ti, tj);
    const int64_t m0 = (int64_t)ti * B, n0 = (int64_t)tj * B;
    const int groups = a.groups, steps = (groups + 1) / 2;

    // What this lane loads.  Codes: row 8 p + lane / 8 of segment p = wave + 4 j, the piece
    // stored at lane % 8.  Scales: 64 rows' words of one group of one operand a segment,
    // a's two groups before b's.
    const int piece = (lane & 7) ^ (((wave & 1) << 2) | (lane >> 4));
    auto inside = [](int64_t r0, int r, const Mx4& x) { return (uint32_t)(r0 + r < x.rows ? r : x.rows - 1 - r0); };
    uint32_t co[NL], so[T];
    unrolled<NL>([&](auto which) {
        constexpr int j = decltype(which)::value;
        const int row = 8 * (wave + 4 * (j < LA ? j : j - LA)) + (lane >> 3);
        co[j] = (j < LA ? inside(m0, row, a) * (uint32_t)a.row_bytes : inside(n0, row, b) * (uint32_t)b.row_bytes) + piece * 16;
    });
    unrolled<T>([&](auto which) {
        constexpr int j = decltype(which)::value;
        const int seg = wave + 4 * j, row = (seg % T) * 64 + lane;
        so[j] = (seg < 2 * T ? inside(m0, row, a) : inside(n0, row, b)) * 4;
    });
    const uint8_t* abase = a.codes + m0 * a.row_bytes;
    const uint8_t* bbase = b.codes + n0 * b.row_bytes;
    // One of a wave's NV loads for stage i.  In a last step of 128 columns the upper
    // pieces (and the second group's scales) are not there: the lower ones are taken again.
    const uint32_t lower = (uint32_t)(((piece & 3) - piece) * 16);
    auto issue = [&](int i, auto which) {
        constexpr int j = decltype(which)::value;
        typedef const void __attribute__((address_space(1)))* From;
        typedef void __attribute__((address_space(3)))* To;
        uint8_t* stage = lds + (i % ST) * kStage;
        if constexpr (j < NL) {
            const uint32_t at = 2 * i + 1 < groups ? 0u : lower;
            const uint8_t* src = (j < LA ? abase : bbase) + (int64_t)i * 128 + (uint32_t)(co[j] + at);
            __builtin_amdgcn_global_load_lds((From)(const void*)src, (To)(stage + wave * 1024 + j * 4096), 16, 0, 0);
        } else {
            const int seg = wave + 4 * (j - NL), second = seg % (2 * T) / T;
            const int64_t g = 2 * i + second < groups ? 2 * i + second : groups - 1;
            const uint8_t* src = seg < 2 * T ? a.scales + (g * a.rows + m0) * 4 : b.scales + (g * b.rows + n0) * 4;
            __builtin_amdgcn_global_load_lds((From)(const void*)(src + so[j - NL]), (To)(stage + kCodes + seg * 256), 4, 0, 0);
        }
    };

    // What this lane multiplies: rows lane % 32 of each 32, columns 32 (lane / 32) on of each 64.
    const int r = lane & 31, h = lane >> 5;
    struct Frags {
        u32x4 a[T], b[T];
    };
    struct Scales {
        uint32_t a[T], b[T];
    };
    // One of the 2 T operands of phase s of stage i; for even s, beyond them, one of the 2 T
    // words of scales of it and the next.
    auto read = [&](Frags& f, Scales& sc, int i, int s, auto which) {
        constexpr int j = decltype(which)::value, t = j % T;
        const uint8_t* stage = lds + (i % ST) * kStage;
        if constexpr (j < 2 * T) {
            const uint8_t* p = stage + r * 128 + (((2 * s + h) ^ (r >> 1 & 7)) << 4);
            if constexpr (j < T)
                f.a[t] = *reinterpret_cast<const u32x4*>(p + (wm * T + t) * 4096);
            else
                f.b[t] = *reinterpret_cast<const u32x4*>(p + B * 128 + (wn * T + t) * 4096);
        } else {
            const uint8_t* p = stage + kCodes + (s >> 1) * (B * 4) + r * 4;
            if constexpr (j < 3 * T)
                sc.a[t] = *reinterpret_cast<const uint32_t*>(p + (wm * T + t) * 128);
            else
                sc.b[t] = *reinterpret_cast<const uint32_t*>(p + B * 8 + (wn * T + t) * 128);
        }
    };
    f32x16 acc[T][T] = {};

    // Phases of 64 columns, T * T matrix instructions each.  Between them, in this order
    // (the scheduling barriers keep it): the reads of the next phase's operands, then
    // loads of a later stage.  Left alone, all reads of a step go first and all products
    // wait for them; a stage's loads in one run keep the matrix cores waiting while the
    // four waves queue at the address unit.
    constexpr int NQ = T * T, QR = NQ > 1 ? NQ / 2 : 1;   // slots; those that read operands
    auto phase = [&](const Frags& f, const Scales& sc, auto odd, auto reads, auto read_op, auto extras, auto extra_op) {
        constexpr int R = decltype(reads)::value, X = decltype(extras)::value, sel = 2 * decltype(odd)::value;
        constexpr int QX = R == 0 || NQ == 1 ? 0 : QR;      // the first slot with other loads
        unrolled<NQ>([&](auto slot) {
            constexpr int q = decltype(slot)::value, t = q / T, u = q % T;
            acc[t][u] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(f.b[u]), operand(f.a[t]), acc[t][u], 4, 4, sel,
                                                                        (int)(sc.b[u] >> (8 * h)), sel, (int)(sc.a[t] >> (8 * h)));
            if constexpr (q < QR) unrolled<R * q / QR, R * (q + 1) / QR>(read_op);
            if constexpr (q >= QX) unrolled<X * (q - QX) / (NQ - QX), X * (q - QX + 1) / (NQ - QX)>(extra_op);
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    using std::integral_constant;
    auto nothing = [](auto) {};
    constexpr integral_constant<int, 0> none{}, first{};
    constexpr integral_constant<int, 1> second{};
    constexpr integral_constant<int, 2 * T> operands{};
    constexpr integral_constant<int, 4 * T> with_scales{};
    constexpr int H = NV / 2;
    constexpr integral_constant<int, H> half{};
    constexpr integral_constant<int, NV - H> rest{};
    constexpr integral_constant<int, 2> third{};
    constexpr integral_constant<int, 3> fourth{};
    constexpr std::true_type yes{};
    constexpr std::false_type no{};
    // Operands are read D phases ahead: one where a phase takes longer than a reading of
    // LDS, else two.
    constexpr int D = T == 4 ? 1 : 2;
    Frags f[2 * D];
    Scales sc[2];
    int i = 0;
    auto reading = [&](int at, auto phase_of) {
        return [&, at](auto j) {
            constexpr int s = decltype(phase_of)::value;
            read(f[s % (2 * D)], sc[s / 2], at, s, j);
        };
    };
    // Phase s of step i; it reads the operands of phase s + D (next: also those of the
    // next step) and issues the loads x.
    auto run = [&](auto phase_of, auto next, auto x, auto x_op) {
        constexpr int s = decltype(phase_of)::value, to = (s + D) % 4;
        constexpr integral_constant<int, s % 2> odd{};
        constexpr integral_constant<int, to> target{};
        const Frags& now = f[s % (2 * D)];
        if constexpr (s + D >= 4 && !decltype(next)::value)
            phase(now, sc[s / 2], odd, none, nothing, x, x_op);
        else if constexpr (to % 2 == 0)
            phase(now, sc[s / 2], odd, with_scales, reading(s + D >= 4 ? i + 1 : i, target), x, x_op);
        else
            phase(now, sc[s / 2], odd, operands, reading(s + D >= 4 ? i + 1 : i, target), x, x_op);
    };
    // A step.  At its barrier this stage is read and the next has arrived, those of the
    // ST - 2 stages after that may be on their way; stage i + ST goes where this one was,
    // half its loads in each of the two phases after the barrier.  L: 2 all loads, 1 only
    // those left of a stage (D = 1: the second phase after the barrier is the next step's
    // first), 0 none.
    auto first_half = [&](auto j) { issue(i + ST, j); };
    auto step = [&](auto kind) {
        constexpr int L = decltype(kind)::value;
        if constexpr (D == 1) {
            if constexpr (L >= 1)
                run(first, yes, rest, [&](auto j) { issue(i + ST - 1, integral_constant<int, H + decltype(j)::value>{}); });
            else
                run(first, yes, none, nothing);
            run(second, yes, none, nothing);
            run(third, yes, none, nothing);
        } else {
            run(first, yes, none, nothing);
            run(second, yes, none, nothing);
        }
        wait_and_meet<L == 2 ? (ST - 2) * NV : 0>();
        if constexpr (D == 2) {
            if constexpr (L == 2)
                run(third, yes, half, first_half);
            else
                run(third, yes, none, nothing);
        }
        if constexpr (D == 1 && L == 2)
            run(fourth, yes, half, first_half);
        else if constexpr (D == 2 && L == 2)
            run(fourth, yes, rest, [&](auto j) { issue(i + ST, integral_constant<int, H + decltype(j)::value>{}); });
        else
            run(fourth, yes, none, nothing);
        ++i;
    };
    unrolled<(D == 1 ? ST - 1 : ST)>([&](auto k) {
        constexpr int stage = decltype(k)::value;
        if (stage < steps) unrolled<NV>([&](auto j) { issue(stage, j); });
    });
    if (steps >= ST) {
        if constexpr (D == 1) unrolled<H>([&](auto j) { issue(ST - 1, j); });
        wait_and_meet<D == 1 ? (ST - 2) * NV + H : (ST - 1) * NV>();
    } else {
        wait_and_meet<0>();
    }
    unrolled<4 * T>(reading(0, first));
    if constexpr (D == 2) unrolled<2 * T>(reading(0, second));
    while (i + ST < steps) step(third);
    if (D == 1 && i + ST == steps) step(second);
    while (i + 1 < steps) step(first);
    run(first, no, none, nothing);
    run(second, no, none, nothing);
    if (2 * i + 1 < groups) {
        run(third, no, none, nothing);
        run(fourth, no, none, nothing);
    }
    // b's rows come first, so a lane has row lane % 32 of a 32 x 32 piece and its columns
    // 8 (i / 4) + 4 (lane / 32) + i % 4: four neighbours at a time.  They go through LDS,
    // 32 rows of the wave's own at a time, and out in whole rows.  (Written straight from
    // the registers, an unrolled store per value is 30 KB of code that runs once.)
    wait_and_meet<0>();
    constexpr int E = BF16 ? 2 : 4;
    constexpr int kPitch = 32 * T * E + 16;
    uint8_t* strip = lds + wave * 32 * kPitch;
    static_assert(4 * 32 * kPitch <= ST * kStage, "the strips fit the stages");
#pragma unroll
    for (int t = 0; t < T; ++t) {
#pragma unroll
        for (int u = 0; u < T; ++u)
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
        constexpr int P = 32 * T * E / 16;   // pieces of 16 bytes in a row
        const int64_t n = n0 + wn * 32 * T + (lane % P) * (16 / E);
        const int64_t m = m0 + (wm * T + t) * 32;
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
