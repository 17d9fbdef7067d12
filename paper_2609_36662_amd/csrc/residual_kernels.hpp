// The norms between two blocks with the gate and the residual scale, on gfx950.
//
//   b = z or wz z rz,   out = x + s gate b,   y = w out r,   r = (mean out^2 + eps)^(-1/2) (rz of z alike)
// and with t = dy w, n = out r:
//   dout' = dout + r (t - n mean(t n)),   dw = sum over rows of dy n
//   dgate = s dout' b,   db = s gate dout',   tz = db wz, nz = z rz:
//   dz = rz (tz - nz mean(tz nz)),   dwz = sum over rows of db nz
//
// A row is read once, by W waves, and stays in their registers, C runs of 8 columns a
// lane, as they lie in memory; sums over a row are fp32, joined over the lanes and then through
// LDS.  In the backward pass a team of waves goes from row to row and keeps its columns' part
// of dw, dwz and a channel's dgate in registers; the workgroups' parts are added up in fp64, in a
// fixed order, by a second kernel.
// Bound by HBM: 16,384 x 2,048 bf16 among other calls 56 to 57 us forward (4.7 TB/s), 84 to 88 us
// backward (4.7 TB/s) and 13 us for the second kernel (96 workgroups that each add up 128 KB); a
// loop over the same rows finds a part of them in the last cache (45, 81 and 7).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "matrix_view.hpp"

namespace autoloco {

constexpr int64_t kMaxNormCols = int64_t(1) << 15;
// Workgroups of the backward pass at most, and partial sums of a column.
constexpr int kNormParts = 1024, kNormPartsWide = 256;
constexpr int norm_parts(int64_t cols) { return cols <= 2048 ? kNormParts : kNormPartsWide; }

struct Residual {
    MatrixView x, z, gate;   // z, gate: data null where absent
    const float* weight;     // null: ones
    const float* z_weight;   // null: z is not normed
    MatrixOut out, y;        // data null where not wanted
    float scale, eps;
};
struct ResidualGrad {
    MatrixView out, z, gate, dy, dout;
    const float* weight;
    const float* z_weight;
    MatrixOut dx, dz, dgate;
    float* dweight;
    float* dz_weight;
    float* work;            // [3][workgroups][cols]
    float scale, eps;
    bool channel;           // dgate is one row, summed over all
};

// Eight neighbours as they lie in memory.
template <bool BF16>
struct Run8 {
    u32x4 w[BF16 ? 1 : 2];
    __device__ __forceinline__ void load(const void* p, int64_t i, int64_t left) {
        if (left >= 8) {
#pragma unroll
            for (int j = 0; j < (BF16 ? 1 : 2); ++j)
                w[j] = __builtin_bit_cast(u32x4, reinterpret_cast<const u32x4_any*>(static_cast<const char*>(p) + i * (BF16 ? 2 : 4))[j]);
        } else {
            float v[8];
            load8<BF16>(v, p, i, left);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (BF16) {
                    w[0][j] = (__float_as_uint(v[2 * j]) >> 16) | (__float_as_uint(v[2 * j + 1]) & 0xffff0000u);
                } else {
                    w[0][j] = __float_as_uint(v[j]);
                    w[1][j] = __float_as_uint(v[4 + j]);
                }
            }
        }
    }
    __device__ __forceinline__ float operator[](int e) const {
        if constexpr (BF16)
            return __uint_as_float(e & 1 ? w[0][e / 2] & 0xffff0000u : w[0][e / 2] << 16);
        else
            return __uint_as_float(w[e / 4][e % 4]);
    }
};

// The sum over a wave, in every lane.
__device__ __forceinline__ float wave_sum(float a) {
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) a += __shfl_xor(a, m);
    return a;
}
// The team's W waves' sums of a and b, in every lane.  Two places in LDS in turn, so that
// one barrier a call is enough.
template <int W>
__device__ __forceinline__ void team_sum(float& a, float& b, float (&lds)[2][2][W], int& turn) {
    a = wave_sum(a);
    b = wave_sum(b);
    if constexpr (W > 1) {
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) {
            lds[turn][0][wave] = a;
            lds[turn][1][wave] = b;
        }
        __syncthreads();
        a = b = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            a += lds[turn][0][w];
            b += lds[turn][1][w];
        }
        turn ^= 1;
    }
}
__device__ __forceinline__ float inverse_rms(float sum, int64_t cols, float eps) {
    return 1.f / sqrtf(sum / (float)cols + eps);
}

constexpr int team_threads(int w) { return w == 1 ? 256 : 64 * w; }   // of a workgroup: four teams of a wave, or one

template <bool BF16, int W, int C>
__global__ void __launch_bounds__(team_threads(W)) residual_norm_kernel(Residual a) {
    __shared__ float lds[2][2][W];
    int turn = 0;
    const int lane = W == 1 ? threadIdx.x & 63 : threadIdx.x;
    const int64_t cols = a.x.cols;
    constexpr int kTeams = W == 1 ? 4 : 1;
    const bool post = a.z_weight != nullptr, has_z = a.z.data != nullptr, gated = a.gate.data != nullptr;
    auto at = [&](int c) { return (int64_t)(c * W * 64 + lane) * 8; };
    for (int64_t row = (int64_t)blockIdx.x * kTeams + (W == 1 ? threadIdx.x >> 6 : 0); row < a.x.rows; row += (int64_t)gridDim.x * kTeams) {
        Run8<BF16> x[C], z[C], g[C];
#pragma unroll
        for (int c = 0; c < C; ++c) x[c].load(a.x.data, row * a.x.stride + at(c), cols - at(c));
        if (has_z) {
#pragma unroll
            for (int c = 0; c < C; ++c) z[c].load(a.z.data, row * a.z.stride + at(c), cols - at(c));
            if (gated)
#pragma unroll
                for (int c = 0; c < C; ++c) g[c].load(a.gate.data, row * a.gate.stride + at(c), cols - at(c));
        }
        float v[C][8], none = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[c][e] = x[c][e];
        if (has_z) {
            float r = 1.f;
            if (post) {
                float ss = 0.f;
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int e = 0; e < 8; ++e) ss += z[c][e] * z[c][e];
                team_sum<W>(ss, none, lds, turn);
                r = inverse_rms(ss, cols, a.eps);
            }
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float wz[8];
                if (post) load8<false>(wz, a.z_weight, at(c), cols - at(c));
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float b = post ? z[c][e] * r * wz[e] : z[c][e];
                    v[c][e] += (gated ? a.scale * g[c][e] : a.scale) * b;
                }
                store8<BF16>(a.out.data, row * a.out.stride + at(c), v[c], cols - at(c));
            }
        }
        if (a.y.data != nullptr) {
            float ss = 0.f;
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int e = 0; e < 8; ++e) ss += at(c) + e < cols ? v[c][e] * v[c][e] : 0.f;
            team_sum<W>(ss, none, lds, turn);
            const float r = inverse_rms(ss, cols, a.eps);
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float w[8], y[8];
                if (a.weight != nullptr) load8<false>(w, a.weight, at(c), cols - at(c));
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = a.weight != nullptr ? v[c][e] * r * w[e] : v[c][e] * r;
                store8<BF16>(a.y.data, row * a.y.stride + at(c), y, cols - at(c));
            }
        }
    }
}

template <bool BF16, int W, int C>
__global__ void __launch_bounds__(team_threads(W)) residual_grad_kernel(ResidualGrad a) {
    __shared__ float lds[2][2][W];
    int turn = 0;
    const int lane = W == 1 ? threadIdx.x & 63 : threadIdx.x;
    const int64_t cols = a.out.cols;
    constexpr int kTeams = W == 1 ? 4 : 1;
    const int wave = W == 1 ? threadIdx.x >> 6 : 0;
    const int64_t teams = (int64_t)gridDim.x * kTeams;
    const bool post = a.z_weight != nullptr, has_z = a.z.data != nullptr, gated = a.gate.data != nullptr, by_y = a.dy.data != nullptr;
    const float inv = 1.f / (float)cols;
    auto at = [&](int c) { return (int64_t)(c * W * 64 + lane) * 8; };
    float dw[C][8] = {}, dwz[C][8] = {}, dg[C][8] = {};
    struct Rows {
        Run8<BF16> o[C], dy[C], z[C], g[C], up[C];
    };
    auto fetch_row = [&](Rows& x, int64_t row) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            x.o[c].load(a.out.data, row * a.out.stride + at(c), cols - at(c));
            if (by_y) x.dy[c].load(a.dy.data, row * a.dy.stride + at(c), cols - at(c));
            if (a.dout.data != nullptr) x.up[c].load(a.dout.data, row * a.dout.stride + at(c), cols - at(c));
            if (has_z) x.z[c].load(a.z.data, row * a.z.stride + at(c), cols - at(c));
            if (gated) x.g[c].load(a.gate.data, row * a.gate.stride + at(c), cols - at(c));
        }
    };
    // one run a lane: the weights stay in registers, and the next row is on its way
    constexpr bool kAhead = C == 1 && (BF16 || W < 16);
    float wk[8], wzk[8];
    if constexpr (kAhead) {
        if (a.weight != nullptr) load8<false>(wk, a.weight, at(0), cols - at(0));
        if (post) load8<false>(wzk, a.z_weight, at(0), cols - at(0));
    }
    auto weights = [&](float (&w)[8], const float (&kept)[8], const float* from, int c) {
        if constexpr (kAhead) {
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = kept[e];
        } else {
            load8<false>(w, from, at(c), cols - at(c));
        }
    };
    Rows next;
    int64_t row = (int64_t)blockIdx.x * kTeams + wave;
    if (kAhead && row < a.out.rows) fetch_row(next, row);
    for (; row < a.out.rows; row += teams) {
        Rows x;
        if constexpr (kAhead) {
            x = next;
            if (row + teams < a.out.rows) fetch_row(next, row + teams);
        } else {
            fetch_row(x, row);
        }
        auto& o = x.o;
        auto& dy = x.dy;
        auto& z = x.z;
        auto& g = x.g;
        auto& up = x.up;
        float r = 0.f, mean = 0.f;
        if (by_y) {
            float ss = 0.f, st = 0.f;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float w[8];
                if (a.weight != nullptr) weights(w, wk, a.weight, c);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    ss += o[c][e] * o[c][e];
                    st += (a.weight != nullptr ? dy[c][e] * w[e] : dy[c][e]) * o[c][e];
                }
            }
            team_sum<W>(ss, st, lds, turn);
            r = inverse_rms(ss, cols, a.eps);
            mean = r * st * inv;
        }
        float d[C][8];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            float w[8];
            if (by_y && a.weight != nullptr) weights(w, wk, a.weight, c);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                d[c][e] = a.dout.data != nullptr ? up[c][e] : 0.f;
                if (by_y) {
                    const float n = o[c][e] * r, t = a.weight != nullptr ? dy[c][e] * w[e] : dy[c][e];
                    dw[c][e] += dy[c][e] * n;
                    d[c][e] += r * (t - n * mean);
                }
            }
            if (a.dx.data != nullptr) store8<BF16>(a.dx.data, row * a.dx.stride + at(c), d[c], cols - at(c));
        }
        if (!has_z) continue;
        float rz = 1.f, mz = 0.f;
        if (post) {
            float zz = 0.f, sz = 0.f;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float wz[8];
                weights(wz, wzk, a.z_weight, c);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    zz += z[c][e] * z[c][e];
                    sz += d[c][e] * (gated ? a.scale * g[c][e] : a.scale) * wz[e] * z[c][e];
                }
            }
            team_sum<W>(zz, sz, lds, turn);
            rz = inverse_rms(zz, cols, a.eps);
            mz = rz * sz * inv;
        }
#pragma unroll
        for (int c = 0; c < C; ++c) {
            float wz[8], dz[8], dgate[8];
            if (post) weights(wz, wzk, a.z_weight, c);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float n = z[c][e] * rz, b = post ? n * wz[e] : n;
                const float db = d[c][e] * (gated ? a.scale * g[c][e] : a.scale);
                dz[e] = post ? rz * (db * wz[e] - n * mz) : db;
                dgate[e] = a.scale * d[c][e] * b;
                dwz[c][e] += db * n;
                dg[c][e] += dgate[e];
            }
            if (a.dz.data != nullptr) store8<BF16>(a.dz.data, row * a.dz.stride + at(c), dz, cols - at(c));
            if (a.dgate.data != nullptr && !a.channel) store8<BF16>(a.dgate.data, row * a.dgate.stride + at(c), dgate, cols - at(c));
        }
    }
    if (a.work == nullptr) return;
    // the workgroup's part of each sum, its teams in order
    __shared__ __align__(16) float join[W == 1 ? 4 * C * 512 : 1];
    static_assert(__alignof__(join) >= 16, "stored four at a time");
    auto put = [&](const float (&v)[C][8], int which) {
        float* to = a.work + ((int64_t)which * gridDim.x + blockIdx.x) * cols;
        if constexpr (W == 1) {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int e = 0; e < 8; e += 4)
                    *reinterpret_cast<f32x4*>(&join[wave * C * 512 + at(c) + e]) = f32x4{v[c][e], v[c][e + 1], v[c][e + 2], v[c][e + 3]};
            __syncthreads();
            for (int i = threadIdx.x; i < C * 512 && i < cols; i += 256)
                to[i] = ((join[i] + join[C * 512 + i]) + join[2 * C * 512 + i]) + join[3 * C * 512 + i];
            __syncthreads();
        } else {
#pragma unroll
            for (int c = 0; c < C; ++c) store8<false>(to, at(c), v[c], cols - at(c));
        }
    };
    if (a.dweight != nullptr) put(dw, 0);
    if (a.dz_weight != nullptr) put(dwz, 1);
    if (a.channel && a.dgate.data != nullptr) put(dg, 2);
}

// The workgroups' parts of a column, in order: 64 columns of one sum a workgroup, 16 parts at a
// time, sixteen loads on their way.
template <bool BF16>
__global__ void __launch_bounds__(1024) residual_join_kernel(ResidualGrad a, int parts) {
    __shared__ double part[16][64];
    const int c = threadIdx.x & 63, p = threadIdx.x >> 6, which = blockIdx.y;
    if (which == 0 ? a.dweight == nullptr : which == 1 ? a.dz_weight == nullptr : !(a.channel && a.dgate.data != nullptr)) return;
    const int64_t cols = a.out.cols, col = (int64_t)blockIdx.x * 64 + c;
    double s = 0.0;
    if (col < cols) {
        const float* from = a.work + (int64_t)which * parts * cols + col;
        for (int t = p; t < parts; t += 256) {
            float v[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = t + 16 * i < parts ? from[(int64_t)(t + 16 * i) * cols] : 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) s += (double)v[i];
        }
    }
    part[p][c] = s;
    __syncthreads();
    if (p != 0 || col >= cols) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) s += part[i][c];
    if (which == 0)
        a.dweight[col] = (float)s;
    else if (which == 1)
        a.dz_weight[col] = (float)s;
    else
        store_one<BF16>(a.dgate.data, col, (float)s);
}

hipError_t launch_residual_norm(bool bf16, const Residual& a, hipStream_t s);
hipError_t launch_residual_grad(bool bf16, const ResidualGrad& a, hipStream_t s);

}  // namespace autoloco
