// Log-probabilities of token sequences and the preference loss over pairs of them,
// with the gradient by the logits, on gfx950.
//
//   lse_r   = log sum_v exp x[r][v],   logp_r = x[r][label_r] - lse_r
//   logp_s  = sum of logp_r over the rows of sequence s
//   z_p     = beta ((logp_p - ref_p) - (logp_{P+p} - ref_{P+p}))
//   loss_p  = -(1 - eps) log sigma(z_p) - eps log sigma(-z_p)
//   dx[r][v] = w_s ([v = label_r] - exp(x[r][v] - lse_r)),
//   w_p = scale beta (sigma(z_p) - (1 - eps)),  w_{P+p} = -w_p
//
// Three kernels: each row's lse from one reading (a running maximum and sum), each
// pair's loss and weights in fp64, each row's gradient.  The first and the last are
// bound by HBM; exponentials are taken in base 2.  A row whose label is masked, or
// that is of no sequence, is not read.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "matrix_view.hpp"

namespace autoloco {

struct SequenceArgs {
    MatrixView logits;
    const int64_t* labels;
    const int64_t* offsets;
    int64_t sequences;
    float* lse;       // [rows]
    float* logp;      // [rows]
    float* weight;    // [sequences]
};

struct PreferenceArgs {
    const float* ref;
    float* losses;     // null: only the sequences' log-probabilities
    float* logps;
    double beta, smoothing, scale;
};

constexpr float kLog2e = 1.4426950408889634f;
constexpr double kLn2 = 0.6931471805599453;

// Offset i, inside 0..rows.
__device__ __forceinline__ int64_t offset_at(const SequenceArgs& a, int64_t i) {
    const int64_t o = a.offsets[i];
    return o < 0 ? 0 : o > a.logits.rows ? a.logits.rows : o;
}

// The label of a row, or -1 if the row is masked.
__device__ __forceinline__ int64_t live_label(const SequenceArgs& a, int64_t row) {
    const int64_t l = a.labels[row];
    if (l < 0 || l >= a.logits.cols || a.sequences == 0) return -1;
    return row >= offset_at(a, 0) && row < offset_at(a, a.sequences) ? l : -1;
}

// A running maximum (base 2, times log2 e) and the sum of 2^(x - max).
struct RunningSum {
    float m = -__builtin_inff(), s = 0.f;
    __device__ __forceinline__ void rescale(float to) {
        if (to > m) {
            s *= __builtin_amdgcn_exp2f(m - to);
            m = to;
        }
    }
    __device__ __forceinline__ void add8(const float (&x)[8]) {
        float top = x[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) top = fmaxf(top, x[i]);
        rescale(top * kLog2e);
        const float base = m == -__builtin_inff() ? 0.f : m;   // nothing but -inf so far
#pragma unroll
        for (int i = 0; i < 8; ++i) s += __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], kLog2e, -base));
    }
    __device__ __forceinline__ void join(float om, float os) {
        const float to = fmaxf(m, om);
        if (to == -__builtin_inff()) {   // both empty, or NaN sums to keep
            s += os;
            return;
        }
        s = s * __builtin_amdgcn_exp2f(m - to) + os * __builtin_amdgcn_exp2f(om - to);
        m = to;
    }
};

// Each row's log sum exp and its label's log-probability; a workgroup a row.
template <bool BF16>
__global__ void __launch_bounds__(kBlock) row_logp_kernel(SequenceArgs a) {
    __shared__ float lm[4], ls[4];
    const int64_t row = blockIdx.x;
    const int64_t label = live_label(a, row);
    if (label < 0) {
        if (threadIdx.x == 0) {
            a.lse[row] = 0.f;
            a.logp[row] = 0.f;
        }
        return;
    }
    const int64_t vocab = a.logits.cols;
    const char* x = static_cast<const char*>(a.logits.data) + row * a.logits.stride * (BF16 ? 2 : 4);
    RunningSum r;
    for (int64_t i = threadIdx.x * 8; i < vocab; i += kBlock * 8) {
        float v[8];
        load8<BF16>(v, x, i, vocab, -__builtin_inff());
        r.add8(v);
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) r.join(__shfl_xor(r.m, d), __shfl_xor(r.s, d));
    if ((threadIdx.x & 63) == 0) {
        lm[threadIdx.x >> 6] = r.m;
        ls[threadIdx.x >> 6] = r.s;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 4; ++w) r.join(lm[w], ls[w]);
        const double lse = (double)r.m * kLn2 + log((double)r.s);
        a.lse[row] = (float)lse;
        a.logp[row] = (float)((double)load_one<BF16>(x, label) - lse);
    }
}

// Sum of the log-probabilities of rows lo..hi, in every thread of a workgroup.
__device__ __forceinline__ double sum_rows(const float* logp, int64_t lo, int64_t hi, double* lds) {
    double t = 0.0;
    for (int64_t i = lo + threadIdx.x; i < hi; i += kBlock) t += (double)logp[i];
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) t += __shfl_xor(t, d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = t;
    __syncthreads();
    return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

// log sigma(z), in fp64 (a NaN comes through the exponential).
__device__ __forceinline__ double log_sigmoid(double z) { return (z < 0.0 ? z : 0.0) - log1p(exp(-fabs(z))); }

// A workgroup a pair (or, without losses, a sequence).
[[maybe_unused]] static __global__ void __launch_bounds__(kBlock) pair_kernel(SequenceArgs a, PreferenceArgs p) {
    __shared__ double lds[4];
    const int64_t i = blockIdx.x;
    const double first = sum_rows(a.logp, offset_at(a, i), offset_at(a, i + 1), lds);
    if (p.losses == nullptr) {
        if (threadIdx.x == 0) {
            p.logps[i] = (float)first;
            a.weight[i] = 0.f;
        }
        return;
    }
    const int64_t j = i + a.sequences / 2;
    const double second = sum_rows(a.logp, offset_at(a, j), offset_at(a, j + 1), lds);
    if (threadIdx.x == 0) {
        const double z = p.beta * ((first - (double)p.ref[i]) - (second - (double)p.ref[j]));
        p.logps[i] = (float)first;
        p.logps[j] = (float)second;
        // a term of weight 0 is left out: 0 times an infinite one is no NaN
        double loss = z != z ? z : 0.0;
        if (p.smoothing < 1.0) loss -= (1.0 - p.smoothing) * log_sigmoid(z);
        if (p.smoothing > 0.0) loss -= p.smoothing * log_sigmoid(-z);
        p.losses[i] = (float)loss;
        const double w = p.scale * p.beta * (1.0 / (1.0 + exp(-z)) - (1.0 - p.smoothing));
        a.weight[i] = (float)w;
        a.weight[j] = (float)-w;
    }
}

// The sequence that row belongs to: the last one that begins at or before it.
__device__ __forceinline__ int64_t sequence_of(const SequenceArgs& a, int64_t row) {
    int64_t lo = 0, hi = a.sequences - 1;
    while (lo < hi) {
        const int64_t mid = (lo + hi + 1) / 2;
        if (offset_at(a, mid) <= row)
            lo = mid;
        else
            hi = mid - 1;
    }
    return lo;
}

// Each row's gradient; a workgroup a row.
template <bool BF16>
__global__ void __launch_bounds__(kBlock) logit_grad_kernel(SequenceArgs a, MatrixOut g) {
    const int64_t row = blockIdx.x;
    const int64_t label = live_label(a, row);
    const int64_t vocab = a.logits.cols;
    char* out = static_cast<char*>(g.data) + row * g.stride * (BF16 ? 2 : 4);
    if (label < 0) {
        const float zero[8] = {};
        for (int64_t i = threadIdx.x * 8; i < vocab; i += kBlock * 8) store8<BF16>(out, i, vocab, zero);
        return;
    }
    const char* x = static_cast<const char*>(a.logits.data) + row * a.logits.stride * (BF16 ? 2 : 4);
    const float w = a.weight[sequence_of(a, row)];
    const float base = a.lse[row] * kLog2e;
    for (int64_t i = threadIdx.x * 8; i < vocab; i += kBlock * 8) {
        float v[8];
        load8<BF16>(v, x, i, vocab);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(v[j], kLog2e, -base));
            v[j] = w * ((i + j == label ? 1.f : 0.f) - p);
        }
        store8<BF16>(out, i, vocab, v);
    }
}

hipError_t launch_row_logp(bool bf16, const SequenceArgs& a, hipStream_t s);
hipError_t launch_pairs(const SequenceArgs& a, const PreferenceArgs& p, hipStream_t s);
hipError_t launch_logit_grad(bool bf16, const SequenceArgs& a, const MatrixOut& g, hipStream_t s);

}  // namespace autoloco
