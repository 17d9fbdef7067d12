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
// Each row's lse from one reading (a running maximum and sum), each pair's loss and
// weights in fp64, each row's gradient; the middle one inside the last where that costs
// no more than a kernel of its own.  The rows' kernels are bound by HBM; exponentials are taken in base
// 2.  A row whose label is masked, or that is of no sequence, is not read.  (16 pairs of
// up to 1,024 tokens, vocabulary 32,000, bf16, 40 % of them prompt: 0.49 ms, 2.98 GB at
// 6.0 TB/s.  Of these 0.87 GB are the second reading of the logits, which the weights
// stand between; pairs that the Infinity Cache holds go only 10 % faster.)
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

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
    if (a.sequences == 0) return -1;
    // all three on their way together
    const int64_t l = a.labels[row], lo = offset_at(a, 0), hi = offset_at(a, a.sequences);
    return l >= 0 && l < a.logits.cols && row >= lo && row < hi ? l : -1;
}

// A row seen as a head of single elements up to a 16-byte boundary, vectors of 16 bytes
// (8 bf16 or 4 fp32) and a tail of single elements.  Rows of an odd vocabulary begin
// anywhere; reading or writing across 16-byte boundaries costs twice.
template <bool BF16>
struct RowSplit {
    static constexpr int V = BF16 ? 8 : 4;
    int64_t head, vectors, n;
    __device__ __forceinline__ RowSplit(const void* p, int64_t count) : n(count) {
        const int64_t off = (int64_t)(reinterpret_cast<uintptr_t>(p) & 15) / (16 / V);
        head = off == 0 ? 0 : V - off;
        if (head > n) head = n;
        vectors = (n - head) / V;
    }
    // Single element j (of the head, then of the tail), or -1 beyond.
    __device__ __forceinline__ int64_t single(int64_t j) const {
        const int64_t i = j < head ? j : j + vectors * V;
        return i < n ? i : -1;
    }
};

template <bool BF16>
__device__ __forceinline__ void unpack(float (&x)[BF16 ? 8 : 4], u32x4 w) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (BF16) {
            x[2 * j] = bf16_lo(w[j]);
            x[2 * j + 1] = bf16_hi(w[j]);
        } else {
            x[j] = __uint_as_float(w[j]);
        }
    }
}

// The larger of three: one instruction, where fmaxf would first quiet each operand.  (A
// NaN may be lost here: it comes back with the sum of the exponentials.)
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

constexpr float kLowest = -3.402823466e38f;
// Up to this power of two an exponent x log2 e - m is as exact as its own size: m, itself a
// rounded product, is taken as it is, so that nothing cancels but what the fused
// multiply-add keeps.  A row whose maximum lies beyond is done again with differences first.
constexpr float kHuge = 0x1p24f;

// A running maximum and a sum of exponentials.  PLAIN: the maximum m is that of x log2 e,
// rounded, the sum that of 2^(x log2 e - m), one multiply-add an exponent.  Else m is that
// of x, the sum that of 2^((x - m) log2 e).
template <bool PLAIN>
struct RunningSum {
    float m = PLAIN ? -kHuge : kLowest, s = 0.f;   // values below the first m add nothing
    static __device__ __forceinline__ float power(float x, float m) {
        if constexpr (PLAIN)
            return __builtin_amdgcn_exp2f(__builtin_fmaf(x, kLog2e, -m));
        else
            return __builtin_amdgcn_exp2f((x - m) * kLog2e);
    }
    // What a sum for maximum m is worth for maximum to.
    static __device__ __forceinline__ float from(float m, float to) {
        return __builtin_amdgcn_exp2f(PLAIN ? m - to : (m - to) * kLog2e);
    }
    template <int N>
    __device__ __forceinline__ void add(const float (&x)[N]) {
        float top = x[0];
#pragma unroll
        for (int i = 1; i + 1 < N; i += 2) top = max3(top, x[i], x[i + 1]);
        if constexpr (N % 2 == 0) top = max3(top, x[N - 1], x[N - 1]);
        if constexpr (PLAIN) top *= kLog2e;
        top = max3(m, top, top);
        s *= from(m, top);
        m = top;
        float part[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < N; ++i) part[i & 1] += power(x[i], m);
        s += part[0] + part[1];
    }
    __device__ __forceinline__ void join(float om, float os) {
        const float to = max3(m, om, om);
        s = s * from(m, to) + os * from(om, to);
        m = to;
    }
};

// The running sum of a whole row over a workgroup of NT threads, in thread 0; m is the
// row's maximum in every thread.
template <bool BF16, int NT, bool PLAIN>
__device__ __forceinline__ RunningSum<PLAIN> row_sum(const char* x, int64_t vocab, float (&lds)[2 * (NT / 64)]) {
    constexpr int U = 4;   // vectors in flight
    constexpr int V = BF16 ? 8 : 4;
    const RowSplit<BF16> row(x, vocab);
    const u32x4* body = reinterpret_cast<const u32x4*>(x + row.head * (16 / V));
    RunningSum<PLAIN> r;
    // the last vectors of the row together too: one after another, each would wait for its
    // own way to memory
    constexpr uint32_t kNothing = BF16 ? 0xFF80FF80u : 0xFF800000u;   // -inf
    auto batch = [&](int64_t i, auto whole) {
        u32x4 w[U];
        float v[U * V];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            w[u] = u32x4{kNothing, kNothing, kNothing, kNothing};
            if (decltype(whole)::value || i + u * NT < row.vectors) w[u] = body[i + u * NT];
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int u = 0; u < U; ++u) unpack<BF16>(reinterpret_cast<float(&)[V]>(v[u * V]), w[u]);
        r.add(v);
    };
    int64_t i = threadIdx.x;
    for (; i + (U - 1) * NT < row.vectors; i += U * NT) batch(i, std::true_type{});
    if (i < row.vectors) batch(i, std::false_type{});
    if (threadIdx.x < 2 * V) {   // head and tail together: fewer than 2 V elements
        const int64_t j = row.single(threadIdx.x);
        if (j >= 0) {
            const float v[1] = {load_one<BF16>(x, j)};
            r.add(v);
        }
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) r.join(__shfl_xor(r.m, d), __shfl_xor(r.s, d));
    if ((threadIdx.x & 63) == 0) {
        lds[threadIdx.x >> 6] = r.m;
        lds[NT / 64 + (threadIdx.x >> 6)] = r.s;
    }
    __syncthreads();
    r.m = lds[0];
    r.s = lds[NT / 64];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) r.join(lds[w], lds[NT / 64 + w]);
    return r;
}

// Each row's log sum exp and its label's log-probability; a workgroup a row (first: the
// launch's first row, since a grid has fewer than 2^32 threads).  Bound by
// HBM with fp32 logits; with bf16 ones the exponentials (a quarter of the rate of other
// instructions) take as long as the reading.
template <bool BF16, int NT>
__global__ void __launch_bounds__(NT) row_logp_kernel(SequenceArgs a, int64_t first) {
    __shared__ float lds[2 * (NT / 64)];
    const int64_t row = first + blockIdx.x;
    const int64_t label = live_label(a, row);
    if (label < 0) {
        if (threadIdx.x == 0) {
            a.lse[row] = 0.f;
            a.logp[row] = 0.f;
        }
        return;
    }
    const char* x = static_cast<const char*>(a.logits.data) + row * a.logits.stride * (BF16 ? 2 : 4);
    const RunningSum<true> r = row_sum<BF16, NT, true>(x, a.logits.cols, lds);
    if (fabsf(r.m) < kHuge) {   // every thread has the same maximum
        if (threadIdx.x == 0) {
            const float at = load_one<BF16>(x, label);
            const double sum = log2((double)r.s);
            a.lse[row] = (float)((r.m + sum) / kLog2e);
            // a large probability with the same rounding as in the sum, so that it is at most 1
            const float power = __builtin_fmaf(at, kLog2e, -r.m);
            const double part = power > -1.f ? log2((double)__builtin_amdgcn_exp2f(power)) : (double)at * kLog2e - r.m;
            a.logp[row] = (float)((part - sum) / kLog2e);
        }
        return;
    }
    __syncthreads();
    const RunningSum<false> d = row_sum<BF16, NT, false>(x, a.logits.cols, lds);
    if (threadIdx.x == 0) {
        const double m = d.m, ln = log((double)d.s);   // apart from m, which may be far larger
        a.lse[row] = (float)(m + ln);
        a.logp[row] = (float)(((double)load_one<BF16>(x, label) - m) - ln);
    }
}

// Sum of the log-probabilities of rows lo..hi, in every thread of a workgroup.
template <int NT>
__device__ __forceinline__ double sum_rows(const float* logp, int64_t lo, int64_t hi, double* lds) {
    double t = 0.0;
    for (int64_t i = lo + threadIdx.x; i < hi; i += NT) t += (double)logp[i];
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) t += __shfl_xor(t, d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = t;
    __syncthreads();
    t = lds[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) t += lds[w];
    return t;
}

// log sigma(z), in fp64 (a NaN comes through the exponential).
__device__ __forceinline__ double log_sigmoid(double z) { return (z < 0.0 ? z : 0.0) - log1p(exp(-fabs(z))); }

// The weight of pair i's chosen sequence in the gradient; z and both log-probabilities.
template <int NT>
__device__ __forceinline__ double pair_weight(const SequenceArgs& a, const PreferenceArgs& p, int64_t i, double* lds,
                                              double& first, double& second, double& z) {
    const int64_t j = i + a.sequences / 2;
    first = sum_rows<NT>(a.logp, offset_at(a, i), offset_at(a, i + 1), lds);
    second = sum_rows<NT>(a.logp, offset_at(a, j), offset_at(a, j + 1), lds);
    z = p.beta * ((first - (double)p.ref[i]) - (second - (double)p.ref[j]));
    // sigma(z) - (1 - eps) = eps sigma(z) - (1 - eps) sigma(-z): where the pair is decided,
    // the difference on the left keeps nothing of a weight of exp(-z)
    const double e = exp(-fabs(z)), larger = 1.0 / (1.0 + e), smaller = e * larger;
    const double up = z < 0.0 ? smaller : larger, down = z < 0.0 ? larger : smaller;
    return p.scale * p.beta * (p.smoothing * up - (1.0 - p.smoothing) * down);
}

// What a workgroup of NT threads writes for pair i (or, without losses, sequence i).
template <int NT>
__device__ __forceinline__ void pair_outputs(const SequenceArgs& a, const PreferenceArgs& p, int64_t i, double* lds) {
    if (p.losses == nullptr) {
        const double sum = sum_rows<NT>(a.logp, offset_at(a, i), offset_at(a, i + 1), lds);
        if (threadIdx.x == 0) {
            p.logps[i] = (float)sum;
            a.weight[i] = 0.f;
        }
        return;
    }
    const int64_t j = i + a.sequences / 2;
    double first, second, z;
    const double w = pair_weight<NT>(a, p, i, lds, first, second, z);
    if (threadIdx.x == 0) {
        p.logps[i] = (float)first;
        p.logps[j] = (float)second;
        // a term of weight 0 is left out: 0 times an infinite one is no NaN
        double loss = z != z ? z : 0.0;
        if (p.smoothing < 1.0) loss -= (1.0 - p.smoothing) * log_sigmoid(z);
        if (p.smoothing > 0.0) loss -= p.smoothing * log_sigmoid(-z);
        p.losses[i] = (float)loss;
        a.weight[i] = (float)w;
        a.weight[j] = (float)-w;
    }
}

template <int NT>
__global__ void __launch_bounds__(NT) pair_kernel(SequenceArgs a, PreferenceArgs p) {
    __shared__ double lds[NT / 64];
    pair_outputs<NT>(a, p, blockIdx.x, lds);
}

// The sequence that row belongs to: the last one that begins at or before it.  A wave
// looks at 64 of them at a time.
__device__ __forceinline__ int64_t sequence_of(const SequenceArgs& a, int64_t row) {
    int64_t lo = 0, n = a.sequences;
    while (n > 1) {
        const int64_t step = (n + 63) / 64, at = lo + (threadIdx.x & 63) * step;
        const int begun = __popcll(__ballot(at < lo + n && offset_at(a, at < lo + n ? at : lo) <= row));
        const int64_t end = lo + n;
        if (begun > 1) lo += (begun - 1) * step;
        n = end - lo < step ? end - lo : step;
    }
    return lo;
}

// One row of the gradient: -wp times the power of RunningSum (PLAIN: with what rounding
// took from m given back, so that a probability of 1 is 1), and w more at the label.  Neither the logits
// nor the gradient are kept in the caches: both pass once (18,500 rows of 32,000 bf16:
// 511 us for the whole call against 541 with cached loads and 558 with cached stores
// too; 3,900 rows of fp32 199, 236 and 256).
template <bool BF16, int NT, bool PLAIN>
__device__ __forceinline__ void row_gradient(const char* x, char* out, int64_t vocab, int64_t label, float w, float wp,
                                             float m, float rest) {
    constexpr int U = NT == 1024 ? 4 : 2;   // vectors in flight
    constexpr int V = BF16 ? 8 : 4;
    const RowSplit<BF16> row(out, vocab);
    const u32x4_any* in = reinterpret_cast<const u32x4_any*>(x + row.head * (16 / V));
    u32x4* body = reinterpret_cast<u32x4*>(out + row.head * (16 / V));
    const int64_t at = label - row.head;
    auto power = [&](float e) {
        return PLAIN ? __builtin_amdgcn_exp2f(__builtin_fmaf(e, kLog2e, -m) + rest) : RunningSum<false>::power(e, m);
    };
    auto one = [&](u32x4 raw, int64_t i) {
        float v[V];
        unpack<BF16>(v, raw);
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = -wp * power(v[j]);
        if ((uint64_t)(at - i * V) < (uint64_t)V) {
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (at - i * V == j) v[j] += w;
        }
        u32x4 to;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (BF16)
                to[j] = bf16_pack(v[2 * j], v[2 * j + 1]);
            else
                to[j] = __float_as_uint(v[j]);
        }
        st_u4(&body[i], to);
    };
    auto batch = [&](int64_t i, auto whole) {
        u32x4 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            raw[u] = u32x4{0, 0, 0, 0};
            if (decltype(whole)::value || i + u * NT < row.vectors) raw[u] = __builtin_nontemporal_load(&in[i + u * NT]);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (decltype(whole)::value || i + u * NT < row.vectors) one(raw[u], i + u * NT);
    };
    int64_t i = threadIdx.x;
    for (; i + (U - 1) * NT < row.vectors; i += U * NT) batch(i, std::true_type{});
    if (i < row.vectors) batch(i, std::false_type{});
    if (threadIdx.x < 2 * V) {
        const int64_t j = row.single(threadIdx.x);
        if (j >= 0) {
            float v = -wp * power(load_one<BF16>(x, j));
            if (j == label) v += w;
            store_one<BF16>(out, j, v);
        }
    }
}

// Each row's gradient; a workgroup a row.  Bound by HBM: a reading and a writing of the
// logits.  PAIRS: there was no pair kernel; each workgroup finds its pair's weight
// itself, and one more workgroup a pair, at the end, writes its outputs.
template <bool BF16, int NT, bool PAIRS>
__global__ void __launch_bounds__(NT) logit_grad_kernel(SequenceArgs a, PreferenceArgs p, MatrixOut g, int64_t first) {
    __shared__ double lds[NT / 64];
    const int64_t row = first + blockIdx.x;
    if constexpr (PAIRS) {
        if (row >= a.logits.rows) {
            pair_outputs<NT>(a, p, row - a.logits.rows, lds);
            return;
        }
    }
    const int64_t label = live_label(a, row);
    const int64_t vocab = a.logits.cols;
    char* out = static_cast<char*>(g.data) + row * g.stride * (BF16 ? 2 : 4);
    if (label < 0) {
        const RowSplit<BF16> split(out, vocab);
        constexpr int V = BF16 ? 8 : 4;
        u32x4* body = reinterpret_cast<u32x4*>(out + split.head * (16 / V));
        for (int64_t i = threadIdx.x; i < split.vectors; i += NT) st_u4(&body[i], u32x4{0, 0, 0, 0});
        if (threadIdx.x < 2 * V) {
            const int64_t j = split.single(threadIdx.x);
            if (j >= 0) store_one<BF16>(out, j, 0.f);
        }
        return;
    }
    const char* x = static_cast<const char*>(a.logits.data) + row * a.logits.stride * (BF16 ? 2 : 4);
    // The row's log sum exp: as stored, or the label's logit less its log-probability,
    // whichever is the smaller number and so the more exact.  Taken before the barrier: the
    // gradient may go where the logits are.
    // Where both numbers are beyond 64, or the exponent is beyond 2^24, the sum is done again.
    __shared__ float norm[2];
    if (threadIdx.x == 0) {
        const float lse = a.lse[row], logp = a.logp[row];
        const double exponent = (fabsf(logp) < fabsf(lse) ? (double)load_one<BF16>(x, label) - logp : (double)lse) * kLog2e;
        const bool exact = fminf(fabsf(lse), fabsf(logp)) < 64.f && fabs(exponent) < kHuge;
        norm[0] = exact ? (float)exponent : kHuge;
        norm[1] = (float)(norm[0] - exponent);
    }
    const int64_t s = sequence_of(a, row), half = a.sequences / 2;
    float w;
    if constexpr (PAIRS) {
        double first, second, z;
        const double chosen = pair_weight<NT>(a, p, s < half ? s : s - half, lds, first, second, z);
        w = (float)(s < half ? chosen : -chosen);
    } else {
        w = a.weight[s];
        __syncthreads();
    }
    if (norm[0] < kHuge) {
        row_gradient<BF16, NT, true>(x, out, vocab, label, w, w, norm[0], norm[1]);
    } else {   // the maximum and the sum apart (and a NaN)
        __shared__ float sums[2 * (NT / 64)];
        const RunningSum<false> r = row_sum<BF16, NT, false>(x, vocab, sums);
        row_gradient<BF16, NT, false>(x, out, vocab, label, w, w / r.s, r.m, 0.f);
    }
}

hipError_t launch_row_logp(bool bf16, const SequenceArgs& a, hipStream_t s);
hipError_t launch_pairs(const SequenceArgs& a, const PreferenceArgs& p, hipStream_t s);
// pairs: the gradient's kernel does what launch_pairs does as well.
hipError_t launch_logit_grad(bool bf16, bool pairs, const SequenceArgs& a, const PreferenceArgs& p, const MatrixOut& g,
                             hipStream_t s);

}  // namespace autoloco
