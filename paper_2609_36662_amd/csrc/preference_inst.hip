// Launchers of the preference loss's kernels.
#include <type_traits>

#include "preference_kernels.hpp"

namespace autoloco {

namespace {

// Threads of a row's workgroup.  With no more rows than the compute units hold
// workgroups of 1,024, a long row's time is what counts (27 rows of 32,000 bf16: the row
// kernels 8.0 and 8.4 us at 256 threads, 6.2 and 5.2 at 1,024).  Else 256 for the log sum
// exp and 512 for the gradient (19,456 rows of 32,000 bf16: a call 511 us with 256 in
// both, 502 so); 256 up to rows of 16 KB; a wave up to 4 KB, where a thread of more has
// no whole vector.
int threads_of(bool few_rows, int64_t row_bytes, int most) {
    if (row_bytes <= 4096) return 64;
    if (row_bytes <= 16384) return 256;
    return few_rows ? 1024 : most;
}
constexpr int64_t kFewRows = 512;

// f(integral_constant) of the threads.
template <typename F>
void with_threads(int threads, F f) {
    switch (threads) {
        case 64: return f(std::integral_constant<int, 64>{});
        case 256: return f(std::integral_constant<int, 256>{});
        case 512: return f(std::integral_constant<int, 512>{});
        default: return f(std::integral_constant<int, 1024>{});
    }
}

// launch(first, count) over all rows (and pairs), at most 2^20 at a time.
template <typename Launch>
hipError_t in_slices(int64_t rows, Launch launch) {
    constexpr int64_t kSlice = int64_t(1) << 20;
    for (int64_t first = 0; first < rows; first += kSlice) {
        launch(first, dim3((unsigned)(rows - first < kSlice ? rows - first : kSlice)));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <bool BF16>
hipError_t row_logp(const SequenceArgs& a, hipStream_t s) {
    const int threads = threads_of(a.logits.rows <= kFewRows, a.logits.cols * (BF16 ? 2 : 4), 256);
    return in_slices(a.logits.rows, [&](int64_t first, dim3 grid) {
        with_threads(threads, [&](auto nt) {
            constexpr int NT = decltype(nt)::value;
            if constexpr (NT != 512) hipLaunchKernelGGL((row_logp_kernel<BF16, NT>), grid, dim3(NT), 0, s, a, first);
        });
    });
}

template <bool BF16>
hipError_t logit_grad(bool pairs, const SequenceArgs& a, const PreferenceArgs& p, const MatrixOut& g, hipStream_t s) {
    // few rows have their pairs in the same kernel, but where there are no pairs: then all is zero
    const int threads = threads_of(pairs && a.logits.rows <= kFewRows, a.logits.cols * (BF16 ? 2 : 4), 512);
    return in_slices(a.logits.rows + (pairs ? a.sequences / 2 : 0), [&](int64_t first, dim3 grid) {
        with_threads(threads, [&](auto nt) {
            constexpr int NT = decltype(nt)::value;
            if (pairs)
                hipLaunchKernelGGL((logit_grad_kernel<BF16, NT, true>), grid, dim3(NT), 0, s, a, p, g, first);
            else if constexpr (NT != 1024)
                hipLaunchKernelGGL((logit_grad_kernel<BF16, NT, false>), grid, dim3(NT), 0, s, a, p, g, first);
        });
    });
}

}  // namespace

hipError_t launch_row_logp(bool bf16, const SequenceArgs& a, hipStream_t s) {
    return bf16 ? row_logp<true>(a, s) : row_logp<false>(a, s);
}

hipError_t launch_pairs(const SequenceArgs& a, const PreferenceArgs& p, hipStream_t s) {
    const dim3 grid((unsigned)(p.losses != nullptr ? a.sequences / 2 : a.sequences));
    hipLaunchKernelGGL(pair_kernel<256>, grid, dim3(256), 0, s, a, p);
    return hipGetLastError();
}

hipError_t launch_logit_grad(bool bf16, bool pairs, const SequenceArgs& a, const PreferenceArgs& p, const MatrixOut& g,
                             hipStream_t s) {
    return bf16 ? logit_grad<true>(pairs, a, p, g, s) : logit_grad<false>(pairs, a, p, g, s);
}

}  // namespace autoloco
