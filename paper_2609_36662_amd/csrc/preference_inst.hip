// Launchers of the preference loss's kernels.
#include "preference_kernels.hpp"

namespace autoloco {

namespace {

// Rows up to which a workgroup has 1,024 threads: with no more rows than the compute
// units hold such workgroups, a row's time is what counts (27 rows of 32,000: the row
// kernels 8.0 and 8.4 us at 256 threads, 6.2 and 5.2 at 1,024).  Beyond, 256 for the log
// sum exp and 512 for the gradient (19,456 rows of 32,000 bf16: a call 511 us
// with 256 in both, 502 so).
constexpr int64_t kFewRows = 512;

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
    return in_slices(a.logits.rows, [&](int64_t first, dim3 grid) {
        if (a.logits.rows <= kFewRows)
            hipLaunchKernelGGL((row_logp_kernel<BF16, 1024>), grid, dim3(1024), 0, s, a, first);
        else
            hipLaunchKernelGGL((row_logp_kernel<BF16, 256>), grid, dim3(256), 0, s, a, first);
    });
}

template <bool BF16>
hipError_t logit_grad(bool pairs, const SequenceArgs& a, const PreferenceArgs& p, const MatrixOut& g, hipStream_t s) {
    const bool few = a.logits.rows <= kFewRows;
    return in_slices(a.logits.rows + (pairs ? a.sequences / 2 : 0), [&](int64_t first, dim3 grid) {
        if (few && pairs)
            hipLaunchKernelGGL((logit_grad_kernel<BF16, 1024, true>), grid, dim3(1024), 0, s, a, p, g, first);
        else if (few)
            hipLaunchKernelGGL((logit_grad_kernel<BF16, 1024, false>), grid, dim3(1024), 0, s, a, p, g, first);
        else if (pairs)
            hipLaunchKernelGGL((logit_grad_kernel<BF16, 512, true>), grid, dim3(512), 0, s, a, p, g, first);
        else
            hipLaunchKernelGGL((logit_grad_kernel<BF16, 512, false>), grid, dim3(512), 0, s, a, p, g, first);
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
