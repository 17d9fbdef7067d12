// Launchers of the preference loss's kernels.
#include "preference_kernels.hpp"

namespace autoloco {

hipError_t launch_row_logp(bool bf16, const SequenceArgs& a, hipStream_t s) {
    const dim3 grid((unsigned)a.logits.rows);
    if (bf16)
        hipLaunchKernelGGL(row_logp_kernel<true>, grid, dim3(kBlock), 0, s, a);
    else
        hipLaunchKernelGGL(row_logp_kernel<false>, grid, dim3(kBlock), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_pairs(const SequenceArgs& a, const PreferenceArgs& p, hipStream_t s) {
    const dim3 grid((unsigned)(p.losses != nullptr ? a.sequences / 2 : a.sequences));
    hipLaunchKernelGGL(pair_kernel, grid, dim3(kBlock), 0, s, a, p);
    return hipGetLastError();
}

hipError_t launch_logit_grad(bool bf16, const SequenceArgs& a, const MatrixOut& g, hipStream_t s) {
    const dim3 grid((unsigned)a.logits.rows);
    if (bf16)
        hipLaunchKernelGGL(logit_grad_kernel<true>, grid, dim3(kBlock), 0, s, a, g);
    else
        hipLaunchKernelGGL(logit_grad_kernel<false>, grid, dim3(kBlock), 0, s, a, g);
    return hipGetLastError();
}

}  // namespace autoloco
