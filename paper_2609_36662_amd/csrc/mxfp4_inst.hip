// Launchers of the 4-bit kernels.
#include "mxfp4_kernels.hpp"

namespace autoloco {

namespace {

// Workgroups of kBlock threads, 16 of them a row's 128 columns.
unsigned group_blocks(const Mx4& q) { return (unsigned)((q.rows * q.groups * 16 + kBlock - 1) / kBlock); }

template <bool BF16>
hipError_t quantize(const MatrixView& x, const Mx4* q, const Mx4* qt, hipStream_t s) {
    if (qt == nullptr) {
        hipLaunchKernelGGL(mx_rows_kernel<BF16>, dim3(group_blocks(*q)), dim3(kBlock), 0, s, x, *q);
        return hipGetLastError();
    }
    // whole groups of 128 columns, so that the padding is written too
    const uint32_t tiles = (uint32_t)((x.cols + 127) / 128) * (BF16 ? 1 : 2);
    const uint32_t blocks = tiles * (uint32_t)((x.rows + 127) / 128);
    if (q != nullptr)
        hipLaunchKernelGGL((mx_cols_kernel<BF16, true>), dim3(blocks), dim3(kBlock), 0, s, x, *q, *qt, tiles);
    else
        hipLaunchKernelGGL((mx_cols_kernel<BF16, false>), dim3(blocks), dim3(kBlock), 0, s, x, *qt, *qt, tiles);
    return hipGetLastError();
}

template <bool BF16>
hipError_t matmul(const Mx4& a, const Mx4& b, const MatrixOut& out, hipStream_t s) {
    if (a.groups == 0) {
        const int64_t blocks = (out.rows * out.cols + kBlock - 1) / kBlock;
        hipLaunchKernelGGL(zero_matrix_kernel<BF16>, dim3((unsigned)blocks), dim3(kBlock), 0, s, out);
        return hipGetLastError();
    }
    const uint32_t mt = (uint32_t)((out.rows + 63) / 64), nt = (uint32_t)((out.cols + 63) / 64);
    hipLaunchKernelGGL(mx_matmul_kernel<BF16>, dim3(mt * nt), dim3(kBlock), 0, s, a, b, out, nt);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_mx_quantize(bool bf16, const MatrixView& x, const Mx4* q, const Mx4* qt, hipStream_t s) {
    return bf16 ? quantize<true>(x, q, qt, s) : quantize<false>(x, q, qt, s);
}

hipError_t launch_mx_values(bool bf16, const Mx4& q, const MatrixOut& out, hipStream_t s) {
    if (bf16)
        hipLaunchKernelGGL(mx_values_kernel<true>, dim3(group_blocks(q)), dim3(kBlock), 0, s, q, out);
    else
        hipLaunchKernelGGL(mx_values_kernel<false>, dim3(group_blocks(q)), dim3(kBlock), 0, s, q, out);
    return hipGetLastError();
}

hipError_t launch_mx_matmul(bool bf16, const Mx4& a, const Mx4& b, const MatrixOut& out, hipStream_t s) {
    return bf16 ? matmul<true>(a, b, out, s) : matmul<false>(a, b, out, s);
}

hipError_t launch_mx_tokens(bool bf16, const MatrixView& x, const Mx4& w, const MatrixOut& y, hipStream_t s) {
    const unsigned blocks = (unsigned)((w.rows + 15) / 16);
    if (bf16)
        hipLaunchKernelGGL(mx_tokens_kernel<true>, dim3(blocks), dim3(kBlock), 0, s, x, w, y);
    else
        hipLaunchKernelGGL(mx_tokens_kernel<false>, dim3(blocks), dim3(kBlock), 0, s, x, w, y);
    return hipGetLastError();
}

}  // namespace autoloco
