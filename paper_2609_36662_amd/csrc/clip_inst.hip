// Launchers of the clipping kernels.
#include "clip_kernels.hpp"

namespace autoloco {

hipError_t launch_tensor_norm(int workers, int blocks, const ClipArgs& a, hipStream_t s) {
    hipLaunchKernelGGL(tensor_norm_kernel, dim3(blocks, workers), dim3(kBlock), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_tensor_clip(int workers, int blocks, const ClipArgs& a, hipStream_t s) {
    hipLaunchKernelGGL(tensor_clip_kernel, dim3(blocks, workers), dim3(kBlock), 0, s, a);
    return hipGetLastError();
}

}  // namespace autoloco
