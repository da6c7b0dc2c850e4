// What the files of the training-step operators share on the host side.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace ones {

inline bool aligned(const void* p, uintptr_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

cudaError_t loss_wait_expired(unsigned* out);    // reads and clears the flag of the loss kernels
cudaError_t update_wait_expired(unsigned* out);  // and of the update's

// Launches a kernel that begins with griddepcontrol.wait beside the tail of the launch before it.
template <class... P, class... A>
cudaError_t launch_after(void (*kernel)(P...), dim3 grid, dim3 block, cudaStream_t stream, A... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}

}  // namespace ones
