// What the files of the training-step operators share on the host side.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

namespace ones {

int device_sms();  // of the current device; 148 where that cannot be asked

inline bool aligned(const void* p, uintptr_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

// Lets the kernel use `bytes` of dynamic shared memory on the current device; `ready` holds the devices that know.
template <class F>
cudaError_t allow_smem(F kernel, int bytes, std::atomic<uint64_t>& ready) {
    int dev = 0;
    cudaError_t err = cudaGetDevice(&dev);
    if (err != cudaSuccess) return err;
    const uint64_t bit = 1ull << (dev & 63);
    if (dev < 64 && (ready.load(std::memory_order_relaxed) & bit)) return cudaSuccess;
    err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (err == cudaSuccess && dev < 64) ready.fetch_or(bit, std::memory_order_relaxed);
    return err;
}

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

// For tests, beside the public functions: the limit of every wait on the current device (0: the default), and a kernel of one
// of the five files (0 to 4) that waits `times` times for what never comes.
extern "C" int ones_train_wait_limit(unsigned long long ns);
extern "C" int ones_train_wait_for_nothing(int which, int times, void* cuda_stream);
// The row of a tile of queries from which on a key is seen, as the attention's kernels have it.
extern "C" int ones_attention_first_row(int behind, int group);
