// Host helper: kernel launch with programmatic dependent launch allowed (the
// kernel may be scheduled while its predecessor on the stream finishes, and
// waits for it in griddepcontrol.wait before it touches global memory).
#pragma once

#include <cuda_runtime.h>

#include <atomic>
#include <utility>

namespace pp {

template <typename... KArgs, typename... Args>
cudaError_t launch_overlapped(void (*kern)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st,
                              Args&&... args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kern, std::forward<Args>(args)...);
}

// Dynamic shared memory above 48 KB for a kernel, set once a device (`done`:
// one flag a device, the caller's own for each kernel).
template <typename Kern>
cudaError_t allow_smem(Kern* kern, int bytes, std::atomic<bool> (&done)[64]) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const bool keep = dev >= 0 && dev < 64;
    if (keep && done[dev].load(std::memory_order_relaxed)) return cudaSuccess;
    e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess && keep) done[dev].store(true, std::memory_order_relaxed);
    return e;
}

}  // namespace pp
