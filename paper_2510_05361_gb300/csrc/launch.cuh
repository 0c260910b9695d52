// launch.cuh -- launching a kernel with more shared memory than needs no asking, and one that may
// start before the kernel ahead of it has ended.
#pragma once

#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>

namespace mtdao {

// Allows the kernel so much dynamic shared memory on the current device; asked once a device (done: a bit for each).
inline cudaError_t allow_shared(const void *kernel, int bytes, std::atomic<uint64_t> &done) {
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    const uint64_t bit = device < 64 ? uint64_t(1) << device : 0;
    if (done.load(std::memory_order_relaxed) & bit) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

// A launch that need not wait for the kernel before it in the stream: the kernel waits itself
// (cudaGridDependencySynchronize) before it reads what that one wrote.
template <typename... Params, typename... Args>
cudaError_t launch_early(void (*kernel)(Params...), dim3 grid, unsigned threads, size_t bytes, cudaStream_t stream,
                         Args... args) {
    cudaLaunchConfig_t config = {};
    config.gridDim = grid;
    config.blockDim = dim3(threads);
    config.dynamicSmemBytes = bytes;
    config.stream = stream;
    cudaLaunchAttribute early;
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    config.attrs = &early;
    config.numAttrs = 1;
    return cudaLaunchKernelEx(&config, kernel, args...);
}

}  // namespace mtdao
