// Kernels that are launched while the kernel before them in the stream drains, and wait for its writes by themselves: the gap
// between two launches shrinks by a microsecond or two.
#pragma once
#include <cuda_runtime.h>

namespace gg {

// Before the first access to memory.  The one after may be launched from here on; it waits for this one's end in turn.
__device__ __forceinline__ void wait_for_the_one_before()
{
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
}

template <typename... P, typename... A>
cudaError_t launch_after(cudaStream_t st, dim3 grid, int threads, size_t shared, void (*kernel)(P...), A... args)
{
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = shared;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}

}  // namespace gg
