// Programmatic launch: the kernel's CTAs are set up while the kernel before it on the stream drains.  A kernel launched this way
// calls wait_for_stream() before it touches memory; from there on everything earlier on the stream is done and visible.  What it
// reads may have been written while it was resident already, so it uses no loads that promise read-only data (__ldg, ld.global.nc):
// those may be moved over the wait and need not see such writes.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

namespace polyspec {

// Every pointer is a multiple of four or null: what arrays of 32-bit words need.
template <class... P>
inline bool aligned4(const P*... p) { return ((reinterpret_cast<uintptr_t>(p) | ...) & 3u) == 0; }

__device__ __forceinline__ void wait_for_stream() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

template <class... P, class... A>
cudaError_t launch_early(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t stream, A... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(static_cast<unsigned>(threads));
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}

}  // namespace polyspec
