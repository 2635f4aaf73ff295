// Launches that follow each other on a stream as programmatic dependents: a kernel may start
// before the one ahead of it has ended, sets up what needs no memory and then waits for that
// end (and, through it, for everything before).
//
// Every kernel launched with launch_after calls dependency_wait in all its threads before it
// reads what the launch ahead of it wrote and before it writes global memory, and dependency_start,
// which lets the next launch start, only after that. A kernel so starts when the last but one before
// it has ended, and at most one kernel runs beside the ones that wait. What that last but one wrote,
// or an older one, may be read before the wait, from the L2 (__ldcg: nothing but the wait says that an
// SM's own cache holds no older copy), by a launch that is always behind another one of the same call
// (whose own wait shows that the call's inputs are complete too).
//
// Behind its wait a kernel reads memory with ordinary loads alone: the non-coherent ones (__ldg, or
// a const __restrict__ pointer) are for what nobody writes while the kernel runs, and may be moved
// ahead of the wait.
#pragma once
#include <cuda_runtime.h>

namespace sqi {
namespace {

__device__ __forceinline__ void dependency_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void dependency_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

template <typename... Params, typename... Args>
cudaError_t launch_after(void (*kernel)(Params...), unsigned grid, int threads, size_t smem, cudaStream_t stream,
                         Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid, 1, 1);
  cfg.blockDim = dim3(threads, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<Params>(args)...);
}

}  // namespace
}  // namespace sqi
