// Programmatic dependent launch for the decode kernels, which run one after the other and are each a few microseconds long.
#pragma once
#include "common.cuh"

// Every kernel of the step lets the next one be scheduled as soon as all of its own
// CTAs have started, and waits for the kernel before it (completion and visibility of its writes) before it touches
// global memory.  The wait comes first in every CTA, also in those that return early, so that "kernel N complete"
// always implies "kernel N - 1 complete".
// One kernel reads before its wait: the join of attention over pages reads the sequences' lengths.  It is always launched behind the attention kernel,
// which does not write them, and whose CTAs release their dependents only behind their own wait, so whatever wrote the lengths is complete
// before a CTA of the join starts.  That rests on the order of the two instructions in pdl_enter.
CCA_DEVINL void pdl_enter() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}
template <typename... KArgs, typename... Args>
inline cudaError_t launch_pdl_smem(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at;
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}
template <typename... KArgs, typename... Args>
inline cudaError_t launch_pdl(void (*kernel)(KArgs...), dim3 grid, dim3 block, cudaStream_t st, Args... args) {
  return launch_pdl_smem(kernel, grid, block, 0, st, args...);
}
