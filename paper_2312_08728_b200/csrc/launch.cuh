// A kernel's start beside the end of the one before it.
#pragma once
#include <cuda_runtime.h>

namespace bmgdk {

// A kernel launched as a dependent of the one before it may start while that one still runs; before it touches memory it
// waits until that one has finished (and with it all before).  What it reads then may have been written while it ran already, so its loads take the ordinary path (__ldca, __ldcs): those of the
// read-only path (__ldg, const __restrict__) are for memory that nobody writes while the kernel lives.
__device__ __forceinline__ void wait_for_previous_kernel() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_next_kernel_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }


}  // namespace bmgdk
