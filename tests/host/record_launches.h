// Forced in front of the layers' and losses' sources: launches are written down instead of made, so that grids can be looked at on the
// CPU.  Kernels become device functions that nothing calls, which a host-only build leaves out.
#pragma once
#include <hip/hip_runtime.h>

void record_launch(const char* kernel, dim3 grid, dim3 block, size_t lds);
#undef hipLaunchKernelGGL
#define hipLaunchKernelGGL(kernel, grid, block, lds, stream, ...) record_launch(#kernel, grid, block, lds)
#undef __global__
#define __global__ __device__
#undef __launch_bounds__
#define __launch_bounds__(...)
