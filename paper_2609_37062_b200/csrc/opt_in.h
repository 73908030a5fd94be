// A kernel's opt-in to more than 48 KB of shared memory, asked of the runtime once for every kernel and device.
#pragma once

#include <cuda_runtime_api.h>

namespace da {

// DA_OK or DA_ERR_CUDA.  `bytes` is the most that any launch of the kernel takes.
int opt_in_shared_memory(const void* kernel, int bytes);

}  // namespace da
