// Launches of the kernel for caches in 4 bits, as the C ABI calls them (kernel_packed.cu).
#pragma once

#include <cuda_runtime_api.h>

#include "decode_attn.h"

namespace da {

struct KernelParams;

// Resident blocks per SM, -1 if that cannot be told; opts the kernel in to its shared memory.  ext: windowed plans.
int packed_query_occupancy(int D, int G, bool ext, int* block_threads, int* dyn_smem);
int packed_launch(const decode_attn_shape_t& s, int G, const KernelParams& kp, unsigned grid, cudaStream_t stream);

}  // namespace da
