// Launches of the kernel for caches in 4 bits, as the C ABI calls them (kernel_packed.cu).
#pragma once

#include <cuda_runtime_api.h>

#include <cstdint>

#include "decode_attn.h"

namespace da {

struct KernelParams;

// A block's team has 8 warps (`big`) or 4; groups of more than 8 heads take two teams of 4 either way.  With 4, four blocks
// share an SM: their ends of units overlap.  With 8 there are half as many records to merge, which is what counts when few
// rows are cut into many pieces.
inline bool packed_big_blocks(int64_t pairs, int sm_count) { return pairs < sm_count; }

// Resident blocks per SM, -1 if that cannot be told; opts the kernel in to its shared memory.  ext: windowed plans.
int packed_query_occupancy(int D, int G, bool ext, bool big, int* block_threads, int* dyn_smem);
int packed_launch(const decode_attn_shape_t& s, int G, bool big, const KernelParams& kp, unsigned grid, cudaStream_t stream);

}  // namespace da
