// Launches of the kernel for caches in 4 bits, as the C ABI calls them (kernel_packed.cu).
#pragma once

#include <cuda_runtime_api.h>

#include <cstdint>

#include "decode_attn.h"

namespace da {

struct KernelParams;

// A block has 8 warps (`big`) or 4; for groups of more than 8 heads, 4 either way.  With 4, four blocks share an SM and
// their ends of units overlap (64 rows of 464 tokens: 12.8 us against 15.5); with 8 there are half as many records to merge,
// which is what counts when few rows are cut into many pieces (one row of 32,768: 15.2 us against 17.5).
inline bool packed_big_blocks(int64_t pairs, int sm_count) { return pairs < sm_count; }

// Resident blocks per SM, -1 if that cannot be told; opts the kernel in to its shared memory.  ext: windowed plans.
int packed_query_occupancy(int D, int G, bool ext, bool big, int* block_threads, int* dyn_smem);
int packed_launch(const decode_attn_shape_t& s, int G, bool big, const KernelParams& kp, unsigned grid, cudaStream_t stream);

}  // namespace da
