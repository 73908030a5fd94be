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

// Between the two, up to a pair for every block of 4 warps, either may be the better: large blocks balance long and short sequences
// without cutting them.  A plan for given lengths is made for both sizes, and the one that the planner thinks faster is taken (us
// with blocks of 4 and of 8, 32/8 heads of 128: 64 rows of 30 to 4,000 tokens 41.2 and 33.6, 32 of 8,000 62.7 and 60.4, 20 of 900 12.2
// and 11.4; 64 of 464 13.1 and 15.7, 64 of 4,000 58.9 and 62.1, 32 of 30 to 4,000 22.6 and 26.0).
inline bool packed_either_size(const decode_attn_shape_t& s, const decode_attn_policy_t& p, int sm_count)
{
    const int64_t pairs = (int64_t)s.batch * s.num_kv_heads;
    return p.split_mode == DA_SPLIT_AUTO && p.capacity_batch == 0 && p.ctas_per_sm == 0 && s.num_q_heads <= 8 * s.num_kv_heads &&
           pairs >= sm_count && pairs <= 4 * (int64_t)sm_count;
}

// Resident blocks per SM, -1 if that cannot be told; opts the kernel in to its shared memory.  ext: windowed plans.
int packed_query_occupancy(int D, int G, bool ext, bool big, int* block_threads, int* dyn_smem);
int packed_launch(const decode_attn_shape_t& s, int G, bool big, const KernelParams& kp, unsigned grid, cudaStream_t stream);

}  // namespace da
