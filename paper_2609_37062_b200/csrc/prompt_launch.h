// One call of the prompt kernels, as the C ABI hands it to the launch code.
#pragma once

#include <cuda_runtime_api.h>

#include "prompt.h"

namespace da {

struct PromptCall {
    const void* q;
    const void* k_cache;
    const void* v_cache;
    const int32_t* block_table;
    const int32_t* seq_lens;
    void* out;
    float* lse;
    float* ws;
    const PromptUnit* units;        // the plan's device buffer
    const int32_t* block_begin;
    const int32_t* merges;
    int32_t* status;
    unsigned n_blocks, n_merges;
    int64_t q_rows;
    int32_t window, sinks;
    float scale;
};

// The attention launch and, if any unit was cut, the merge launch.
int prompt_launch(const decode_attn_shape_t& s, const PromptCall& c, cudaStream_t stream);

}  // namespace da
