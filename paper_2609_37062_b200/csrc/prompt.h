// Attention of prompts (several new tokens per sequence) over the paged cache: the work list and
// what the host hands to the kernels.  Pure host types; the planner makes no CUDA call.
#pragma once

#include <cstdint>
#include <vector>

#include "decode_attn.h"

namespace da {

constexpr int kPromptRows = 128;        // query rows of one MMA tile: floor(128 / G) tokens x G heads
constexpr int kPromptTiles = 2;         // MMA tiles of a unit
constexpr int kPromptKvTokens = 128;    // a K/V tile: positions [128 t, 128 t + 128)
constexpr int kPromptDeterministicChunk = 4096;   // tokens, DETERMINISTIC's default

// Up to 2 floor(128 / G) consecutive new tokens of one sequence, all query heads of one KV head, against
// the tiles [tile_begin, tile_end) of the unit's list: the first sink_tiles tiles of the sequence, then
// the tiles from window_tile on.
typedef decode_attn_prompt_unit_t PromptUnit;

struct PromptLayout {
    std::vector<PromptUnit> units;          // in launch order: block b walks units block_begin[b] .. block_begin[b + 1]
    std::vector<int32_t> block_begin;
    std::vector<int32_t> merges;            // index of the first unit of every group of units that shares query rows
    int64_t n_slots = 0;                    // records (one per unit of such a group)
    int32_t longest = 0;                    // of the sequences
    int64_t q_rows = 0;                     // new tokens of all sequences
};

int validate_prompt_policy(const decode_attn_shape_t& s, const decode_attn_policy_t& p);
int make_prompt_layout(const decode_attn_shape_t& s, const decode_attn_policy_t& p, const int32_t* new_lens,
                       const int32_t* seq_lens, int sm_count, PromptLayout& out);

// floats of one record: 256 rows of D unnormalised outputs, then (maximum in the log2 domain, sum) of each
inline int64_t prompt_record_floats(int D) { return (int64_t)kPromptTiles * kPromptRows * (D + 2); }

}  // namespace da
