// The cache in 4 bits: where a tile of 16 tokens of one KV head holds what (the layout is the C ABI's).
//
// A value is a code in e2m1 times the fp16 scale of its 32 dims.  The order of the bytes is that in which the attending
// warps want their mma operands (kernel_packed.cuh): a lane's K codes of a row are one 16-byte load (8 bytes at head_dim
// 64) whose words are the dims of one scale each, its V scales of four tokens one 8-byte load, and no load of a warp has
// a bank conflict.
#pragma once

#include <cstdint>

#ifdef __CUDACC__
#define DA_PACKED_HD __host__ __device__
#else
#define DA_PACKED_HD
#endif

namespace da {

// bytes of a tile and of its parts
DA_PACKED_HD constexpr int packed_tile_bytes(int D) { return 16 * D + 64 * (D / 32); }
DA_PACKED_HD constexpr int packed_v_codes(int D) { return 8 * D; }
DA_PACKED_HD constexpr int packed_k_scales(int D) { return 16 * D; }
DA_PACKED_HD constexpr int packed_v_scales(int D) { return 16 * D + 32 * (D / 32); }

// The word (4 bytes) of a row's K codes, counted within the tile's K codes, that holds dims 8 w .. 8 w + 7.
DA_PACKED_HD constexpr int packed_k_word(int D, int row, int w) { return row * (D / 8) + (w % 4) * (D / 32) + w / 4; }
// The same for V, within the tile's V codes: at head_dim 128 the halves of a row change places in rows 8 to 15.
DA_PACKED_HD constexpr int packed_v_word(int D, int row, int w) { return row * (D / 8) + (D == 128 ? w ^ (row & 8) : w); }
// The fp16 scale of a row's block of 32 dims, within the tile's K and V scales.
DA_PACKED_HD constexpr int packed_k_scale(int D, int row, int block) { return row * (D / 32) + block; }
DA_PACKED_HD constexpr int packed_v_scale(int row, int block) { return 16 * block + (row & ~3) + ((row & 3) ^ (row >> 2)); }

}  // namespace da
