// Planner for prompts.  A unit is a run of up to 2 floor(128 / G) new tokens of one sequence (the
// two 128-row tiles a block works on) with all query heads of one KV head, against a range of the
// 128-token K/V tiles that any of its queries sees.
//
//  * AUTO deals the tiles out evenly: the units of the batch lie one behind the other, every block gets the
//    same share of their cost (tiles, and a fixed charge per unit), and a unit that straddles two
//    blocks is cut there; the pieces leave partial records that a second kernel merges.  Cuts keep away from a
//    unit's ends, and a share is never below kMinShare tiles, so short prompts stay whole.  (Whole units on
//    148 SMs: 512 equal units take 4 rounds where 3.46 would do.)
//  * DETERMINISTIC cuts every unit at multiples of chunk_tokens of its own tile list, so that a sequence's
//    bits depend on its lengths and the policy alone.
#include "prompt.h"

#include <algorithm>
#include <new>

#include "planner.h"

namespace da {

namespace {

constexpr int kUnitTiles = 1;     // a unit's set-up and epilogue, in tiles
constexpr int kMinShare = 6;      // tiles: below this a cut costs more (the merge launch) than it spreads
constexpr int kMinPiece = 3;
constexpr int64_t kMaxUnits = 1 << 22;    // 200 MB of work list, far beyond what one call is worth making for

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

}  // namespace

int validate_prompt_policy(const decode_attn_shape_t& s, const decode_attn_policy_t& p)
{
    const int rc = validate_policy(s, p);
    if (rc != DA_OK) return rc;
    if (p.split_mode == DA_SPLIT_FIXED_COUNT || p.kernel != DA_KERNEL_AUTO || p.fuse_combine || p.capacity_batch > 0 ||
        p.shared_prefix_tokens > 0 || p.track_weights || p.max_splits > 0 || p.ctas_per_sm > 0)
        return DA_ERR_UNSUPPORTED;
    if (p.split_mode == DA_SPLIT_DETERMINISTIC && p.chunk_tokens % kPromptKvTokens != 0) return DA_ERR_INVALID_ARG;
    return DA_OK;
}

static int fill_layout(const decode_attn_shape_t& s, const decode_attn_policy_t& p, const int32_t* new_lens,
                       const int32_t* seq_lens, int sm_count, PromptLayout& out)
{
    if (sm_count <= 0) return DA_ERR_INVALID_ARG;
    if (s.batch > 0 && (!new_lens || !seq_lens)) return DA_ERR_INVALID_ARG;
    const int G = s.num_q_heads / s.num_kv_heads;
    const int per_unit = kPromptTiles * (kPromptRows / G);
    out = PromptLayout();
    std::vector<PromptUnit> whole;
    int64_t row0 = 0, n_units = 0;
    for (int b = 0; b < s.batch; ++b) {
        if (new_lens[b] < 0 || seq_lens[b] < new_lens[b]) return DA_ERR_INVALID_ARG;
        if (ceil_div(seq_lens[b], s.page_size) > s.max_pages_per_seq) return DA_ERR_INVALID_ARG;
        n_units += ceil_div(new_lens[b], per_unit) * s.num_kv_heads;
        if (n_units > kMaxUnits) return DA_ERR_UNSUPPORTED;
    }
    whole.reserve((size_t)n_units);
    for (int b = 0; b < s.batch; ++b) {
        const int64_t first = (int64_t)seq_lens[b] - new_lens[b];
        out.longest = std::max(out.longest, seq_lens[b]);
        for (int g = 0; g < s.num_kv_heads; ++g) {
            // the longest units of a sequence first: its last tokens see the most
            for (int64_t t0 = (ceil_div(new_lens[b], per_unit) - 1) * per_unit; t0 >= 0; t0 -= per_unit) {
                PromptUnit u;
                u.seq = b;
                u.kv_head = g;
                u.n_tok = (int32_t)std::min<int64_t>(per_unit, new_lens[b] - t0);
                u.row = (int32_t)(row0 + t0);
                u.pos = (int32_t)(first + t0);
                u.seq_len = seq_lens[b];
                const int64_t lo = p.window_tokens > 0 ? std::max<int64_t>(0, u.pos - (int64_t)p.window_tokens + 1) : 0;
                const int64_t end = u.pos + (int64_t)u.n_tok;
                u.window_tile = (int32_t)(lo / kPromptKvTokens);
                u.sink_tiles = (int32_t)std::min<int64_t>(u.window_tile, ceil_div(std::min<int64_t>(p.sink_tokens, lo), kPromptKvTokens));
                u.tile_begin = 0;
                u.tile_end = (int32_t)(u.sink_tiles + ceil_div(end, kPromptKvTokens) - u.window_tile);
                u.slot = -1;
                u.n_pieces = 1;
                whole.push_back(u);
            }
        }
        row0 += new_lens[b];
        if (row0 > INT32_MAX) return DA_ERR_UNSUPPORTED;
    }
    out.q_rows = row0;
    out.block_begin.push_back(0);
    if (whole.empty()) return DA_OK;

    // Cuts of a unit: ascending tile indexes strictly inside it.  emit() adds the unit's pieces.
    std::vector<int32_t> cuts;
    auto emit = [&](const PromptUnit& u, const std::vector<int32_t>& at, auto&& each) {
        const int32_t n = (int32_t)at.size() + 1;
        if (n > 1) out.merges.push_back((int32_t)out.units.size());
        for (int32_t i = 0; i < n; ++i) {
            PromptUnit x = u;
            x.tile_begin = i == 0 ? u.tile_begin : at[i - 1];
            x.tile_end = i + 1 == n ? u.tile_end : at[i];
            x.n_pieces = n;
            if (n > 1) x.slot = (int32_t)(out.n_slots + i);
            out.units.push_back(x);
            each(i);
        }
        if (n > 1) out.n_slots += n;
    };

    if (p.split_mode == DA_SPLIT_DETERMINISTIC) {
        const int64_t chunk = std::max<int64_t>(1, (p.chunk_tokens > 0 ? p.chunk_tokens : kPromptDeterministicChunk) / kPromptKvTokens);
        int64_t pieces = 0;
        for (const PromptUnit& u : whole) pieces += ceil_div(u.tile_end, chunk);
        if (pieces > kMaxUnits) return DA_ERR_UNSUPPORTED;
        for (const PromptUnit& u : whole) {
            cuts.clear();
            for (int64_t t = chunk; t < u.tile_end; t += chunk) cuts.push_back((int32_t)t);
            emit(u, cuts, [](int32_t) {});
        }
        // pieces dealt round robin would break the runs that block_begin describes: equal shares of the list by cost
        int64_t total = 0;
        for (const PromptUnit& u : out.units) total += u.tile_end - u.tile_begin + kUnitTiles;
        const int64_t blocks = std::min<int64_t>(sm_count, (int64_t)out.units.size());
        int64_t done = 0, b = 1;
        for (size_t i = 0; i < out.units.size(); ++i) {
            const int64_t c = out.units[i].tile_end - out.units[i].tile_begin + kUnitTiles;
            // block b starts at the unit in whose first half its share begins
            while (b < blocks && done + c / 2 >= b * total / blocks && (int64_t)out.block_begin.size() == b) {
                out.block_begin.push_back((int32_t)i);
                ++b;
            }
            done += c;
        }
        while ((int64_t)out.block_begin.size() <= blocks) out.block_begin.push_back((int32_t)out.units.size());
        return DA_OK;
    }

    int64_t total = 0;
    for (const PromptUnit& u : whole) total += u.tile_end + kUnitTiles;
    // shares: at most one per SM, and not so many that a share falls below the smallest worth cutting for -
    // but never fewer than there are units to hand out
    const int64_t n_whole = (int64_t)whole.size();
    int64_t blocks = std::min<int64_t>(sm_count, std::max<int64_t>(n_whole, total / (kMinShare + kUnitTiles)));
    blocks = std::max<int64_t>(1, blocks);
    int64_t done = 0, b = 1;               // cost of the units before; the next block whose share begins
    for (const PromptUnit& u : whole) {
        const int64_t n = u.tile_end, c = n + kUnitTiles;
        cuts.clear();
        std::vector<int64_t> starts;       // for every block that begins inside this unit: the piece it begins with
        int64_t at_end = 0;                // blocks that begin right behind it
        for (; b < blocks; ++b) {
            const int64_t x = b * total / blocks - done;          // where the share begins, in tiles of this unit
            if (x >= c) break;
            int64_t cut = x;
            const int64_t lowest = cuts.empty() ? 0 : cuts.back();
            if (cut - lowest < kMinPiece) cut = lowest;            // too close to the piece before
            if (n - cut < kMinPiece && cut != 0) cut = n;          // too close to the end
            if (n < 2 * kMinPiece) cut = 2 * x < c ? 0 : n;        // short units stay whole: the nearer end
            if (cut >= n) {
                ++at_end;
            } else if (cut == 0) {
                starts.push_back(0);
            } else {
                if (cut != lowest) cuts.push_back((int32_t)cut);
                starts.push_back((int64_t)cuts.size());
            }
        }
        const int32_t first_unit = (int32_t)out.units.size();
        size_t next = 0;
        emit(u, cuts, [&](int32_t i) {
            while (next < starts.size() && starts[next] == i) {
                out.block_begin.push_back(first_unit + i);
                ++next;
            }
        });
        for (; at_end > 0; --at_end) out.block_begin.push_back((int32_t)out.units.size());
        done += c;
    }
    while ((int64_t)out.block_begin.size() <= blocks) out.block_begin.push_back((int32_t)out.units.size());
    return DA_OK;
}

int make_prompt_layout(const decode_attn_shape_t& s, const decode_attn_policy_t& p, const int32_t* new_lens,
                       const int32_t* seq_lens, int sm_count, PromptLayout& out)
{
    try {
        return fill_layout(s, p, new_lens, seq_lens, sm_count, out);
    } catch (const std::bad_alloc&) {
        return DA_ERR_UNSUPPORTED;        // (nothing throws across the C boundary)
    }
}

}  // namespace da

extern "C" int decode_attn_prompt_plan_layout(const decode_attn_shape_t* shape, const decode_attn_policy_t* policy,
                                              const int32_t* new_lens_host, const int32_t* seq_lens_host, int32_t sm_count,
                                              decode_attn_prompt_unit_t* units_out, int64_t max_units, int64_t* n_units_out,
                                              int32_t* block_begin_out, int64_t max_blocks, int64_t* n_blocks_out)
{
    if (!shape || !policy || !n_units_out || !n_blocks_out) return DA_ERR_INVALID_ARG;
    int rc = da::validate_shape(*shape);
    if (rc != DA_OK) return rc;
    rc = da::validate_prompt_policy(*shape, *policy);
    if (rc != DA_OK) return rc;
    da::PromptLayout lay;
    *n_units_out = *n_blocks_out = 0;
    rc = da::make_prompt_layout(*shape, *policy, new_lens_host, seq_lens_host, sm_count, lay);
    if (rc != DA_OK) return rc;
    *n_units_out = (int64_t)lay.units.size();
    *n_blocks_out = (int64_t)lay.block_begin.size() - 1;
    if (units_out) {
        if (max_units < *n_units_out) return DA_ERR_INVALID_ARG;
        std::copy(lay.units.begin(), lay.units.end(), units_out);
    }
    if (block_begin_out) {
        if (max_blocks < *n_blocks_out) return DA_ERR_INVALID_ARG;
        std::copy(lay.block_begin.begin(), lay.block_begin.end(), block_begin_out);
    }
    return DA_OK;
}
