// Attention of prompts on the tcgen05 tensor cores: many query rows per sequence over the paged
// cache, causal, with an optional sliding window and sinks.
//
// The query at position i sees the positions t <= i with i - t < window or t < sinks (all of t <= i without a
// window).  A unit (prompt.h) is two 128-row MMA tiles A and B - floor(128 / G) consecutive tokens
// each, with the G query heads of one KV head side by side, so that a K/V byte serves them all -
// against a list of 128-token K/V tiles.  Per K/V tile j and MMA tile x:
//
//   S_x = Q_x K_j^T       128 x 128 x D, accumulator in tensor-memory columns [128 x, 128 x + 128)
//   softmax               one thread per row: the row's maximum, p = 2^(s * scale * log2 e - m), the row sum;
//                         p as two 16-bit values per column back over the logits.  p is rounded once to the 16-bit
//                         input type (the MMA takes no mixed types); its relative error, at most 2^-8 in bf16 and 2^-11
//                         in fp16, averages out over the tokens, and the row sum is of the unrounded p.
//   O_x += P_x V_j        accumulator in columns [256 + 128 x, 256 + 128 x + D), kept over all tiles
//
// m only follows the row's maximum when that has grown by more than 2^8 (p stays below 2^8, well inside fp16):
// until then O and the sum keep their scale; when it does, the row's O is fetched, scaled and put back.
//
// Threads: four softmax warps for A, four for B, one warp of which one lane issues the MMAs, two that issue the
// TMA boxes.  The MMA order is  P_A V_j, Q_A K_{j+1}, P_B V_j, Q_B K_{j+1}:  while one MMA tile's softmax runs,
// the tensor core works for the other.  Blocks are persistent and walk their run of the work list; tensor memory
// and shared memory stay set up, the barriers count on.
//
// Tiles the mask leaves whole are not masked.  16-token boxes no query of the unit sees, and what lies past the
// end, are fetched from outside the pool (the TMA unit fills zeros) and their pages are never looked at; a box
// that holds both visible and hidden rows is copied by hand for V with the hidden rows cleared, because a zero
// weight does not silence what such a row may hold.
//
// Bound: a step of both MMA tiles against 128 tokens is 2,048 cycles of MMA (32 of 64 cycles at D 128) and 2,048 of the
// exponential unit, and takes about 3,100: one MMA tile's chain of logits, weights, P V and the next logits is that long,
// and there is tensor memory for two such chains.  What it is made of (timing builds, 4,096 queries, window 4,096,
// 32/8 heads of 128, 243 us): without exponentials 213 us, without maxima and loads either 203, without the MMAs too 142 - the
// hand-overs between the warps and the tensor core, the moves through tensor memory, a unit's set-up and output.
#pragma once

#include <type_traits>

#include "kernel_umma.cuh"
#include "prompt.h"

namespace da {

struct PromptParams {
    const __nv_bfloat16* v;
    const int32_t* block_table;
    const int32_t* seq_lens;
    void* out;
    float* lse;
    float* ws;
    const PromptUnit* units;
    const int32_t* block_begin;
    const int32_t* merges;
    int32_t* status;
    int64_t v_stride_page, v_stride_token, v_stride_head;
    int64_t num_pages;
    int32_t num_q_heads, num_kv_heads, max_pages_per_seq;
    int32_t group, tokens_per_tile;  // floor(128 / group)
    int32_t window, sinks;
    int32_t tile_shift;              // log2(page_size / 16)
    int32_t out_kind;
    float scale_log2;
};

constexpr int kPromptSoftmaxWarps = 8;
constexpr int kPromptMmaWarp = 8, kPromptLoadWarp = 9;   // and 10
constexpr int kPromptThreads = 384;       // three warpgroups: two of softmax, the third with the MMA and the load warps
// Registers: 384 x 168 at launch; the softmax warpgroups take what the third gives back, 256 x 216 + 128 x 72 in all.
constexpr int kPromptSoftmaxRegs = 216, kPromptOtherRegs = 72;
static_assert(256 * kPromptSoftmaxRegs + 128 * kPromptOtherRegs <= 384 * 168, "more registers than the block was launched with");

constexpr int kPromptStageBytes = kPromptSoftmaxWarps * 32 * 128;   // outputs on their way out: 128 bytes of a row per thread

template <int D>
struct PromptCfg {
    static constexpr int kHalves = D / 64;                       // 128-byte column blocks of a row
    static constexpr int kHalfBytes = 128 * 128;                 // 128 rows x 64 dims
    static constexpr int kTileBytes = kHalves * kHalfBytes;      // Q tile, K tile, V tile
    static constexpr int kStages = D == 128 ? 2 : 4;             // of K, and of V
    static constexpr int kBarriers = 14 + 4 * kStages + 1;
    static constexpr int kSmemBytes = (2 + 2 * kStages) * kTileBytes + kPromptStageBytes + 512 + 1024 /* alignment */;
    static_assert(kSmemBytes > 114 * 1024 && kSmemBytes <= 227 * 1024, "one block per SM: each takes all of tensor memory");
};
constexpr float kPromptRescale = 8.f;                            // log2: how far a row's maximum may run ahead of its scale

// One lane of a converged warp, always the same one.  The MMAs are issued under this predicate, at the place: the
// compiler knows it for what it is and keeps descriptors in uniform registers.  (Under lane == 0 every operand of every MMA
// is moved there first, which paced the issue: 85 to 95 cycles an MMA instead of 64.)
__device__ __forceinline__ bool elect_one()
{
    uint32_t is;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(is));
    return is != 0;
}

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2)
                 : "memory");
}

// Bits 0 .. n - 1, for any n.
__device__ __forceinline__ uint32_t low_bits(int n) { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; }

// Two fp32 values in a register pair: one instruction works on both.
__device__ __forceinline__ uint64_t pack2(float lo, float hi)
{
    uint64_t v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(lo), "f"(hi));
    return v;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t v;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(v) : "l"(a), "l"(b), "l"(c));
    return v;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b)
{
    uint64_t v;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(a), "l"(b));
    return v;
}
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float v;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(v) : "f"(a), "f"(b), "f"(c));
    return v;
}

// Whole warp.
__device__ __forceinline__ bool prompt_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag)
{
    return __all_sync(0xffffffffu, umma_wait(bar, parity, abort_flag));
}

// The same wait without suspending the warp: for the waits that the tensor core stands still behind (a suspended
// warp comes back some 400 cycles after the last arrival).
__device__ __forceinline__ bool prompt_spin(uint32_t bar, uint32_t parity, volatile int* abort_flag)
{
    const long long t0 = clock64();
    for (int i = 1;; ++i) {
        if (__any_sync(0xffffffffu, mbar_test_wait(bar, parity))) return true;
        if ((i & 63) == 0) {
            bool stop = *abort_flag != 0;
            if (!stop && clock64() - t0 > kWaitLimitCycles) {
                *abort_flag = 1;
                stop = true;
            }
            if (__any_sync(0xffffffffu, stop)) return false;
        }
    }
}

template <int D, bool F16>
__global__ void __launch_bounds__(kPromptThreads, 1)
decode_attn_prompt_kernel(const PromptParams p, const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map,
                          const __grid_constant__ CUtensorMap v_map)
{
    using Cfg = PromptCfg<D>;
    constexpr int NS = Cfg::kStages;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    uint8_t* const gbase = smem_raw + (base - raw);
    const uint32_t q_base = base, k_base = base + 2 * Cfg::kTileBytes, v_base = k_base + NS * Cfg::kTileBytes;
    const uint32_t stage_base = v_base + NS * Cfg::kTileBytes;
    const uint32_t bar_base = stage_base + kPromptStageBytes;
    // per MMA tile x: q (its rows have landed), qe (no longer read), s (logits complete), p (weights written: of the first 96
    // tokens, of the last 32), o (P V complete), of (output read); per stage: K and V landed (kf, vf), K and V no longer read (ke, ve); drain
    auto bar_q = [&](int x) { return bar_base + 8 * x; };
    auto bar_s = [&](int x) { return bar_base + 16 + 8 * x; };
    auto bar_p = [&](int x, int half) { return bar_base + 32 + 16 * x + 8 * half; };
    auto bar_o = [&](int x) { return bar_base + 64 + 8 * x; };
    auto bar_of = [&](int x) { return bar_base + 80 + 8 * x; };
    auto bar_qe = [&](int x) { return bar_base + 96 + 8 * x; };
    const uint32_t bar_kf = bar_base + 112, bar_ke = bar_kf + 8 * NS, bar_vf = bar_ke + 8 * NS, bar_ve = bar_vf + 8 * NS;
    const uint32_t bar_drain = bar_ve + 8 * NS;
    uint8_t* const misc = gbase + (bar_base - base);
    static_assert(8 * Cfg::kBarriers <= 256, "barriers");
    volatile uint32_t* const sm_tmem = reinterpret_cast<volatile uint32_t*>(misc + 256);
    volatile int* const sm_abort = reinterpret_cast<volatile int*>(misc + 260);

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int ubeg = __ldg(p.block_begin + blockIdx.x), uend = __ldg(p.block_begin + blockIdx.x + 1);
    if (ubeg >= uend) {
        if (blockIdx.x == 0) pdl_wait_primary();
        return;
    }
    if (tid == 0) {
        tma_prefetch_descriptor(&q_map);
        tma_prefetch_descriptor(&k_map);
        tma_prefetch_descriptor(&v_map);
        for (int x = 0; x < 2; ++x) {
            mbar_init(bar_q(x), 1);
            mbar_init(bar_qe(x), 1);
            mbar_init(bar_s(x), 1);
            mbar_init(bar_p(x, 0), 4);
            mbar_init(bar_p(x, 1), 4);
            mbar_init(bar_o(x), 1);
            mbar_init(bar_of(x), 4);
        }
        for (int i = 0; i < 4 * NS; ++i) mbar_init(bar_kf + 8 * i, 1);
        mbar_init(bar_drain, 1);
        *sm_abort = 0;
        mbar_init_fence();
    }
    if (warp == kPromptMmaWarp) umma::tmem_alloc(smem_u32(const_cast<uint32_t*>(sm_tmem)), 512);
    umma::fence_before_thread_sync();
    __syncthreads();
    umma::fence_after_thread_sync();
    const uint32_t tmem = *sm_tmem;
    pdl_wait_primary();

    const int G = p.group, TQ = p.tokens_per_tile;
    auto tile_at = [](const PromptUnit& u, int i) { return i < u.sink_tiles ? i : i - u.sink_tiles + u.window_tile; };

    // The warp's number as a value known to be the same in all its lanes: branches on it then keep what the roles
    // share in uniform registers (without: 188 bytes spilled instead of 96, 297 us instead of 284 for 4,096 queries).
    const int role = __shfl_sync(0xffffffffu, warp, 0);
    if (role >= kPromptSoftmaxWarps) {
        // (one instruction for the whole warpgroup, its idle fourth warp included, ahead of the roles; and inside the
        // branch: the compiler allocates the code behind it by what it sees there)
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kPromptOtherRegs));
        if (role == kPromptLoadWarp || role == kPromptLoadWarp + 1) {
            // ------------------------------------------------------------ TMA: a warp for Q and K, a warp for V
            // (a warp takes 1,400 cycles to issue the 16 boxes of a tile, 90 each, while the softmax warps beside it are busy, so
            // that one warp for both tensors falls behind: 251 against 247 us)
            const bool is_v = warp == kPromptLoadWarp + 1;
            const CUtensorMap* const map = is_v ? &v_map : &k_map;
            const uint32_t ring = is_v ? v_base : k_base, bar_full = is_v ? bar_vf : bar_kf, bar_empty = is_v ? bar_ve : bar_ke;
            const uint64_t keep = l2_policy_evict_normal();
            const int ts = p.tile_shift;
            const int sub = (lane / Cfg::kHalves) & 7, hf = lane % Cfg::kHalves;    // lane's box: 16 tokens, half of the head dimension
            constexpr int BOXES = 8 * Cfg::kHalves;
            int n = 0;                                                              // tiles so far
            int cu[2] = {0, 0};                                                     // units so far, per MMA tile
            bool ok = true;
            for (int ui = ubeg; ui < uend && ok; ++ui) {
                const PromptUnit u = p.units[ui];
                const int lo = p.window > 0 ? max(0, u.pos - p.window + 1) : 0;     // what the first query sees through its window
                const int end = min(u.pos + u.n_tok, u.seq_len);
                const int32_t* const bt = p.block_table + (int64_t)u.seq * p.max_pages_per_seq;
                auto seen = [&](int s0) { return s0 < end && (s0 + 15 >= lo || s0 < p.sinks); };
                auto whole = [&](int s0) { return s0 + 15 < u.seq_len && (s0 >= lo || s0 + 15 < p.sinks); };
                auto page_of = [&](int i) {                                         // of this lane's 16 tokens in list tile i
                    if (i >= u.tile_end) return (int)p.num_pages;
                    const int s0 = tile_at(u, i) * kPromptKvTokens + sub * 16;
                    return seen(s0) ? __ldg(bt + (s0 >> (ts + 4))) : (int)p.num_pages;
                };
                int page = page_of(u.tile_begin);
                for (int i = u.tile_begin; i < u.tile_end && ok; ++i, ++n) {
                    const int s0 = tile_at(u, i) * kPromptKvTokens + sub * 16;
                    const int next_page = page_of(i + 1);
                    if ((unsigned)page >= (unsigned)p.num_pages && seen(s0)) {
                        record_status(p.status, DA_ERR_BAD_PAGE);                   // such a box is read as zeros
                        page = (int)p.num_pages;
                    }
                    const int slot0 = (s0 >> 4 & ((1 << ts) - 1)) << 4;
                    const int st = n % NS;
                    if (n >= NS) ok = prompt_wait(bar_empty + 8 * st, (uint32_t)(n / NS + 1) & 1u, sm_abort);
                    if (!ok) break;
                    // V boxes with rows to clear are copied by hand
                    const bool part = is_v && seen(s0) && !whole(s0);
                    const uint32_t parts = __ballot_sync(0xffffffffu, part && hf == 0 && lane < BOXES);
                    for (uint32_t m = parts; m != 0; m &= m - 1) {
                        const int from = __ffs(m) - 1;                              // the lane whose box it is
                        const int pg = __shfl_sync(0xffffffffu, page, from), k0 = __shfl_sync(0xffffffffu, s0, from);
                        const int sl = __shfl_sync(0xffffffffu, slot0, from), sb = __shfl_sync(0xffffffffu, sub, from);
                        for (int c = lane; c < 16 * (D / 8); c += 32) {
                            const int r = c / (D / 8), ch = c % (D / 8), k = k0 + r;
                            uint4 x = make_uint4(0u, 0u, 0u, 0u);
                            if (k < u.seq_len && (k >= lo || k < p.sinks) && pg < p.num_pages)
                                x = __ldg(reinterpret_cast<const uint4*>(p.v + (int64_t)pg * p.v_stride_page +
                                                                         (int64_t)(sl + r) * p.v_stride_token +
                                                                         (int64_t)u.kv_head * p.v_stride_head) + ch);
                            *reinterpret_cast<uint4*>(gbase + (v_base - base) + st * Cfg::kTileBytes + (ch >> 3) * Cfg::kHalfBytes +
                                                      sb * 2048 + swz(r, ch & 7)) = x;
                        }
                    }
                    if (parts != 0) {
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        __syncwarp();
                    }
                    if (lane == 0) mbar_arrive_expect_tx(bar_full + 8 * st, Cfg::kTileBytes - __popc(parts) * (16 * D * 2));
                    __syncwarp();
                    if (lane < BOXES && !part)
                        tma_load_4d(ring + st * Cfg::kTileBytes + hf * Cfg::kHalfBytes + sub * 2048, map, bar_full + 8 * st, hf * 64, slot0,
                                    u.kv_head, page, keep);
                    if (!is_v && i == u.tile_begin) {
                        // The unit's query rows: TQ tokens x the group's heads, rows of the MMA tile in that order.  (Tokens of
                        // a ragged end are other rows of q, or zeros behind the last: what comes of them is not stored.)
                        for (int x = 0; x < (u.n_tok > TQ ? 2 : 1) && ok; ++x) {
                            if (cu[x] > 0) ok = prompt_wait(bar_qe(x), (uint32_t)(cu[x] - 1) & 1u, sm_abort);
                            if (!ok) break;
                            ++cu[x];
                            if (lane == 0) {
                                mbar_arrive_expect_tx(bar_q(x), Cfg::kHalves * G * TQ * 128);
                                for (int h = 0; h < Cfg::kHalves; ++h)
                                    tma_load_3d(q_base + x * Cfg::kTileBytes + h * Cfg::kHalfBytes, &q_map, bar_q(x), h * 64, u.kv_head * G,
                                                u.row + x * TQ);
                            }
                            __syncwarp();
                        }
                    }
                    page = next_page;
                }
            }
            if (*sm_abort != 0) {
                // given up somewhere: nothing may land in shared memory after the block has left (a copy always lands)
                for (int i = max(0, n - NS); i <= n; ++i)
                    if (i < n || !ok) mbar_wait(bar_full + 8 * (i % NS), (uint32_t)(i / NS) & 1u, i < n ? kWaitLimitCycles : 1000000LL);
                for (int x = 0; x < 2; ++x)
                    if (cu[x] > 0) mbar_wait(bar_q(x), (uint32_t)(cu[x] - 1) & 1u);
            }
        } else if (role == kPromptMmaWarp) {
            // ------------------------------------------------------------ MMAs (the warp together, one lane issues)
            {
                constexpr uint32_t idesc_qk = umma::instr_desc_16(128, 128, false, F16);
                constexpr uint32_t idesc_pv = umma::instr_desc_16(128, D, true, F16);
                constexpr uint32_t kTileUnits = Cfg::kTileBytes >> 4, kHalfUnits = Cfg::kHalfBytes >> 4;
                const uint64_t q_desc = umma::smem_desc_sw128(q_base, 16, 1024);
                const uint64_t k_desc = umma::smem_desc_sw128(k_base, 16, 1024);
                const uint64_t v_desc = umma::smem_desc_sw128(v_base, Cfg::kHalfBytes, 1024);
                int n = 0;                                        // K/V tiles before the unit
                int cs[2] = {0, 0}, cu[2] = {0, 0};               // per MMA tile: P V issued, units begun
                bool ok = true;
                for (int ui = ubeg; ui < uend && ok; ++ui) {
                    const PromptUnit u = p.units[ui];
                    const int T = u.tile_end - u.tile_begin;
                    const int X = u.n_tok > TQ ? 2 : 1;
                    auto qk = [&](int x, int j) {
                        const int st = (n + j) % NS;
                        umma::fence_after_thread_sync();
                        const uint64_t qd = q_desc + (uint64_t)(x * kTileUnits), kd = k_desc + (uint64_t)(st * kTileUnits);
                        if (elect_one()) {
#pragma unroll
                            for (int ks = 0; ks < D / 16; ++ks) {
                                const uint32_t off = (ks >> 2) * kHalfUnits + (ks & 3) * 2;
                                umma::mma_ss(tmem + x * 128, qd + off, kd + off, idesc_qk, ks > 0);
                            }
                            umma::commit(bar_s(x));
                            if (x == X - 1) umma::commit(bar_ke + 8 * st);
                            if (j == T - 1) umma::commit(bar_qe(x));
                        }
                        __syncwarp();
                    };
                    auto pv = [&](int x, int j, int part) {                        // the first 96 tokens, the last 32
                        const int st = (n + j) % NS;
                        umma::fence_after_thread_sync();
                        const uint64_t vd = v_desc + (uint64_t)(st * kTileUnits);
                        const uint32_t pd = tmem + x * 128, od = tmem + 256 + x * 128;
                        if (elect_one()) {
                            if (part == 0) {
#pragma unroll
                                for (int k = 0; k < 6; ++k) umma::mma_ts(od, pd + k * 8, vd + k * 128, idesc_pv, j > 0 || k > 0);
                            } else {
#pragma unroll
                                for (int k = 6; k < 8; ++k) umma::mma_ts(od, pd + k * 8, vd + k * 128, idesc_pv, true);
                                umma::commit(bar_o(x));
                                if (x == X - 1) umma::commit(bar_ve + 8 * st);
                            }
                        }
                        __syncwarp();
                    };
                    auto k_landed = [&](int j) {
                        return prompt_wait(bar_kf + 8 * ((n + j) % NS), (uint32_t)((n + j) / NS) & 1u, sm_abort);
                    };
                    for (int x = 0; x < X && ok; ++x) {
                        ok = prompt_wait(bar_q(x), (uint32_t)cu[x] & 1u, sm_abort) && k_landed(0);
                        if (ok) qk(x, 0);
                    }
                    for (int j = 0; j < T && ok; ++j) {
                        for (int x = 0; x < X && ok; ++x) {
                            // (the weights last: every wait behind theirs would be time the tensor core stands still)
                            ok = prompt_wait(bar_vf + 8 * ((n + j) % NS), (uint32_t)((n + j) / NS) & 1u, sm_abort) &&
                                 (j > 0 || cu[x] == 0 || prompt_wait(bar_of(x), (uint32_t)(cu[x] - 1) & 1u, sm_abort)) &&
                                 prompt_spin(bar_p(x, 0), (uint32_t)cs[x] & 1u, sm_abort);
                            if (!ok) break;
                            pv(x, j, 0);
                            ok = prompt_spin(bar_p(x, 1), (uint32_t)cs[x] & 1u, sm_abort);
                            if (!ok) break;
                            pv(x, j, 1);
                            ++cs[x];
                            if (j + 1 < T) {
                                ok = k_landed(j + 1);
                                if (ok) qk(x, j + 1);
                            }
                        }
                    }
                    for (int x = 0; x < X; ++x) ++cu[x];
                    n += T;
                }
                // nothing may arrive on a barrier, or be written, after the block has left
                if (ok)
                    for (int i = max(0, n - NS); i < n; ++i) {
                        ok = ok && prompt_wait(bar_ke + 8 * (i % NS), (uint32_t)(i / NS) & 1u, sm_abort);
                        ok = ok && prompt_wait(bar_ve + 8 * (i % NS), (uint32_t)(i / NS) & 1u, sm_abort);
                    }
                for (int x = 0; x < 2; ++x)
                    if (cu[x] > 0) ok = ok && prompt_wait(bar_qe(x), (uint32_t)(cu[x] - 1) & 1u, sm_abort);
                if (!ok) {
                    if (elect_one()) umma::commit(bar_drain);
                    mbar_wait(bar_drain, 0);
                }
            }
            __syncwarp();
        }
    } else {
        // ------------------------------------------------------------ softmax, output: one thread per row
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kPromptSoftmaxRegs));
        const int x = warp >> 2, r = (warp & 3) * 32 + lane;
        const int tok = r / G, h = r - tok * G;
        const uint32_t lane_base = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const uint32_t sc = lane_base + x * 128, oc = lane_base + 256 + x * 128;
        int cs = 0;                                                            // K/V tiles of this MMA tile so far
        bool ok = true;
        auto in_unit = [&](const PromptUnit& u) { return x == 0 || u.n_tok > TQ; };
        auto row_valid = [&](const PromptUnit& u) { return tok < TQ && x * TQ + tok < u.n_tok; };
        int ui = ubeg;
        PromptUnit u = p.units[ui];
        if (!in_unit(u)) {
            for (++ui; ui < uend; ++ui) {
                u = p.units[ui];
                if (in_unit(u)) break;
            }
        }
        while (ui < uend && ok) {
            const bool valid = row_valid(u);
            const int q_lo = u.pos + x * TQ, q_hi = min(u.pos + u.n_tok, q_lo + TQ) - 1;     // this MMA tile's queries
            const int qi = valid ? q_lo + tok : q_lo;
            float m = -INFINITY, l = 0.f;
            for (int i = u.tile_begin; i < u.tile_end; ++i, ++cs) {
                const int t0 = tile_at(u, i) * kPromptKvTokens;
                ok = prompt_wait(bar_s(x), (uint32_t)cs & 1u, sm_abort);
                if (!ok) break;
                umma::fence_after_thread_sync();
                uint32_t s[2][64];
                umma::ld64(sc, s[0]);
                umma::wait_ld();
                umma::ld64(sc + 64, s[1]);                                     // on its way while the first half is looked through
                const bool masked = t0 + kPromptKvTokens - 1 > q_lo ||
                                    (p.window > 0 && t0 <= q_hi - p.window && t0 + kPromptKvTokens > p.sinks);
                float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int hh = 0; hh < 2; ++hh) {
                    if (hh == 1) umma::wait_ld();
                    if (masked) {
                        // one bit per column, 32 at a time, then 32 selects on known bits (conditions column by column
                        // become branches: 15,000 cycles a tile instead of a few hundred)
                        const int hi = qi - t0 + 1, lo = p.window > 0 ? qi - p.window + 1 - t0 : 0, sk = p.sinks - t0;
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            const int c0 = 64 * hh + 32 * q;
                            const uint32_t vis = low_bits(hi - c0) & (~low_bits(lo - c0) | low_bits(sk - c0));
#pragma unroll
                            for (int c = 0; c < 32; ++c) {
                                uint32_t& v = s[hh][32 * q + c];
                                v = (vis & (1u << c)) != 0u ? v : 0xff800000u;                   // -inf
                            }
                        }
                    }
#pragma unroll
                    for (int c = 0; c < 64; c += 2)
                        mx[(c >> 1) & 3] = max3(mx[(c >> 1) & 3], __uint_as_float(s[hh][c]), __uint_as_float(s[hh][c + 1]));
                }
                const float m_new = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * p.scale_log2;   // the scale is positive
                const bool grow = m_new > m + kPromptRescale || (m == -INFINITY && m_new > m);
                if (__any_sync(0xffffffffu, grow)) {
                    const float a = grow ? ex2f(m - m_new) : 1.f;              // a row that has seen nothing: 0
                    if (i > u.tile_begin) {
                        // P V of the tile before has to be complete; the next one waits for this warp
                        ok = prompt_wait(bar_o(x), (uint32_t)(cs - 1) & 1u, sm_abort);
                        if (!ok) break;
                        umma::fence_after_thread_sync();
#pragma unroll
                        for (int c = 0; c < D; c += 32) {
                            uint32_t o[32];
                            umma::ld32(oc + c, o);
                            umma::wait_ld();
#pragma unroll
                            for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * a);
                            umma::st32(oc + c, o);
                        }
                    }
                    l *= a;
                    if (grow) m = m_new;
                }
                const float ref = m == -INFINITY ? 0.f : m;                    // nothing seen yet: every p is 2^-inf = 0
                const uint64_t scale2 = pack2(p.scale_log2, p.scale_log2), ref2 = pack2(-ref, -ref);
                uint64_t sum[2] = {0, 0};
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    uint32_t w[16];
#pragma unroll
                    for (int c = 0; c < 16; ++c) {
                        const uint32_t* const v = &s[q >> 1][(q & 1) * 32 + 2 * c];
                        float p0, p1;
                        unpack2(fma2(pack2(__uint_as_float(v[0]), __uint_as_float(v[1])), scale2, ref2), p0, p1);
                        p0 = ex2f(p0);
                        p1 = ex2f(p1);
                        sum[c & 1] = add2(sum[c & 1], pack2(p0, p1));
                        w[c] = In16<F16>::pack(p0, p1);
                    }
                    umma::st16(sc + q * 16, w);
                    if (q >= 2) {
                        // P V may start on the first 96 tokens, then on the rest: what follows the last weight is short
                        umma::wait_st();
                        umma::fence_before_thread_sync();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(bar_p(x, q - 2));
                    }
                }
                float l0, l1;
                unpack2(add2(sum[0], sum[1]), l0, l1);
                l += l0 + l1;
            }
            if (!ok) break;
            const PromptUnit done = u;
            for (++ui; ui < uend; ++ui) {
                u = p.units[ui];
                if (in_unit(u)) break;
            }
            ok = prompt_wait(bar_o(x), (uint32_t)(cs - 1) & 1u, sm_abort);
            if (!ok) break;
            umma::fence_after_thread_sync();
            const bool stale = __ldg(p.seq_lens + done.seq) != done.seq_len;   // stale plan: void the result, report it
            if (stale && r == 0) record_status(p.status, DA_ERR_STALE_PLAN);
            if (stale) {
                m = -INFINITY;
                l = 0.f;
            }
            // Out by way of shared memory, 128 bytes of every row at a time, so that the warp stores whole lines.  `to`: the
            // thread's row, counted from the unit's first, of out (rows of D values) or of the record; -1: none.
            const bool rec = done.slot >= 0;
            const int to = !valid ? -1 : rec ? x * kPromptRows + r : (x * TQ + tok) * p.num_q_heads + h;
            const float scale = rec ? 1.f : 1.f / l;
            const bool none = l == 0.f;                                      // (of a piece: no tile of it is seen by this row)
            float* const recs = p.ws + (int64_t)(rec ? done.slot : 0) * (kPromptTiles * kPromptRows * (D + 2));
            const int64_t row0 = (int64_t)done.row * p.num_q_heads + done.kv_head * G;
            const int kind = rec ? 0 : p.out_kind;                             // 0: fp32, 32 columns are 128 bytes; else 64 columns
            char* const dst = rec ? reinterpret_cast<char*>(recs) : static_cast<char*>(p.out) + row0 * (D * (kind == 0 ? 4 : 2));
            uint8_t* const stage = gbase + (stage_base - base) + warp * (32 * 128);
            const int row_bytes = D * (kind == 0 ? 4 : 2);
            auto send = [&](int chunk) {                                       // the staged 128 bytes of every row of the warp
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int rr = i * 4 + (lane >> 3), c = lane & 7;
                    const int at = __shfl_sync(0xffffffffu, to, rr);
                    const uint4 v = *reinterpret_cast<const uint4*>(stage + rr * 128 + ((c ^ (rr & 7)) << 4));
                    if (at >= 0) __stcg(reinterpret_cast<uint4*>(dst + (int64_t)at * row_bytes + chunk * 128) + c, v);
                }
                __syncwarp();
            };
#pragma unroll
            for (int c0 = 0; c0 < D; c0 += 64) {
                uint32_t o[64];
                umma::ld64(oc + c0, o);
                umma::wait_ld();
                if (c0 + 64 == D) {
                    umma::fence_before_thread_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar_of(x));                     // the next unit may write O
                }
#pragma unroll
                for (int k = 0; k < 64; ++k) o[k] = none ? 0u : __float_as_uint(__uint_as_float(o[k]) * scale);
                uint4* const mine = reinterpret_cast<uint4*>(stage + lane * 128);
                if (kind == 0) {
#pragma unroll
                    for (int hh = 0; hh < 2; ++hh) {
#pragma unroll
                        for (int c = 0; c < 8; ++c)
                            mine[c ^ (lane & 7)] = make_uint4(o[32 * hh + 4 * c], o[32 * hh + 4 * c + 1], o[32 * hh + 4 * c + 2], o[32 * hh + 4 * c + 3]);
                        send(c0 / 32 + hh);
                    }
                } else {
                    uint32_t w[32];
#pragma unroll
                    for (int c = 0; c < 32; ++c) {
                        const float a = __uint_as_float(o[2 * c]), b = __uint_as_float(o[2 * c + 1]);
                        w[c] = kind == 1 ? In16<false>::pack(a, b) : In16<true>::pack(a, b);
                    }
#pragma unroll
                    for (int c = 0; c < 8; ++c) mine[c ^ (lane & 7)] = make_uint4(w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]);
                    send(c0 / 64);
                }
            }
            if (valid) {
                if (rec)
                    __stcg(reinterpret_cast<float2*>(recs + kPromptTiles * kPromptRows * D) + x * kPromptRows + r, make_float2(m, l));
                else if (p.lse != nullptr)
                    p.lse[row0 + to] = none ? -INFINITY : (m + log2f(l)) * kLn2;
            }
        }
    }
    umma::fence_before_thread_sync();
    __syncthreads();
    umma::fence_after_thread_sync();
    if (tid == 0 && *sm_abort != 0) record_status(p.status, DA_ERR_TIMEOUT);
    pdl_launch_dependents();
    if (warp == kPromptMmaWarp) umma::tmem_dealloc(tmem, 512);
}

// Merge of the pieces of a cut unit: one thread per four output columns of a row, pieces in order.
template <int D>
__global__ void __launch_bounds__(256) decode_attn_prompt_merge_kernel(const PromptParams p)
{
    pdl_launch_dependents();
    constexpr int D4 = D / 4, BLOCKS = kPromptTiles * kPromptRows * D4 / 256;
    const PromptUnit u = p.units[__ldg(p.merges + blockIdx.x / BLOCKS)];
    const int i = (blockIdx.x % BLOCKS) * 256 + threadIdx.x;
    const int row = i / D4, d4 = i % D4, x = row / kPromptRows, r = row % kPromptRows;
    const int tok = r / p.group, h = r - tok * p.group;
    pdl_wait_primary();
    if (tok >= p.tokens_per_tile || x * p.tokens_per_tile + tok >= u.n_tok) return;
    constexpr int64_t RF = (int64_t)kPromptTiles * kPromptRows * (D + 2);
    const float* const rec = p.ws + (int64_t)u.slot * RF;
    const float2* const ml = reinterpret_cast<const float2*>(rec + kPromptTiles * kPromptRows * D) + row;
    const float4* const col = reinterpret_cast<const float4*>(rec) + row * D4 + d4;
    // (the first two pieces - most cut units have no more - are asked for together)
    const float2 s0 = __ldcg(ml), s1 = __ldcg(ml + RF / 2);
    const float4 v0 = __ldcg(col), v1 = __ldcg(col + RF / 4);
    float M = fmaxf(s0.x, s1.x);
    for (int k = 2; k < u.n_pieces; ++k) M = fmaxf(M, __ldcg(ml + k * (RF / 2)).x);
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float ls = 0.f;
    auto add = [&](const float2& s, const float4& v) {
        const float w = M == -INFINITY ? 1.f : ex2f(s.x - M);     // nothing seen: zeros; no number in q: none in the sum
        acc.x = fmaf(w, v.x, acc.x);
        acc.y = fmaf(w, v.y, acc.y);
        acc.z = fmaf(w, v.z, acc.z);
        acc.w = fmaf(w, v.w, acc.w);
        ls = fmaf(w, s.y, ls);
    };
    add(s0, v0);
    add(s1, v1);
    for (int k = 2; k < u.n_pieces; ++k) add(__ldcg(ml + k * (RF / 2)), __ldcg(col + k * (RF / 4)));
    const float inv = ls == 0.f ? 0.f : 1.f / ls;
    acc.x *= inv; acc.y *= inv; acc.z *= inv; acc.w *= inv;
    const int64_t orow = (int64_t)(u.row + x * p.tokens_per_tile + tok) * p.num_q_heads + u.kv_head * p.group + h;
    store_out4(p.out, orow * D + d4 * 4, acc, p.out_kind);
    if (p.lse != nullptr && d4 == 0) p.lse[orow] = ls == 0.f ? -INFINITY : (M + log2f(ls)) * kLn2;
}

}  // namespace da
