// Split-KV partial kernel over a cache held in 4 bits (packed.h).
//
// The plan is that of the 16-bit kernel: a block walks its range of the work list, a unit being one sequence, one KV head
// and a run of 16-token tiles; its result goes to `out` or to a record of the workspace in the same format, and the
// combine kernel and the merge blocks of fused launches are shared.  What differs is what a byte costs: a token and KV head
// are 144 bytes at head_dim 128 instead of 512, so at the same DRAM rate 3.6 times as many values have to be unpacked and
// multiplied, and the kernel is bound by issued instructions as much as by memory: 263 of them a tile and warp, issued at
// 0.62 a cycle and scheduler, of which the conversions from e2m1 and the half-precision products take a pipe two cycles each.
// (At head_dim 128 these include spills: 64 to 80 bytes a thread stored and 44 to 52 loaded, more in the forms for windows and for groups
// of more than 8, up to 444 and 292.)
// 64 sequences of 28,000 to 32,768 tokens, 32 / 8 heads of 128: 2.2 GB in 372 us, 5.96 TB/s (405 to 450 us where the same step
// runs without a pause and the power limit lowers the clock).
//
// A block is W warps, 4 or 8.  Every warp has a ring of its own and works in steps of two tiles (32 tokens): step w of
// a unit belongs to warp w mod W.  Its lanes copy a step's tiles (cp.async, 16 bytes a lane, contiguous in the pool) as soon
// as the warp is done with the step that lay there, across the ends of units.  (Bulk copies cost more here: one takes its
// operands from uniform registers, and two lanes issuing one each are two passes through some thirty instructions.)  No
// warp waits for another but at the end of a unit, where the partial states of its warps are merged.
//
//   S^T[16 x 8] = sum over blocks b of 32 dims:  k_scale[16, b] * (K codes[16 x 32] . Q^T[32 x 8])
//   O^T[D x 8] += (V codes * v_scale)^T[D x 16] . P^T[16 x 8]
//
// by mma.sync m16n8k16 in fp16 with fp32 sums.  Codes are exact in fp16; a lane's K words hold dims of one block at a time, so the
// K scale multiplies fp32 sums (two mma, four multiplications).  For V the scale varies along the sum, so it goes onto the
// operand: a pair of tokens' codes times their pair of scales, rounded to fp16 (half a step of 2^-11).  A lane's V operand wants
// pairs of tokens of one dim while bytes hold pairs of dims of one token: words of two tokens are interleaved by nibbles
// ahead of the conversion, half an instruction per pair.  Queries are brought to a largest magnitude in [1, 2) by a power of two
// so that bf16 values fit fp16's range: exact, but for dims below 2^-14 of the head's largest, which are subnormal there and off by
// up to 2^-25 of it (bf16 ones from 2^-17 on).  Next to the largest dim these matter only where K is that much larger in them.
//
// Softmax runs on the accumulators in fp32, base 2.  The running maximum of a head is renewed only when a logit runs more
// than 8 above it (weights stay below 2^8, representable with the same relative step), so that most steps need no
// exchange between lanes but one vote.  Weights are rounded once to fp16; when inputs are fp16 (and so, as a rule, the
// output) they keep a second part, p - fp16(p): in columns 4 to 7 for groups of up to 4 heads (DUP: the query is there twice),
// in a second mma for larger ones.
#pragma once

#include <type_traits>

#include "common.cuh"
#include "packed.cuh"

namespace da {

// W: warps of a block; NT: 8-column tiles of query heads, 2 for groups of more than 8.
template <int D, int W, int NT>
struct PackedCfg {
    static constexpr int kThreads = 32 * W;
    static constexpr int kBlocks = (NT == 1 ? 16 : 12) / W;   // on an SM: 128 registers a thread, or 168
    static constexpr int kTile = packed_tile_bytes(D);
    static constexpr int kStep = 2 * kTile;                   // what a warp takes at a time: two tiles
    static constexpr int kStages = D == 128 ? 2 : 4;          // steps in the ring of a warp
    static constexpr int kScratchOff = W * kStages * kStep;
    static constexpr int kCols = 4;                            // heads that meet in the scratch at a time
    static constexpr int kScratch = W * kCols * D * 4 + 2 * W * kCols * 4;
    static constexpr int kQOff = kScratchOff + kScratch;       // NT 2: Q^T as B operands, then what logits are multiplied with
    static constexpr int kQ = NT == 1 ? 0 : (D / 32) * NT * 32 * 16 + NT * 8 * 4;
    static constexpr int kSmem = (kQOff + kQ + 15) / 16 * 16;
    static_assert(kScratchOff % 128 == 0 && kScratch % 16 == 0 && kTile % 128 == 0, "shared memory layout");
};

__device__ __forceinline__ void copy_16(uint32_t dst, const void* src, uint64_t l2_policy)
{
    asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "l"(l2_policy) : "memory");
}

// Hints to L2: nothing to wait for.
__device__ __forceinline__ void prefetch_tile(const void* src, uint32_t bytes)
{
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(src), "r"(bytes) : "memory");
}

__device__ __forceinline__ void prefetch_line(const void* src) { asm volatile("prefetch.global.L2 [%0];" ::"l"(src) : "memory"); }

__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }

template <int N>
__device__ __forceinline__ void copy_wait()
{
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

__device__ __forceinline__ uint64_t packed_l2_policy()
{
    uint64_t pol;
    asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(pol));
    return pol;
}

// The product alone, and added to c.
__device__ __forceinline__ void packed_mma0(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}

__device__ __forceinline__ void packed_mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t packed_transpose(uint32_t a)
{
    uint32_t d;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}

__device__ __forceinline__ uint32_t half2_mul(uint32_t a, uint32_t b)
{
    const __half2 r = __hmul2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&r);
}

template <int N>
__device__ __forceinline__ void lds_words(uint32_t addr, uint32_t (&w)[N])
{
    static_assert(N == 1 || N == 2 || N == 4, "one load");
    if (N == 4)
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1 % N]), "=r"(w[2 % N]), "=r"(w[3 % N]) : "r"(addr));
    else if (N == 2)
        asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1 % N]) : "r"(addr));
    else
        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[0]) : "r"(addr));
}

// DUP: fp16 inputs, groups of up to 4; EXT: windowed plans.
template <int D, bool F16, bool DUP, bool EXT, int W, int NT>
__global__ void __launch_bounds__(32 * W, PackedCfg<D, W, NT>::kBlocks) decode_attn_packed_kernel(const KernelParams p, const int G)
{
    using Cfg = PackedCfg<D, W, NT>;
    constexpr int NB = D / 32;                                // blocks of 32 dims: K words of a lane and row
    constexpr int NW = D / 64;                                // V words of a lane and token
    constexpr int NS = Cfg::kStages;
    constexpr int MT = D / 16;                                // 16-row tiles of O^T
    constexpr bool LOW = F16 && !DUP;                         // the weights' second part takes an mma of its own
    static_assert((F16 && NT == 1) || !DUP, "duplicated columns: small groups of fp16");
    extern __shared__ __align__(128) uint8_t smem[];
    const uint32_t base = smem_u32(smem);
    float* const sm_wo = reinterpret_cast<float*>(smem + Cfg::kScratchOff);      // [W][kCols][D]
    float* const sm_wm = sm_wo + W * Cfg::kCols * D;                              // [W][kCols]
    float* const sm_wl = sm_wm + W * Cfg::kCols;
    __shared__ int sm_flag;                                   // of merge blocks

    if (p.fused && (int)blockIdx.x >= p.n_work_blocks) {
        pdl_launch_dependents();
        pdl_wait_primary();
        fused_merge_blocks<D>(p, G, Cfg::kThreads, sm_wo, &sm_flag);
        return;
    }
    const int ubeg = __ldg(p.block_begin + blockIdx.x), uend = __ldg(p.block_begin + blockIdx.x + 1);
    if (ubeg >= uend) {                                       // a surplus block of a capacity launch
        if (blockIdx.x == 0) pdl_wait_primary();
        return;
    }
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int g = lane >> 2, t = lane & 3;                    // mma row / column group, and lane within it
    const uint32_t ring = base + warp * NS * Cfg::kStep;
    const uint32_t q_at = base + Cfg::kQOff + lane * 16;
    float* const sm_mult = reinterpret_cast<float*>(smem + Cfg::kQOff + NB * NT * 32 * 16);          // [NT][8]
    decode_attn_unit_t u = load_unit(p.units, ubeg);
    {
        // Hints, while the kernel before this one drains: the tiles of every warp's first steps and the lines that its
        // critical path reads are asked into L2.  What is read for it here may be about to change; it steers prefetches only
        // and is read again behind the wait.
        const WindowCut cut = EXT ? window_cut(u.seq_len, p.window, p.sinks) : WindowCut{0, 0, 0};
        const int tile = 2 * (warp + W * (lane >> 1)) + (lane & 1), at = (u.tok_begin >> 4) + tile;
        const bool masked = p.run_mask != nullptr && __ldcg(p.run_mask + u.seq) == 0;
        if (!masked && lane < 2 * NS && tile < (u.tok_end - u.tok_begin + 15) >> 4) {
            const int where = EXT ? window_tile(cut, at) : at;
            const int page = __ldcg(p.block_table + (int64_t)u.seq * p.max_pages_per_seq + (where >> p.tile_shift));
            if ((unsigned)page < (unsigned)p.num_pages)
                prefetch_tile(reinterpret_cast<const char*>(p.k) + page * p.k_stride_page + u.kv_head * p.k_stride_head +
                                  (where & ((1 << p.tile_shift) - 1)) * Cfg::kTile, Cfg::kTile);
        }
        if (warp == 0 && lane * 128 < G * D * 2)
            prefetch_line(reinterpret_cast<const char*>(p.q + ((int64_t)u.seq * p.num_q_heads + u.kv_head * G) * D) + lane * 128);
        if (warp == 1 && lane == 31) prefetch_line(p.seq_lens + u.seq);
    }
    pdl_wait_primary();
    // (What the kernels before may have written is read by ordinary loads: the wait makes their writes visible to those.)

    auto cut_of = [&](const decode_attn_unit_t& x) { return EXT ? window_cut(x.seq_len, p.window, p.sinks) : WindowCut{0, 0, 0}; };
    // tiles of a unit that this launch reads
    auto tiles_of = [&](const decode_attn_unit_t& x) {
        if (p.run_mask != nullptr && p.run_mask[x.seq] == 0) return 0;
        return (x.tok_end - x.tok_begin + 15) >> 4;
    };

    // ------------------------------------------------------------ asking for steps
    const uint64_t l2_policy = packed_l2_policy();
    // of unit iu, this warp's step ij comes next, into stage `slot` of its ring
    int iu = ubeg, ij = 0;
    uint32_t slot = ring + lane * 16;
    int i_tiles = tiles_of(u), i_tile0 = u.tok_begin >> 4;
    const char* i_pool = reinterpret_cast<const char*>(p.k) + u.kv_head * p.k_stride_head + lane * 16;
    const int32_t* i_row = p.block_table + (int64_t)u.seq * p.max_pages_per_seq;
    WindowCut i_cut = cut_of(u);
    // lane l: where tile l % 2 of step ij / 16 * 16 + l / 2 lies in the pool (pages outside it are reported and none read)
    int64_t i_where = 0;
    auto take_ids = [&]() {
        const int tile = 2 * (warp + W * (ij + (lane >> 1))) + (lane & 1);
        i_where = 0;
        if (tile < i_tiles) {
            const int at = EXT ? window_tile(i_cut, i_tile0 + tile) : i_tile0 + tile;
            int page = i_row[at >> p.tile_shift];
            if ((unsigned)page >= (unsigned)p.num_pages) {
                record_status(p.status, DA_ERR_BAD_PAGE);
                page = 0;
            }
            i_where = page * p.k_stride_page + (at & ((1 << p.tile_shift) - 1)) * Cfg::kTile;
        }
    };
    take_ids();
    auto ask = [&]() {
        while (iu < uend && 2 * (warp + W * ij) >= i_tiles) {
            if (++iu < uend) {
                const decode_attn_unit_t x = load_unit(p.units, iu);
                i_tiles = tiles_of(x);
                i_tile0 = x.tok_begin >> 4;
                i_pool = reinterpret_cast<const char*>(p.k) + x.kv_head * p.k_stride_head + lane * 16;
                i_row = p.block_table + (int64_t)x.seq * p.max_pages_per_seq;
                i_cut = cut_of(x);
                ij = 0;
                take_ids();
            }
        }
        if (iu < uend) {
            if (ij != 0 && (ij & 15) == 0) take_ids();
            const bool second = 2 * (warp + W * ij) + 1 < i_tiles;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const char* const src = i_pool + __shfl_sync(0xffffffffu, i_where, (2 * ij + i) & 31);
                if (i == 1 && !second) break;
                constexpr int kWhole = Cfg::kTile / 512;
#pragma unroll
                for (int c = 0; c < kWhole; ++c) copy_16(slot + i * Cfg::kTile + c * 512, src + c * 512, l2_policy);
                if (lane * 16 < Cfg::kTile % 512) copy_16(slot + i * Cfg::kTile + kWhole * 512, src + kWhole * 512, l2_policy);
            }
        }
        copy_commit();                                        // (a group for every call: the waits below count them)
        ++ij;
        slot += Cfg::kStep;
        if (slot >= ring + NS * Cfg::kStep) slot -= NS * Cfg::kStep;
    };
    for (int s = 0; s < NS; ++s) ask();

    // The lane's rows of a tile: k index 2 t' + e (+ 8) of the mma is token 4 t' + ((2 h + e) ^ t'), so that the four tokens
    // of a lane as a column of V are neighbours and no load of K, V or scales has a bank conflict.
    const int gt = g >> 1, ge = g & 1;
    const int row_a = 4 * gt + (ge ^ gt), row_b = 4 * gt + ((2 + ge) ^ gt);
    const uint32_t k_off = row_a * (D / 2) + t * (D / 8), ks_off = packed_k_scales(D) + row_a * NB * 2;
    const uint32_t k_two = (row_b - row_a) * (D / 2), ks_two = (row_b - row_a) * NB * 2;
    const uint32_t vs_off = packed_v_scales(D) + (g * (D / 8) / 32) * 32 + 8 * t;
    uint32_t v_off[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
        v_off[j] = packed_v_codes(D) + (4 * t + (j ^ t)) * (D / 2) + (D == 128 ? (8 * g) ^ (32 * (t >> 1)) : 4 * g);
    uint32_t at = ring;                                       // the step that is worked on

    // a head's query, 8 dims of every block of 32 to a lane (NT 2: this warp's of the two tiles)
    const int q_head = DUP ? (g & 3) : NT == 1 ? g : (warp & 1) * 8 + g;
    auto load_q = [&](const decode_attn_unit_t& x, uint4 (&w)[NB]) {
        const bool live = q_head < G;
        const uint4* const row = reinterpret_cast<const uint4*>(p.q + ((int64_t)x.seq * p.num_q_heads + x.kv_head * G + (live ? q_head : 0)) * D);
#pragma unroll
        for (int b = 0; b < NB; ++b) w[b] = live ? row[4 * b + t] : make_uint4(0, 0, 0, 0);
    };
    uint4 q_raw[NB];
    load_q(u, q_raw);
    int dev_len = p.seq_lens[u.seq];

    for (int uid = ubeg; uid < uend; ++uid) {
        const bool last_unit = uid + 1 >= uend;
        const int n_tiles = tiles_of(u);
        const int tok_begin = u.tok_begin, tok_end = u.tok_end;
        const WindowCut cut = cut_of(u);
        const bool stale = dev_len != u.seq_len;
        if (n_tiles == 0) {
            if (last_unit) pdl_launch_dependents();
            if (stale && tid == 0) record_status(p.status, DA_ERR_STALE_PLAN);
            block_finish_empty<D>(p, u, G, tid, Cfg::kThreads);
            if (!last_unit) {
                u = load_unit(p.units, uid + 1);
                load_q(u, q_raw);
                dev_len = p.seq_lens[u.seq];
            }
            continue;
        }
        // ---- Q^T as B operands, every head's largest magnitude brought to [1, 2); mult: what a logit is multiplied with
        uint32_t qb[NB][4];                                   // (NT 2: prepared here, read from shared memory)
        float mult[NT][2];
        {
            float amax = 0.f;
            float2 f[NB][4];
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const uint32_t x[4] = {q_raw[b].x, q_raw[b].y, q_raw[b].z, q_raw[b].w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    f[b][i] = F16 ? __half22float2(*reinterpret_cast<const __half2*>(&x[i]))
                                  : make_float2(__uint_as_float(x[i] << 16), __uint_as_float(x[i] & 0xffff0000u));
                    amax = fmaxf(amax, fmaxf(fabsf(f[b][i].x), fabsf(f[b][i].y)));
                }
            }
            amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
            amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
            int e = (int)(__float_as_uint(amax) >> 23) - 127;                         // (zero: -127, infinite: 128)
            e = amax > 0.f ? min(max(e, -126), 126) : 0;
            const float down = __uint_as_float((uint32_t)(127 - e) << 23), up = __uint_as_float((uint32_t)(127 + e) << 23);
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const __half2 h = __floats2half2_rn(f[b][i].x * down, f[b][i].y * down);
                    qb[b][i] = *reinterpret_cast<const uint32_t*>(&h);
                }
            const float own = p.scale_log2 * up;              // of column g; the accumulators hold columns 2 t, 2 t + 1
            if (NT == 1) {
                mult[0][0] = __shfl_sync(0xffffffffu, own, 8 * t);
                mult[0][1] = __shfl_sync(0xffffffffu, own, 8 * t + 4);
            } else {
                // (the barriers at the end of the unit before say that everybody is done with its queries)
                if (warp < NT) {
#pragma unroll
                    for (int b = 0; b < NB; ++b)
                        *reinterpret_cast<uint4*>(smem + Cfg::kQOff + ((b * NT + warp) * 32 + lane) * 16) = make_uint4(qb[b][0], qb[b][1], qb[b][2], qb[b][3]);
                    if (t == 0) sm_mult[warp * 8 + g] = own;
                }
                block_sync(1, Cfg::kThreads);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    mult[nt][0] = sm_mult[nt * 8 + 2 * t];
                    mult[nt][1] = sm_mult[nt * 8 + 2 * t + 1];
                }
            }
        }
        float oacc[MT][NT][4], m_run[NT][2], l_run[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            m_run[nt][0] = m_run[nt][1] = -INFINITY;
            l_run[nt][0] = l_run[nt][1] = 0.f;
#pragma unroll
            for (int i = 0; i < MT; ++i) oacc[i][nt][0] = oacc[i][nt][1] = oacc[i][nt][2] = oacc[i][nt][3] = 0.f;
        }
        for (int tile0 = 2 * warp; tile0 < n_tiles; tile0 += 2 * W) {
            copy_wait<NS - 1>();
            __syncwarp();                                     // every lane's copies of the step are there
            const int tok0 = tok_begin + tile0 * 16;
            const int left = tok_end - tok0;                  // tokens of the unit from here on
            // Rows of tile i that are seen are [0, hide0) and [hide1, left - 16 i).  A step at neither the unit's end nor a gap
            // sees all: it takes a form of its own without masks (they cost it a fifth of its instructions).
            bool whole = left >= 32;
            int hide0[2] = {16, 16}, hide1[2] = {0, 0};
            if (EXT) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int pos = window_tile(cut, (tok0 >> 4) + i) << 4;
                    hide0[i] = min(max(p.sinks - pos, 0), 16);
                    hide1[i] = max(cut.first - pos, 0);
                    if (hide0[i] < min(hide1[i], 16)) whole = false;
                }
            }
            auto seen = [&](int i, int r) { return r < left - 16 * i && !(EXT && r >= hide0[i] && r < hide1[i]); };
            auto step = [&](auto masked) {
                constexpr bool MASKED = decltype(masked)::value;
                // ---- S^T (the second tile may not be there: what lies in its place is not used)
                float sacc[2][NT][4];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint32_t tile = at + i * Cfg::kTile;
                    uint32_t ka[NB], kb[NB], sa[NB / 2], sb[NB / 2];
                    lds_words<NB>(tile + k_off, ka);
                    lds_words<NB>(tile + k_off + k_two, kb);
                    lds_words<NB / 2>(tile + ks_off, sa);
                    lds_words<NB / 2>(tile + ks_off + ks_two, sb);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) sacc[i][nt][0] = sacc[i][nt][1] = sacc[i][nt][2] = sacc[i][nt][3] = 0.f;
#pragma unroll
                    for (int b = 0; b < NB; ++b) {
                        uint32_t ha[4], hb[4];
                        packed_unpack(ka[b], ha);
                        packed_unpack(kb[b], hb);
                        const __half2 xa = *reinterpret_cast<const __half2*>(&sa[b / 2]), xb = *reinterpret_cast<const __half2*>(&sb[b / 2]);
                        const float fa = b & 1 ? __high2float(xa) : __low2float(xa), fb = b & 1 ? __high2float(xb) : __low2float(xb);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            uint32_t q[4];
                            if (NT > 1) {
                                lds_words<4>(q_at + (b * NT + nt) * 512, q);
                            } else {
#pragma unroll
                                for (int k = 0; k < 4; ++k) q[k] = qb[b][k];
                            }
                            float c[4];
                            packed_mma0(c, ha[0], hb[0], ha[1], hb[1], q[0], q[1]);
                            packed_mma(c, ha[2], hb[2], ha[3], hb[3], q[2], q[3]);
                            sacc[i][nt][0] = fmaf(c[0], fa, sacc[i][nt][0]);
                            sacc[i][nt][1] = fmaf(c[1], fa, sacc[i][nt][1]);
                            sacc[i][nt][2] = fmaf(c[2], fb, sacc[i][nt][2]);
                            sacc[i][nt][3] = fmaf(c[3], fb, sacc[i][nt][3]);
                        }
                    }
                }
                // ---- softmax: rows (tokens) row_a, row_b of each tile, columns (heads) 2 t, 2 t + 1
                if (MASKED) {
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                if (!seen(i, k < 2 ? row_a : row_b)) sacc[i][nt][k] = -INFINITY;
                }
                float top[NT][2];
                bool ahead = false;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        top[nt][k] = fmaxf(fmaxf(sacc[0][nt][k], sacc[0][nt][k + 2]), fmaxf(sacc[1][nt][k], sacc[1][nt][k + 2])) * mult[nt][k];
                        ahead |= top[nt][k] > m_run[nt][k] + 8.f;
                    }
                if (__any_sync(0xffffffffu, ahead)) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
#pragma unroll
                            for (int off = 4; off <= 16; off <<= 1) top[nt][k] = fmaxf(top[nt][k], __shfl_xor_sync(0xffffffffu, top[nt][k], off));
                            const float m = fmaxf(m_run[nt][k], top[nt][k]), al = ex2f(m_run[nt][k] - m);
                            m_run[nt][k] = m;
                            l_run[nt][k] *= al;
#pragma unroll
                            for (int r = 0; r < MT; ++r) {
                                oacc[r][nt][k] *= al;
                                oacc[r][nt][k + 2] *= al;
                            }
                        }
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if (MASKED && i == 1 && left <= 16) break;
                    const uint32_t tile = at + i * Cfg::kTile;
                    uint32_t pb[NT][2], pl[NT][2];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const float p0 = ex2f(fmaf(sacc[i][nt][2 * h], mult[nt][0], -m_run[nt][0]));
                            const float p1 = ex2f(fmaf(sacc[i][nt][2 * h + 1], mult[nt][1], -m_run[nt][1]));
                            l_run[nt][0] += p0;
                            l_run[nt][1] += p1;
                            __half2 x = __floats2half2_rn(p0, p1);
                            if (F16) {
                                const float2 y = __half22float2(x);
                                const __half2 z = __floats2half2_rn(p0 - y.x, p1 - y.y);
                                if (DUP) {
                                    if (t >= 2) x = z;
                                } else {
                                    pl[nt][h] = packed_transpose(*reinterpret_cast<const uint32_t*>(&z));
                                }
                            }
                            pb[nt][h] = packed_transpose(*reinterpret_cast<const uint32_t*>(&x));
                        }
                    // ---- O^T: the lane's tokens 4 t + (j ^ t), its dims (D / 8) g ..
                    uint32_t v[4][NW], vs[2];
                    lds_words<2>(tile + vs_off, vs);
#pragma unroll
                    for (int j = 0; j < 4; ++j) lds_words<NW>(tile + v_off[j], v[j]);
                    if (MASKED) {
                        // (codes are finite whatever the bytes hold; a scale that is not would spoil a weight of zero)
                        uint32_t keep[2] = {0, 0};
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            if (seen(i, 4 * t + (j ^ t))) keep[j >> 1] |= j & 1 ? 0xffff0000u : 0x0000ffffu;
                        vs[0] &= keep[0];
                        vs[1] &= keep[1];
                    }
#pragma unroll
                    for (int w = 0; w < NW; ++w) {
                        uint32_t l1[4], h1[4], l2[4], h2[4];
                        constexpr uint32_t kLow = 0x0f0f0f0fu;
                        packed_unpack((v[0][w] & kLow) | ((v[1][w] << 4) & ~kLow), l1);
                        packed_unpack(((v[0][w] >> 4) & kLow) | (v[1][w] & ~kLow), h1);
                        packed_unpack((v[2][w] & kLow) | ((v[3][w] << 4) & ~kLow), l2);
                        packed_unpack(((v[2][w] >> 4) & kLow) | (v[3][w] & ~kLow), h2);
#pragma unroll
                        for (int m = 0; m < 4; ++m) {
                            const uint32_t a0 = half2_mul(l1[m], vs[0]), a1 = half2_mul(h1[m], vs[0]);
                            const uint32_t a2 = half2_mul(l2[m], vs[1]), a3 = half2_mul(h2[m], vs[1]);
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) {
                                packed_mma(oacc[4 * w + m][nt], a0, a1, a2, a3, pb[nt][0], pb[nt][1]);
                                if (LOW) packed_mma(oacc[4 * w + m][nt], a0, a1, a2, a3, pl[nt][0], pl[nt][1]);
                            }
                        }
                    }
                }
            };
            if (whole)
                step(std::false_type{});
            else
                step(std::true_type{});
            __syncwarp();                                     // every lane has read the step
            at += Cfg::kStep;
            if (at >= ring + NS * Cfg::kStep) at = ring;
            ask();
        }
        if (last_unit) pdl_launch_dependents();
        // (read again rather than kept in registers: the line is in L1)
        const decode_attn_unit_t done = load_unit(p.units, uid);
        if (!last_unit) {                                     // in flight during this unit's end
            u = load_unit(p.units, uid + 1);
            load_q(u, q_raw);
            dev_len = p.seq_lens[u.seq];
        }

        // ------------------------------------------------------------ end of the unit
        if (stale && tid == 0) record_status(p.status, DA_ERR_STALE_PLAN);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int off = 4; off <= 16; off <<= 1) {
                l_run[nt][0] += __shfl_xor_sync(0xffffffffu, l_run[nt][0], off);
                l_run[nt][1] += __shfl_xor_sync(0xffffffffu, l_run[nt][1], off);
            }
            if (stale) {
                m_run[nt][0] = m_run[nt][1] = -INFINITY;
                l_run[nt][0] = l_run[nt][1] = 0.f;
            }
        }
        if (DUP) {                                            // columns 4 to 7 carried the second parts of heads 0 to 3
#pragma unroll
            for (int r = 0; r < MT; ++r)
#pragma unroll
                for (int k = 0; k < 4; ++k) oacc[r][0][k] += __shfl_down_sync(0xffffffffu, oacc[r][0][k], 2);
        }
#pragma unroll
        for (int q = 0; q < (DUP ? 1 : 2 * NT); ++q) {         // four heads at a time
            if (4 * q >= G) break;
            const int nt = q >> 1;
            block_sync(1, Cfg::kThreads);                     // the scratch is free
            if ((t >> 1) == (q & 1)) {
                const int lc = 2 * (t & 1);
                if (g == 0) {
                    sm_wm[warp * Cfg::kCols + lc] = m_run[nt][0];
                    sm_wm[warp * Cfg::kCols + lc + 1] = m_run[nt][1];
                    sm_wl[warp * Cfg::kCols + lc] = l_run[nt][0];
                    sm_wl[warp * Cfg::kCols + lc + 1] = l_run[nt][1];
                }
                float* const wo = sm_wo + (warp * Cfg::kCols + lc) * D + g * (D / 8);
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    *reinterpret_cast<float2*>(wo + 2 * i) = make_float2(oacc[i][nt][0], oacc[i][nt][2]);
                    *reinterpret_cast<float2*>(wo + D + 2 * i) = make_float2(oacc[i][nt][1], oacc[i][nt][3]);
                }
            }
            block_sync(1, Cfg::kThreads);
            block_finish<D, W, Cfg::kCols, false, W>(p, done, G, sm_wo, sm_wm, sm_wl, tid, Cfg::kThreads, 1, 4 * q, min(4, G - 4 * q),
                                                  DUP || 4 * (q + 1) >= G);
        }
    }
}

}  // namespace da
