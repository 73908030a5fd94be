// Split-KV partial kernel over a cache held in 4 bits (packed.h).
//
// The plan is that of the 16-bit kernel: a block walks its range of the work list, a unit being one sequence, one KV head
// and a run of 16-token tiles; its result goes to `out` or to a record of the workspace in the same format, and the
// combine kernel and the merge blocks of fused launches are shared.  What differs is what a byte costs: a token and KV head
// are 144 bytes at head_dim 128 instead of 512, so at the same DRAM rate 3.6 times as many values have to be unpacked and
// multiplied, and the kernel is bound by issued instructions as much as by memory.
//
// Eight warps to a block, each with a ring of tiles of its own: lane 0 asks for a tile (one bulk copy, contiguous in the
// pool) as soon as the warp is done with the one that lay there, kStages tiles ahead, across the ends of units.  Tile t of a unit belongs to warp t mod
// 8.  No warp waits for another but at the end of a unit, where the eight partial states are merged.
//
//   S^T[16 x 8] = sum over blocks b of 32 dims:  k_scale[16, b] * (K codes[16 x 32] . Q^T[32 x 8])
//   O^T[D x 8] += (V codes * v_scale)^T[D x 16] . P^T[16 x 8]
//
// by mma.sync m16n8k16 in fp16 with fp32 sums.  Codes are exact in fp16; a lane's K words hold dims of one block at a time, so the
// K scale multiplies fp32 sums (two mma, four multiplications).  For V the scale varies along the sum, so it goes onto the
// operand: a pair of tokens' codes times their pair of scales, rounded to fp16 (half a step of 2^-11).  A lane's V operand wants
// pairs of tokens of one dim while bytes hold pairs of dims of one token: words of two tokens are interleaved by nibbles
// ahead of the conversion, half an instruction per pair.  Queries are brought to a largest magnitude in [1, 2) by a power of two
// (exact) so that bf16 values fit fp16's range.
//
// Softmax runs on the accumulators in fp32, base 2.  The running maximum of a head is renewed only when a logit runs more
// than 8 above it (weights stay below 2^8, representable with the same relative step), so that most tiles need no
// exchange between lanes but one vote.
#pragma once

#include "common.cuh"
#include "packed.cuh"

namespace da {

constexpr int kPackedWarps = 8;
constexpr int kPackedThreads = kPackedWarps * 32;

template <int D>
struct PackedCfg {
    static constexpr int kTile = packed_tile_bytes(D);
    static constexpr int kStages = D == 128 ? 4 : 8;          // tiles in flight per warp
    static constexpr int kBarriers = kPackedWarps * kStages * 8;
    static constexpr int kScratchOff = kPackedWarps * kStages * kTile;
    static constexpr int kCols = 4;                            // heads that meet in the scratch at a time
    static constexpr int kScratch = kPackedWarps * kCols * D * 4 + 2 * kPackedWarps * kCols * 4;
    static constexpr int kFlagOff = kScratchOff + kScratch + kBarriers;
    static constexpr int kSmem = kFlagOff + 16;
    static_assert(kScratchOff % 128 == 0 && kScratch % 8 == 0 && kFlagOff % 4 == 0, "shared memory layout");
};

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar, uint64_t l2_policy)
{
    asm volatile("cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar), "l"(l2_policy)
                 : "memory");
}

__device__ __forceinline__ uint64_t packed_l2_policy()
{
    uint64_t pol;
    asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(pol));
    return pol;
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

// WIDE: groups of 9 to 16 query heads, two 8-column tiles of heads; EXT: windowed plans.
template <int D, bool F16, bool WIDE, bool EXT>
__global__ void __launch_bounds__(kPackedThreads, WIDE && D == 128 ? 1 : 2) decode_attn_packed_kernel(const KernelParams p, const int G)
{
    using Cfg = PackedCfg<D>;
    constexpr int NB = D / 32;                                // blocks of 32 dims: K words of a lane and row
    constexpr int NW = D / 64;                                // V words of a lane and token
    constexpr int NT = WIDE ? 2 : 1;                          // tiles of 8 query heads
    constexpr int NS = Cfg::kStages;
    constexpr int MT = D / 16;                                // 16-row tiles of O^T
    extern __shared__ __align__(128) uint8_t smem[];
    const uint32_t base = smem_u32(smem);
    float* const sm_wo = reinterpret_cast<float*>(smem + Cfg::kScratchOff);                  // [8][kCols][D]
    float* const sm_wm = sm_wo + kPackedWarps * Cfg::kCols * D;                               // [8][kCols]
    float* const sm_wl = sm_wm + kPackedWarps * Cfg::kCols;
    volatile int* const sm_flag = reinterpret_cast<volatile int*>(smem + Cfg::kFlagOff);

    if (p.fused && (int)blockIdx.x >= p.n_work_blocks) {
        pdl_launch_dependents();
        pdl_wait_primary();
        fused_merge_blocks<D>(p, G, kPackedThreads, sm_wo, const_cast<int*>(sm_flag));
        return;
    }
    const int ubeg = __ldg(p.block_begin + blockIdx.x), uend = __ldg(p.block_begin + blockIdx.x + 1);
    if (ubeg >= uend) {                                       // a surplus block of a capacity launch
        if (blockIdx.x == 0) pdl_wait_primary();
        return;
    }
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int g = lane >> 2, t = lane & 3;                    // mma row / column group, and lane within it
    const uint32_t ring = base + warp * NS * Cfg::kTile;
    const uint32_t bars = base + Cfg::kScratchOff + Cfg::kScratch + warp * NS * 8;
    if (lane == 0)
        for (int s = 0; s < NS; ++s) mbar_init(bars + 8 * s, 1);
    if (tid == 0) *sm_flag = 0;
    mbar_init_fence();
    __syncthreads();
    pdl_wait_primary();

    auto cut_of = [&](const decode_attn_unit_t& x) { return EXT ? window_cut(x.seq_len, p.window, p.sinks) : WindowCut{0, 0, 0}; };
    // tiles of a unit that this launch reads
    auto tiles_of = [&](const decode_attn_unit_t& x) {
        if (p.run_mask != nullptr && __ldg(p.run_mask + x.seq) == 0) return 0;
        return (x.tok_end - x.tok_begin + 15) >> 4;
    };

    // ------------------------------------------------------------ asking for tiles
    const uint64_t l2_policy = packed_l2_policy();
    const char* const pool = reinterpret_cast<const char*>(p.k);
    int iu = ubeg, in_tiles = 0, it0 = 0, ij = 0, i_ids = 0, i_issued = 0;
    decode_attn_unit_t ix = load_unit(p.units, ubeg);
    WindowCut icut = cut_of(ix);
    auto take_ids = [&]() {                                   // page ids of this warp's next 32 tiles
        const int tile = warp + kPackedWarps * (ij + lane);
        const int32_t* const row = p.block_table + (int64_t)ix.seq * p.max_pages_per_seq;
        const int at = it0 + tile;
        i_ids = tile < in_tiles ? __ldg(row + ((EXT ? window_tile(icut, at) : at) >> p.tile_shift)) : 0;
    };
    in_tiles = tiles_of(ix);
    it0 = ix.tok_begin >> 4;
    take_ids();
    auto ask = [&]() {
        while (iu < uend && warp + kPackedWarps * ij >= in_tiles) {
            if (++iu < uend) {
                ix = load_unit(p.units, iu);
                icut = cut_of(ix);
                in_tiles = tiles_of(ix);
                it0 = ix.tok_begin >> 4;
                ij = 0;
                take_ids();
            }
        }
        if (iu >= uend || p.debug_drop_loads) return;
        if (ij != 0 && (ij & 31) == 0) take_ids();
        int page = __shfl_sync(0xffffffffu, i_ids, ij & 31);
        if (lane == 0) {
            if ((unsigned)page >= (unsigned)p.num_pages) {    // nothing outside the pool is read
                record_status(p.status, DA_ERR_BAD_PAGE);
                page = 0;
            }
            const int at = it0 + warp + kPackedWarps * ij;
            const int in_page = (EXT ? window_tile(icut, at) : at) & ((1 << p.tile_shift) - 1);
            const uint32_t s = (uint32_t)i_issued % NS;
            mbar_arrive_expect_tx(bars + 8 * s, Cfg::kTile);
            bulk_load(ring + s * Cfg::kTile, pool + page * p.k_stride_page + ix.kv_head * p.k_stride_head + in_page * Cfg::kTile, Cfg::kTile,
                      bars + 8 * s, l2_policy);
        }
        ++i_issued;
        ++ij;
    };
    for (int s = 0; s < NS; ++s) ask();

    // The lane's rows of a tile: k index 2 t' + e (+ 8) of the mma is token 4 t' + ((2 h + e) ^ t'), so that the four tokens
    // of a lane as a column of V are neighbours and no load of K, V or scales has a bank conflict.
    const int gt = g >> 1, ge = g & 1;
    const int row_a = 4 * gt + (ge ^ gt), row_b = 4 * gt + ((2 + ge) ^ gt);
    uint32_t taken = 0;                                       // tiles consumed, over all units

    for (int uid = ubeg; uid < uend; ++uid) {
        const decode_attn_unit_t u = load_unit(p.units, uid);
        const bool last_unit = uid + 1 >= uend;
        const int n_tiles = tiles_of(u);
        const int dev_len = __ldg(p.seq_lens + u.seq);
        const WindowCut cut = cut_of(u);
        if (n_tiles == 0) {
            if (last_unit) pdl_launch_dependents();
            if (dev_len != u.seq_len && tid == 0) record_status(p.status, DA_ERR_STALE_PLAN);
            block_finish_empty<D>(p, u, G, tid, kPackedThreads);
            continue;
        }
        // ---- Q^T as B operands, every head's largest magnitude brought to [1, 2); mult: what a logit is multiplied with
        uint32_t qb[NB][NT][4];
        float mult[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int head = nt * 8 + g;
            const bool live = head < G;
            const uint4* const qrow = reinterpret_cast<const uint4*>(p.q + ((int64_t)u.seq * p.num_q_heads + u.kv_head * G + (live ? head : 0)) * D);
            uint4 w[NB];
            float amax = 0.f;
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                w[b] = live ? __ldg(qrow + 4 * b + t) : make_uint4(0, 0, 0, 0);       // dims 32 b + 8 t ..
                const uint32_t* const x = reinterpret_cast<const uint32_t*>(&w[b]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 f = F16 ? __half22float2(*reinterpret_cast<const __half2*>(&x[i]))
                                         : make_float2(__uint_as_float(x[i] << 16), __uint_as_float(x[i] & 0xffff0000u));
                    amax = fmaxf(amax, fmaxf(fabsf(f.x), fabsf(f.y)));
                }
            }
            amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
            amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
            int e = (int)(__float_as_uint(amax) >> 23) - 127;                         // (zero: -127, infinite: 128)
            e = amax > 0.f ? min(max(e, -126), 126) : 0;
            const float down = __uint_as_float((uint32_t)(127 - e) << 23), up = __uint_as_float((uint32_t)(127 + e) << 23);
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const uint32_t* const x = reinterpret_cast<const uint32_t*>(&w[b]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 f = F16 ? __half22float2(*reinterpret_cast<const __half2*>(&x[i]))
                                         : make_float2(__uint_as_float(x[i] << 16), __uint_as_float(x[i] & 0xffff0000u));
                    const __half2 h = __floats2half2_rn(f.x * down, f.y * down);
                    qb[b][nt][i] = *reinterpret_cast<const uint32_t*>(&h);
                }
            }
            const float own = p.scale_log2 * up;              // of column g; the accumulators hold columns 2 t, 2 t + 1
            mult[nt][0] = __shfl_sync(0xffffffffu, own, 8 * t);
            mult[nt][1] = __shfl_sync(0xffffffffu, own, 8 * t + 4);
        }
        float oacc[MT][NT][4], m_run[NT][2], l_run[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            m_run[nt][0] = m_run[nt][1] = -INFINITY;
            l_run[nt][0] = l_run[nt][1] = 0.f;
#pragma unroll
            for (int i = 0; i < MT; ++i) oacc[i][nt][0] = oacc[i][nt][1] = oacc[i][nt][2] = oacc[i][nt][3] = 0.f;
        }
        bool failed = false;
        for (int tile = warp; tile < n_tiles; tile += kPackedWarps) {
            const uint32_t s = taken % NS;
            if (!mbar_wait(bars + 8 * s, (taken / NS) & 1, p.wait_limit) || *sm_flag != 0) {
                if (lane == 0) {
                    record_status(p.status, DA_ERR_TIMEOUT);
                    *sm_flag = 1;
                }
                failed = true;
                break;
            }
            const uint32_t at = ring + s * Cfg::kTile;
            const int tok0 = u.tok_begin + tile * 16;
            const int n_valid = min(16, u.tok_end - tok0);
            // rows [hide0, hide1) lie between the sinks and the window
            int hide0 = 0, hide1 = 0;
            if (EXT) {
                const int pos = window_tile(cut, tok0 >> 4) << 4;
                hide0 = min(max(p.sinks - pos, 0), 16);
                hide1 = min(max(cut.first - pos, 0), n_valid);
            }
            auto seen = [&](int r) { return r < n_valid && !(EXT && r >= hide0 && r < hide1); };
            // ---- S^T
            float sacc[NT][4];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) sacc[nt][0] = sacc[nt][1] = sacc[nt][2] = sacc[nt][3] = 0.f;
            {
                uint32_t ka[NB], kb[NB], sa[NB / 2], sb[NB / 2];
                lds_words<NB>(at + row_a * (D / 2) + t * (D / 8), ka);
                lds_words<NB>(at + row_b * (D / 2) + t * (D / 8), kb);
                lds_words<NB / 2>(at + packed_k_scales(D) + row_a * NB * 2, sa);
                lds_words<NB / 2>(at + packed_k_scales(D) + row_b * NB * 2, sb);
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    uint32_t ha[4], hb[4];
                    packed_unpack(ka[b], ha);
                    packed_unpack(kb[b], hb);
                    const __half2 xa = *reinterpret_cast<const __half2*>(&sa[b / 2]), xb = *reinterpret_cast<const __half2*>(&sb[b / 2]);
                    const float fa = b & 1 ? __high2float(xa) : __low2float(xa), fb = b & 1 ? __high2float(xb) : __low2float(xb);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        float c[4] = {0.f, 0.f, 0.f, 0.f};
                        packed_mma(c, ha[0], hb[0], ha[1], hb[1], qb[b][nt][0], qb[b][nt][1]);
                        packed_mma(c, ha[2], hb[2], ha[3], hb[3], qb[b][nt][2], qb[b][nt][3]);
                        sacc[nt][0] = fmaf(c[0], fa, sacc[nt][0]);
                        sacc[nt][1] = fmaf(c[1], fa, sacc[nt][1]);
                        sacc[nt][2] = fmaf(c[2], fb, sacc[nt][2]);
                        sacc[nt][3] = fmaf(c[3], fb, sacc[nt][3]);
                    }
                }
            }
            // ---- softmax: rows (tokens) row_a, row_b, columns (heads) 2 t, 2 t + 1
            const bool see_a = seen(row_a), see_b = seen(row_b);
            uint32_t pb[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float s00 = see_a ? sacc[nt][0] * mult[nt][0] : -INFINITY, s01 = see_a ? sacc[nt][1] * mult[nt][1] : -INFINITY;
                const float s10 = see_b ? sacc[nt][2] * mult[nt][0] : -INFINITY, s11 = see_b ? sacc[nt][3] * mult[nt][1] : -INFINITY;
                float mx0 = fmaxf(s00, s10), mx1 = fmaxf(s01, s11);
                if (__any_sync(0xffffffffu, mx0 > m_run[nt][0] + 8.f || mx1 > m_run[nt][1] + 8.f)) {
#pragma unroll
                    for (int off = 4; off <= 16; off <<= 1) {
                        mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, off));
                        mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, off));
                    }
                    const float mn0 = fmaxf(m_run[nt][0], mx0), mn1 = fmaxf(m_run[nt][1], mx1);
                    const float al0 = ex2f(m_run[nt][0] - mn0), al1 = ex2f(m_run[nt][1] - mn1);
                    m_run[nt][0] = mn0;
                    m_run[nt][1] = mn1;
                    l_run[nt][0] *= al0;
                    l_run[nt][1] *= al1;
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        oacc[i][nt][0] *= al0; oacc[i][nt][1] *= al1;
                        oacc[i][nt][2] *= al0; oacc[i][nt][3] *= al1;
                    }
                }
                const float p00 = ex2f(s00 - m_run[nt][0]), p01 = ex2f(s01 - m_run[nt][1]);
                const float p10 = ex2f(s10 - m_run[nt][0]), p11 = ex2f(s11 - m_run[nt][1]);
                l_run[nt][0] += p00 + p10;
                l_run[nt][1] += p01 + p11;
                const __half2 h0 = __floats2half2_rn(p00, p01), h1 = __floats2half2_rn(p10, p11);
                pb[nt][0] = packed_transpose(*reinterpret_cast<const uint32_t*>(&h0));
                pb[nt][1] = packed_transpose(*reinterpret_cast<const uint32_t*>(&h1));
            }
            // ---- O^T: the lane's tokens 4 t + (j ^ t), its dims (D / 8) g ..
            {
                uint32_t v[4][NW], vs[2];
                lds_words<2>(at + packed_v_scales(D) + (g * (D / 8) / 32) * 32 + 8 * t, vs);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int r = 4 * t + (j ^ t);
                    lds_words<NW>(at + packed_v_codes(D) + r * (D / 2) + (D == 128 ? (8 * g) ^ (32 * (t >> 1)) : 4 * g), v[j]);
                }
                if (n_valid < 16 || (EXT && hide0 < hide1)) {
                    // (codes are finite whatever the bytes hold; a scale that is not would spoil a weight of zero)
                    uint32_t keep[2] = {0, 0};
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (seen(4 * t + (j ^ t))) keep[j >> 1] |= j & 1 ? 0xffff0000u : 0x0000ffffu;
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
                        for (int nt = 0; nt < NT; ++nt) packed_mma(oacc[4 * w + m][nt], a0, a1, a2, a3, pb[nt][0], pb[nt][1]);
                    }
                }
            }
            ++taken;
            __syncwarp();                                     // every lane has read the tile
            ask();
        }
        if (last_unit) pdl_launch_dependents();

        // ------------------------------------------------------------ end of the unit
        const bool stale = dev_len != u.seq_len;
        if (stale && tid == 0) record_status(p.status, DA_ERR_STALE_PLAN);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int off = 4; off <= 16; off <<= 1) {
                l_run[nt][0] += __shfl_xor_sync(0xffffffffu, l_run[nt][0], off);
                l_run[nt][1] += __shfl_xor_sync(0xffffffffu, l_run[nt][1], off);
            }
        // (the barrier also says that every warp is done with the scratch of the unit before)
        const bool gave_up = block_sync_or(1, kPackedThreads, failed || *sm_flag != 0);
        if (gave_up || stale) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                m_run[nt][0] = m_run[nt][1] = -INFINITY;
                l_run[nt][0] = l_run[nt][1] = 0.f;
            }
        }
#pragma unroll
        for (int q = 0; q < 2 * NT; ++q) {                     // four heads at a time
            if (4 * q >= G) break;
            const int nt = q >> 1;
            if (q > 0) block_sync(1, kPackedThreads);
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
            block_sync(1, kPackedThreads);
            block_finish<D, kPackedWarps, Cfg::kCols, false>(p, u, G, sm_wo, sm_wm, sm_wl, tid, kPackedThreads, 1, 4 * q,
                                                             min(4, G - 4 * q), 4 * (q + 1) >= G);
        }
        if (gave_up) break;
    }
    // a block that gave up leaves no copy of its own in flight (each of these waits has its limit too)
    for (; (int)taken < i_issued; ++taken)
        if (!mbar_wait(bars + 8 * (taken % NS), (taken / NS) & 1, p.wait_limit)) break;
}

}  // namespace da
