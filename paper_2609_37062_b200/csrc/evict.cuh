// Eviction from a paged cache by accumulated attention weight.
//
// For every (sequence, KV head) that holds more than `budget` tokens: the
// first `sinks` and the last `recent` tokens stay, and of the tokens between
// them the budget - sinks - recent with the largest totals; among equal totals
// the lowest position stays.  What stays keeps its order and moves to fresh
// pages.  Two launches:
//
//   select  one block per (sequence, KV head).  The totals become 32-bit keys whose unsigned order is the
//           order of the floats, and the key of rank k is found by three counting passes over 11, 11 and 10 bits
//           (the later ones only over what shares the leading bits).  Then one ordered pass: every warp takes
//           a run of neighbouring positions, counts what it keeps, and with the sums of the warps before it
//           writes positions and totals to their places.  The totals sit in shared memory meanwhile (longer
//           rows are walked in chunks), so they can be compacted in place.
//   move    K and V rows of the kept positions, 16 bytes a lane, 32 tokens of one KV head per warp.
//
// Select reads 4 bytes per token and KV head, move reads and writes 4 D of them for every kept one: the
// second is the bound, by memory.
#pragma once

#include "common.cuh"

namespace da {

constexpr int kEvictDigits = 2048;                 // bins of a counting pass
constexpr int kEvictChunk = 48 * 1024;             // totals a block holds in shared memory
constexpr int kMoveThreads = 256;
constexpr int kMoveTokens = 32;                    // of one (sequence, KV head) per warp
constexpr int kMoveUnroll = 8;                     // 16-byte loads a lane keeps in flight

struct EvictParams {
    const int32_t* seq_lens;
    const int32_t* block_table;
    const int32_t* dst_block_table;
    __nv_bfloat16* k;
    __nv_bfloat16* v;
    const float* weights;
    float* weights_out;
    int32_t* kept;              // [batch][Hkv][budget]
    int32_t* seq_lens_out;
    int32_t* status;            // may be NULL
    int64_t weight_tokens, stride_seq, stride_head;
    int64_t k_stride_page, k_stride_token, k_stride_head;
    int64_t v_stride_page, v_stride_token, v_stride_head;
    int64_t num_pages;
    int32_t batch, num_kv_heads, max_pages_per_seq, dst_max_pages, page_shift;
    int32_t budget, sinks, recent;
    int32_t chunk;              // totals the launch's shared memory holds
};

// Unsigned integers in the order of the floats; -0 equals +0, NaN counts as -inf.
__device__ __forceinline__ uint32_t weight_key(float f)
{
    if (f != f) f = -INFINITY;
    const uint32_t u = __float_as_uint(f + 0.f);
    return (u >> 31) ? ~u : (u | 0x80000000u);
}

// A row's length as both launches read it: -1 if it does not fit the tables or the totals (nothing is touched).
__device__ __forceinline__ int evict_length(const EvictParams& p, int b)
{
    const int L = __ldg(p.seq_lens + b);
    if (L < 0 || L > p.weight_tokens || ((int64_t)L + (1 << p.page_shift) - 1) >> p.page_shift > p.max_pages_per_seq) return -1;
    return L;
}

// Sum over the threads before this one, and over all of them.
template <int NT>
__device__ __forceinline__ int block_scan(int x, int* sm /* [NT / 32] */, int& total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int inc = x;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, inc, off);
        if (lane >= off) inc += y;
    }
    if (lane == 31) sm[warp] = inc;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < NT / 32; ++w) {
        const int s = sm[w];
        if (w < warp) before += s;
        total += s;
    }
    __syncthreads();
    return before + inc - x;
}

template <int NT>
__global__ void __launch_bounds__(NT) decode_attn_evict_select_kernel(const EvictParams p)
{
    extern __shared__ float sm_w[];                           // [chunk] totals
    __shared__ int sm_hist[kEvictDigits];
    __shared__ int sm_scan[NT / 32], sm_gt[NT / 32], sm_eq[NT / 32];
    __shared__ int sm_found[2];
    constexpr int WARPS = NT / 32;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int b = blockIdx.x / p.num_kv_heads, g = blockIdx.x % p.num_kv_heads;
    pdl_launch_dependents();
    pdl_wait_primary();
    const int L = evict_length(p, b);
    int32_t* const kept = p.kept + ((int64_t)b * p.num_kv_heads + g) * p.budget;
    const int n = min(max(L, 0), p.budget);
    if (g == 0 && tid == 0) p.seq_lens_out[b] = L < 0 ? __ldg(p.seq_lens + b) : n;
    for (int i = n + tid; i < p.budget; i += NT) kept[i] = -1;
    if (L < 0) {
        if (tid == 0 && p.status) record_status(p.status, DA_ERR_STALE_PLAN);
        return;
    }
    const int64_t row = (int64_t)b * p.stride_seq + (int64_t)g * p.stride_head;
    const float* const w = p.weights + row;
    float* const o = p.weights_out + row;
    if (L <= p.budget) {                                      // nothing to evict: the row stays as it is
        for (int t = tid; t < L; t += NT) {
            kept[t] = t;
            if (o != w) o[t] = w[t];
        }
        return;
    }
    const int last = L - p.recent;                            // [sinks, last) compete
    const bool whole = L <= p.chunk;
    if (whole) {
#pragma unroll 8
        for (int t = tid; t < L; t += NT) sm_w[t] = w[t];
    }
    __syncthreads();
    auto total_of = [&](int t) { return whole ? sm_w[t] : w[t]; };

    // ---- the key of rank k among the competitors, and how many of its equals stay
    int k = p.budget - p.sinks - p.recent;
    uint32_t key = 0xffffffffu;                               // k = 0: above every key
    int ties = 0;
    if (k > 0) {
        key = 0;
#pragma unroll 1
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
            const uint32_t digits = pass == 2 ? 1023u : 2047u;
            const uint32_t above = pass == 0 ? 0u : (pass == 1 ? ~((1u << 21) - 1) : ~((1u << 10) - 1));
            for (int i = tid; i < kEvictDigits; i += NT) sm_hist[i] = 0;
            __syncthreads();
            for (int t0 = p.sinks + warp * 32; t0 < last; t0 += NT) {
                const int t = t0 + lane;
                bool in = t < last;
                uint32_t x = 0;
                if (in) x = weight_key(total_of(t));
                in = in && (x & above) == key;
                const uint32_t d = (x >> shift) & digits;
                const uint32_t m = __ballot_sync(0xffffffffu, in);
                if (m == 0) continue;
                // Totals of one warp often share their leading bits (all of them zero, at worst): the first
                // lane's digit is counted once for all lanes that have it, the rest one by one.
                const uint32_t d0 = __shfl_sync(0xffffffffu, d, __ffs(m) - 1);
                const uint32_t same = __ballot_sync(0xffffffffu, in && d == d0);
                if (in && d != d0) atomicAdd(sm_hist + d, 1);
                if (lane == 0) atomicAdd(sm_hist + d0, __popc(same));
            }
            __syncthreads();
            // bins from the top: the one in which the count reaches k
            constexpr int PER = kEvictDigits / NT;
            int c[PER], sum = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                c[i] = sm_hist[kEvictDigits - 1 - (tid * PER + i)];
                sum += c[i];
            }
            int all;
            int before = block_scan<NT>(sum, sm_scan, all);
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                if (before < k && before + c[i] >= k) {
                    sm_found[0] = kEvictDigits - 1 - (tid * PER + i);
                    sm_found[1] = before;
                }
                before += c[i];
            }
            __syncthreads();
            key |= (uint32_t)sm_found[0] << shift;
            k -= sm_found[1];
            __syncthreads();
        }
        ties = k;
    }

    // ---- positions and totals of what stays, in order
    int at = 0, equal = 0;                                    // kept, equals met: in the chunks before
    for (int c0 = 0; c0 < L; c0 += p.chunk) {
        const int cn = min(p.chunk, L - c0);
        if (!whole) {
            __syncthreads();
            for (int t = tid; t < cn; t += NT) sm_w[t] = w[c0 + t];
            __syncthreads();
        }
        const int seg = (cn + 32 * WARPS - 1) / (32 * WARPS) * 32;
        const int s0 = warp * seg, s1 = min(s0 + seg, cn);
        auto look = [&](int i, bool& gt, bool& eq) {
            const int t = c0 + i;
            const uint32_t x = i < s1 ? weight_key(sm_w[i]) : 0u;
            const bool sure = t < p.sinks || t >= last;
            gt = i < s1 && (sure || x > key);
            eq = i < s1 && !sure && x == key;
        };
        int n_gt = 0, n_eq = 0;
        for (int i0 = s0; i0 < s1; i0 += 32) {
            bool gt, eq;
            look(i0 + lane, gt, eq);
            n_gt += __popc(__ballot_sync(0xffffffffu, gt));
            n_eq += __popc(__ballot_sync(0xffffffffu, eq));
        }
        if (lane == 0) {
            sm_gt[warp] = n_gt;
            sm_eq[warp] = n_eq;
        }
        __syncthreads();
        int my_at = at, my_eq = equal;
#pragma unroll
        for (int x = 0; x < WARPS; ++x) {
            const int e = sm_eq[x];
            const int add = sm_gt[x] + min(max(ties - equal, 0), e);
            if (x < warp) {
                my_at += add;
                my_eq += e;
            }
            at += add;
            equal += e;
        }
        const uint32_t lower = (1u << lane) - 1;
        for (int i0 = s0; i0 < s1; i0 += 32) {
            bool gt, eq;
            look(i0 + lane, gt, eq);
            const uint32_t me = __ballot_sync(0xffffffffu, eq);
            const bool stay = gt || (eq && my_eq + __popc(me & lower) < ties);
            const uint32_t ms = __ballot_sync(0xffffffffu, stay);
            if (stay) {
                const int to = my_at + __popc(ms & lower);
                kept[to] = c0 + i0 + lane;
                o[to] = sm_w[i0 + lane];
            }
            my_at += __popc(ms);
            my_eq += __popc(me);
        }
        __syncthreads();                                      // the chunk, and the warps' counts, may be replaced
    }
    for (int t = p.budget + tid; t < L; t += NT) o[t] = 0.f;      // tokens to come start from nothing
}

template <int D>
__global__ void __launch_bounds__(kMoveThreads) decode_attn_evict_move_kernel(const EvictParams p)
{
    constexpr int LT = D / 4;                                 // lanes of a token: 16-byte chunks of its K row, then of its V row
    constexpr int TP = 32 / LT;                               // tokens a warp moves at a time
    pdl_launch_dependents();
    pdl_wait_primary();
    const int lane = threadIdx.x & 31;
    // KV heads of one token range next to each other: their rows share the fresh pages
    const int per_row = (p.budget + kMoveTokens - 1) / kMoveTokens;
    const int64_t unit = (int64_t)blockIdx.x * (kMoveThreads / 32) + (threadIdx.x >> 5);
    const int g = (int)(unit % p.num_kv_heads);
    const int64_t rest = unit / p.num_kv_heads;
    const int b = (int)(rest / per_row), j0 = (int)(rest % per_row) * kMoveTokens;
    if (b >= p.batch || evict_length(p, b) <= p.budget) return;
    // lane i: source and destination page of token j0 + i
    const int j = j0 + lane;
    int src = 0, src_page = -1, dst_page = -1;
    if (j < p.budget) {
        src = __ldcg(p.kept + ((int64_t)b * p.num_kv_heads + g) * p.budget + j);
        dst_page = __ldg(p.dst_block_table + (int64_t)b * p.dst_max_pages + (j >> p.page_shift));
        src_page = __ldg(p.block_table + (int64_t)b * p.max_pages_per_seq + (src >> p.page_shift));
        if ((unsigned)src_page >= (unsigned)p.num_pages || (unsigned)dst_page >= (unsigned)p.num_pages) {
            if (p.status) record_status(p.status, DA_ERR_BAD_PAGE);   // the row is not moved
            src_page = dst_page = -1;
        }
    }
    const int mask = (1 << p.page_shift) - 1;
    const int part = lane % LT, ch = part % (D / 8);          // which row (K, V), which 16 bytes of it
    const bool is_v = part >= D / 8;
    __nv_bfloat16* const pool = (is_v ? p.v : p.k) + (int64_t)g * (is_v ? p.v_stride_head : p.k_stride_head) + ch * 8;
    const int64_t sp = is_v ? p.v_stride_page : p.k_stride_page, st = is_v ? p.v_stride_token : p.k_stride_token;
#pragma unroll
    for (int i0 = 0; i0 < kMoveTokens; i0 += TP * kMoveUnroll) {
        uint4 x[kMoveUnroll];
        int to_page[kMoveUnroll];
#pragma unroll
        for (int u = 0; u < kMoveUnroll; ++u) {
            const int i = i0 + u * TP + lane / LT;
            const int from = __shfl_sync(0xffffffffu, src_page, i), slot = __shfl_sync(0xffffffffu, src, i) & mask;
            to_page[u] = __shfl_sync(0xffffffffu, dst_page, i);
            if (from >= 0) x[u] = __ldcs(reinterpret_cast<const uint4*>(pool + from * sp + slot * st));
        }
#pragma unroll
        for (int u = 0; u < kMoveUnroll; ++u) {
            const int i = i0 + u * TP + lane / LT;
            if (to_page[u] >= 0) *reinterpret_cast<uint4*>(pool + to_page[u] * sp + ((j0 + i) & mask) * st) = x[u];
        }
    }
}

}  // namespace da
