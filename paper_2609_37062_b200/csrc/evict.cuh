// Eviction from a paged cache by accumulated attention weight.
//
// For every (sequence, KV head) that holds more than `budget` tokens: the
// first `sinks` and the last `recent` tokens stay, and of the tokens between
// them the budget - sinks - recent with the largest totals; among equal totals
// the lowest position stays.  What stays keeps its order and moves to fresh
// pages.  Two steps:
//
//   select  one block per (sequence, KV head).  The totals become 32-bit keys whose unsigned order is the order
//           of the floats, and the key of rank k is found by counting them into bins between the least and the
//           greatest, then looking into the bin that holds rank k the same way.  Then one ordered pass: every warp
//           takes a run of neighbouring positions, counts what it keeps, and with the sums of the warps before it
//           writes positions and totals to their places.  The totals sit in shared memory meanwhile (the longest
//           rows are walked in runs), so they can be compacted in place.  (A cluster of eight blocks per row
//           loses: the exchange of a counting step through distributed shared memory takes 1,300 cycles.)
//   move    K and V rows of the kept positions, 16 bytes a lane, 32 tokens of one KV head per warp.
//
// Where each of a block's warps would move once, the select blocks move their rows themselves, in one launch.
//
// Select reads 4 bytes per token and KV head, move reads and writes 4 D of them for every kept one: the
// second is the bound, by memory.
#pragma once

#include "common.cuh"

namespace da {

constexpr int kEvictChunk = 48 * 1024;             // totals a block holds in shared memory
constexpr int kMoveThreads = 256;
constexpr int kMoveTokens = 32;                    // of one (sequence, KV head) per warp
constexpr int kMoveUnroll = 8;                     // 16-byte loads a lane keeps in flight
constexpr int kEvictPasses = 4;                    // 32 bits of key in passes of 10 (three would do for 11)

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

// What stays whatever its total, and what is not there: above and below the key of every float.
constexpr uint32_t kKeyStays = 0xffffffffu, kKeyNone = 0u;

// Unsigned integers in the order of the floats; -0 equals +0, NaN counts as -inf.
__device__ __forceinline__ uint32_t weight_key(float f)
{
    if (f != f) f = -INFINITY;
    const uint32_t u = __float_as_uint(f + 0.f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

// A row's length as both launches read it: -1 if it does not fit the tables or the totals (nothing is touched).
__device__ __forceinline__ int evict_length(const EvictParams& p, int b)
{
    const int L = __ldg(p.seq_lens + b);
    if (L < 0 || L > p.weight_tokens || ((int64_t)L + (1 << p.page_shift) - 1) >> p.page_shift > p.max_pages_per_seq) return -1;
    return L;
}

// K and V rows of the kept tokens j0 .. j0 + 31 of one (sequence, KV head), by one warp.
template <int D>
__device__ __forceinline__ void move_tokens(const EvictParams& p, int b, int g, int j0, int lane)
{
    constexpr int LT = D / 4;                                 // lanes of a token: 16-byte chunks of its K row, then of its V row
    constexpr int TP = 32 / LT;                               // tokens a warp moves at a time
    // lane i: source and destination page of token j0 + i
    const int j = j0 + lane;
    int src = 0, src_page = -1, dst_page = -1;
    if (j < p.budget) {
        src = __ldcg(p.kept + ((int64_t)b * p.num_kv_heads + g) * p.budget + j);
        if (src >= 0) {                                       // (-1: select gave the row up, and has said so)
            dst_page = __ldg(p.dst_block_table + (int64_t)b * p.dst_max_pages + (j >> p.page_shift));
            src_page = __ldg(p.block_table + (int64_t)b * p.max_pages_per_seq + (src >> p.page_shift));
            if ((unsigned)src_page >= (unsigned)p.num_pages || (unsigned)dst_page >= (unsigned)p.num_pages) {
                if (p.status) record_status(p.status, DA_ERR_BAD_PAGE);   // the row is not moved
                src_page = dst_page = -1;
            }
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

// One block of NT threads per (sequence, KV head).  BINS: of a counting pass.  HELD: totals a thread keeps the
// keys of in registers, where the row has no more.  D: the block moves its rows itself (0: the other launch does).
template <int NT, int BINS, int HELD, int D>
__global__ void __launch_bounds__(NT) decode_attn_evict_select_kernel(const EvictParams p)
{
    constexpr int WARPS = NT / 32, PER = BINS / NT;
    extern __shared__ float sm_w[];                           // [chunk] totals
    __shared__ int sm_hist[BINS];
    __shared__ int2 sm_warp[WARPS];
    __shared__ int sm_found[3];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int b = blockIdx.x / p.num_kv_heads, g = blockIdx.x % p.num_kv_heads;
    pdl_launch_dependents();
    pdl_wait_primary();
    const int L = evict_length(p, b);
    int32_t* const kept = p.kept + (int64_t)blockIdx.x * p.budget;
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
    // The row is walked in runs of up to p.chunk totals; a row of a single run (all but the longest) stays in shared
    // memory from the first look to the last.  A warp looks after `seg` neighbouring totals of a run, a lane after
    // every 32nd of them.
    const bool whole = L <= p.chunk;
    const int run = min(L, p.chunk);
    const int seg = (run + 32 * WARPS - 1) / (32 * WARPS) * 32;
    const bool held = whole && seg <= 32 * HELD;
    // the key of total f at position t, 0 <= t < L
    auto key_of = [&](int t, float f) { return t < p.sinks || t >= last ? kKeyStays : weight_key(f); };
    auto load = [&](int r0) {                                 // the totals of the run at r0
        const int m = min(run, L - r0);
        for (int i0 = tid; i0 < m; i0 += 16 * NT) {
            float x[16];                                      // (in flight together: a store would hold up the load behind it)
#pragma unroll
            for (int u = 0; u < 16; ++u) x[u] = i0 + u * NT < m ? __ldcg(w + r0 + i0 + u * NT) : 0.f;
#pragma unroll
            for (int u = 0; u < 16; ++u)
                if (i0 + u * NT < m) sm_w[i0 + u * NT] = x[u];
        }
    };
    uint32_t keys[HELD];
    if (held) {
        const int i0 = warp * seg + lane;
        float x[HELD];
#pragma unroll
        for (int u = 0; u < HELD; ++u) x[u] = 32 * u < seg && i0 + 32 * u < L ? __ldcg(w + i0 + 32 * u) : 0.f;
#pragma unroll
        for (int u = 0; u < HELD; ++u) {
            const bool in = 32 * u < seg && i0 + 32 * u < L;
            if (in) sm_w[i0 + 32 * u] = x[u];                 // (read again by this thread alone)
            keys[u] = in ? key_of(i0 + 32 * u, x[u]) : kKeyNone;
        }
    } else if (whole) {
        load(0);
        __syncthreads();
    }
    auto each_key = [&](auto&& f) {                           // whole warps call f
        if (held) {
#pragma unroll
            for (int u = 0; u < HELD; ++u)
                if (32 * u < seg) f(keys[u]);
        } else {
            for (int r0 = 0; r0 < L; r0 += run)
#pragma unroll 4
                for (int i0 = 32 * warp; i0 < run; i0 += NT) {
                    const int i = i0 + lane, t = r0 + i;
                    f(i < run && t < L ? key_of(t, whole ? sm_w[i] : __ldcg(w + t)) : kKeyNone);
                }
        }
    };

    // ---- the key of rank k among the competitors, and how many of its equals stay.  The keys between the least
    // and the greatest are counted in BINS bins of equal width; the bin with rank k is looked into the same way until it is
    // one key wide or all of it stays.  (Keys are the floats' bits, so totals that spread over powers of two spread
    // over the bins; three passes at most, as a rule.)
    int k = p.budget - p.sinks - p.recent;
    // A row of more than one run is read anew by every pass.  Should its totals change meanwhile (they must not),
    // the counts no longer fit together: no bin holds rank k, or the range is not down to one key after as many passes
    // as 32 bits take.  The row is then given up, see below.
    bool lost = false;
    uint32_t key = kKeyStays - 1;                             // k = 0: above every float's
    int ties = 0;
    if (k > 0) {
        uint32_t least = 0xffffffffu, most = 0u;
        each_key([&](uint32_t x) {
            if (x != kKeyNone) least = min(least, x);
            if (x != kKeyStays) most = max(most, x);
        });
        least = __reduce_min_sync(0xffffffffu, least);
        most = __reduce_max_sync(0xffffffffu, most);
        if (lane == 0) sm_warp[warp] = make_int2((int)least, (int)most);
        __syncthreads();
        if (lane < WARPS) {
            least = (uint32_t)sm_warp[lane].x;
            most = (uint32_t)sm_warp[lane].y;
        }
        uint32_t lo = __reduce_min_sync(0xffffffffu, least), hi = __reduce_max_sync(0xffffffffu, most) + 1;
        for (int pass = 0;; ++pass) {
            if (hi - lo == 1) {
                key = lo;
                ties = k;
                break;
            }
            if (pass == kEvictPasses) {
                lost = true;
                break;
            }
            const int bits = 32 - __clz((int)(hi - lo - 1));
            constexpr int LOG_BINS = BINS == 2048 ? 11 : 10;
            static_assert(1 << LOG_BINS == BINS, "bins");
            const int shift = max(0, bits - LOG_BINS);
            for (int i = tid; i < BINS; i += NT) sm_hist[i] = 0;
            __syncthreads();
            if (tid == 0) sm_found[0] = -1;
            each_key([&](uint32_t x) {
                // Where totals are equal (all of them zero, at worst) the lanes meet in one bin: the first lane's is
                // counted once for all that share it, the rest one by one.
                const bool in = x - lo < hi - lo;
                const uint32_t d = in ? (x - lo) >> shift : (uint32_t)BINS;
                const uint32_t d0 = __shfl_sync(0xffffffffu, d, 0);
                const uint32_t same = __ballot_sync(0xffffffffu, d == d0);
                if (in && d != d0) atomicAdd(sm_hist + d, 1);
                if (in && lane == 0) atomicAdd(sm_hist + d, __popc(same));
            });
            __syncthreads();
            int c[PER], sum = 0;                              // bins from the top
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                c[i] = sm_hist[BINS - 1 - (tid * PER + i)];
                sum += c[i];
            }
            int inc = sum;
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, inc, off);
                if (lane >= off) inc += y;
            }
            if (lane == 31) sm_warp[warp].x = inc;
            __syncthreads();
            int before = __reduce_add_sync(0xffffffffu, lane < warp ? sm_warp[lane].x : 0) + inc - sum;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                if (before < k && before + c[i] >= k) {       // one thread, one bin
                    sm_found[0] = BINS - 1 - (tid * PER + i);
                    sm_found[1] = before;
                    sm_found[2] = c[i];
                }
                before += c[i];
            }
            __syncthreads();
            if (sm_found[0] < 0) {
                lost = true;
                break;
            }
            lo += (uint32_t)sm_found[0] << shift;
            k -= sm_found[1];
            if (k == sm_found[2]) {                           // all of the bin stays
                key = lo - 1;
                break;
            }
            hi = min(hi, lo + (1u << shift));
        }
    }

    // ---- positions and totals of what stays, in order
    int at = 0, equal = 0;                                    // kept, equals met: in the runs before
    for (int r0 = 0; r0 < L && !lost; r0 += run) {
        __syncthreads();                                      // sm_warp, sm_w are free
        if (!whole) {
            load(r0);
            __syncthreads();
        }
        const int m = min(run, L - r0);
        const int s0 = warp * seg, s1 = min(s0 + seg, m);
        auto run_key = [&](int i) { return i < s1 ? key_of(r0 + i, sm_w[i]) : kKeyNone; };
        int n_gt = 0, n_eq = 0;
        if (held) {
#pragma unroll
            for (int u = 0; u < HELD; ++u)
                if (32 * u < seg) {
                    n_gt += keys[u] > key;
                    n_eq += keys[u] == key;
                }
        } else {
#pragma unroll 4
            for (int i0 = s0; i0 < s0 + seg; i0 += 32) {
                const uint32_t x = run_key(i0 + lane);
                n_gt += x > key;
                n_eq += x == key;
            }
        }
        n_gt = __reduce_add_sync(0xffffffffu, n_gt);
        n_eq = __reduce_add_sync(0xffffffffu, n_eq);
        if (lane == 0) sm_warp[warp] = make_int2(n_gt, n_eq);
        __syncthreads();                                      // (in place: the whole run has been read)
        const int2 said = lane < WARPS ? sm_warp[lane] : make_int2(0, 0);
        const int run_gt = __reduce_add_sync(0xffffffffu, said.x), run_eq = __reduce_add_sync(0xffffffffu, said.y);
        int my_eq = equal + __reduce_add_sync(0xffffffffu, lane < warp ? said.y : 0);
        // kept so far: all above the key, and the first `ties` equals
        int to0 = at + __reduce_add_sync(0xffffffffu, lane < warp ? said.x : 0) + min(my_eq, ties) - min(equal, ties);
        const uint32_t lower = (1u << lane) - 1;
        auto place = [&](int i, uint32_t x) {
            bool stay = x > key;
            if (ties > 0) {
                const bool eq = x == key;
                const uint32_t mask_eq = __ballot_sync(0xffffffffu, eq);
                stay = stay || (eq && my_eq + __popc(mask_eq & lower) < ties);
                my_eq += __popc(mask_eq);
            }
            const uint32_t mask = __ballot_sync(0xffffffffu, stay);
            const int to = to0 + __popc(mask & lower);
            if (stay && to < p.budget) {                      // (always, of totals that stood still)
                kept[to] = r0 + i;
                o[to] = sm_w[i];
            }
            to0 += __popc(mask);
        };
        if (held) {
#pragma unroll
            for (int u = 0; u < HELD; ++u)
                if (32 * u < seg) place(s0 + 32 * u + lane, keys[u]);
        } else {
            for (int i0 = s0; i0 < s0 + seg; i0 += 32) place(i0 + lane, run_key(i0 + lane));
        }
        at += run_gt + min(equal + run_eq, ties) - min(equal, ties);
        equal += run_eq;
    }
    if (lost || at != p.budget) {                             // given up: no position stays, no row moves, reported
        __syncthreads();
        for (int i = tid; i < p.budget; i += NT) kept[i] = -1;
        if (tid == 0 && p.status) record_status(p.status, DA_ERR_STALE_PLAN);
        return;
    }
    for (int t = p.budget + tid; t < L; t += NT) o[t] = 0.f;      // tokens to come start from nothing
    if (D != 0) {
        __syncthreads();                                      // the block's kept positions are written
        for (int j0 = warp * kMoveTokens; j0 < p.budget; j0 += WARPS * kMoveTokens) move_tokens<D == 0 ? 64 : D>(p, b, g, j0, lane);
    }
}

template <int D>
__global__ void __launch_bounds__(kMoveThreads) decode_attn_evict_move_kernel(const EvictParams p)
{
    pdl_launch_dependents();
    pdl_wait_primary();
    // KV heads of one token range next to each other: their rows share the fresh pages
    const int per_row = (p.budget + kMoveTokens - 1) / kMoveTokens;
    const int64_t unit = (int64_t)blockIdx.x * (kMoveThreads / 32) + (threadIdx.x >> 5);
    const int g = (int)(unit % p.num_kv_heads);
    const int64_t rest = unit / p.num_kv_heads;
    const int b = (int)(rest / per_row), j0 = (int)(rest % per_row) * kMoveTokens;
    if (b >= p.batch || evict_length(p, b) <= p.budget) return;
    move_tokens<D>(p, b, g, j0, threadIdx.x & 31);
}

}  // namespace da
