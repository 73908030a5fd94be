// Rows of new tokens: per-head norms, rotation and the cache write in one pass (decode_attn_prepare_rows).
//
// Bound by memory, with issued instructions close behind: a row's heads are read once and written once.  A warp takes one row
// after the other, or a share of a row's heads where there are few rows.  A group of D / 16 of its lanes owns one head at a
// time, sixteen dims a lane in two units of eight, a unit being two runs of four: for the rotation of halves a unit is four
// dims of the first half and their partners of the second, so that a pair never leaves its lane; otherwise its eight dims
// are neighbours.  What weight and angle do to a pair (a, b) is one 2 x 2 matrix, the same for all heads that share the weight:
// it is made once a row and kept in registers, a head costs four products a pair and the root of its mean of squares (a butterfly
// over the group's lanes) two more.
//
// A lane copies its own 32 bytes of the heads ahead to a ring in shared memory (cp.async), three tasks of 512 / D heads ahead
// and across rows, and the angles of the row after this one: held in registers, loads ahead wait for one another (8,192 rows of
// 48 heads of 128, 206 MB: 38.2 us, 5.4 TB/s, where registers took 54 to 65 in every arrangement).
#pragma once

#include <type_traits>

#include "common.cuh"
#include "packed.cuh"

namespace da {

constexpr int kRowsThreads = 256;
constexpr int kRowsRing = 4;                     // tasks in a warp's ring
constexpr int kRowsLane = kRowsRing * 32 + 128;  // bytes of shared memory of a lane: the ring, angles of two rows
constexpr int kRowsSmem = kRowsThreads * kRowsLane;
constexpr int kRowsBlocks = 2;                   // on an SM

struct RowsParams {
    const uint16_t *q, *k, *v;
    int64_t q_stride, k_stride, v_stride;
    const uint16_t *q_weight, *k_weight;
    int64_t q_weight_stride, k_weight_stride;
    const float* cos_sin;
    const int32_t* positions;
    const int64_t* slots;
    uint16_t *q_out, *k_out;
    int64_t q_out_stride, k_out_stride;
    void *k_cache, *v_cache;
    int32_t* status;
    int64_t num_pages;
    // 16-bit pools: elements; the pool in 4 bits (k_* alone): bytes
    int64_t k_stride_page, k_stride_token, k_stride_head;
    int64_t v_stride_page, v_stride_token, v_stride_head;
    int32_t rows, n_q, n_k, n_v;      // heads of a row to work on
    int32_t rotary_dim, max_positions;
    int32_t page_shift;
    int32_t split;                    // warps to a row
    float eps;
};

// 16-bit input types: two values of a word, and back with one rounding.
template <bool F16>
__device__ __forceinline__ float2 rows_pair(uint32_t w)
{
    if (F16) return __half22float2(*reinterpret_cast<const __half2*>(&w));
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}

template <bool F16>
__device__ __forceinline__ uint32_t rows_pack(float lo, float hi)
{
    if (F16) {
        const __half2 h = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}

template <int BYTES>
__device__ __forceinline__ void rows_copy(uint32_t dst, const void* src)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(BYTES) : "memory");
}

// Where the runs of a head's unit i (of D / 8) begin.  With HALVES the units of the dims that turn come first.
struct RowDims {
    int a, b;
};

template <bool HALVES>
__device__ __forceinline__ RowDims row_dims(int i, int rotary_dim)
{
    if (HALVES && i < (rotary_dim >> 3)) return {4 * i, (rotary_dim >> 1) + 4 * i};
    return {8 * i, 8 * i + 4};
}

// A lane's units are 2 l and 2 l + 1 (NEAR: the runs of the first half that it holds lie behind each other, as do those of the
// second; a quantised block of 32 dims lies with two lanes), or l and D / 16 + l, where neither matters.
template <int D, bool NEAR>
__device__ __forceinline__ int row_unit(int l, int k)
{
    return NEAR ? 2 * l + k : l + k * (D / 16);
}

// A lane's sixteen dims.  wide: 16 bytes at a time (the runs of a half begin at multiples of eight dims).
template <int D, bool HALVES, bool ALL, bool NEAR>
__device__ __forceinline__ void row_load(const uint16_t* src, int l, int rotary_dim, bool wide, uint2 (&u)[2][2])
{
    if (wide) {
        const RowDims x = row_dims<HALVES>(row_unit<D, NEAR>(l, 0), rotary_dim), y = row_dims<HALVES>(row_unit<D, NEAR>(l, 1), rotary_dim);
        const bool halves = HALVES && (ALL || 16 * l < rotary_dim);   // runs a of both units, then runs b; else unit by unit
        const uint4 p = *reinterpret_cast<const uint4*>(src + x.a), q = *reinterpret_cast<const uint4*>(src + (halves ? x.b : y.a));
        u[0][0] = make_uint2(p.x, p.y);
        (halves ? u[1][0] : u[0][1]) = make_uint2(p.z, p.w);
        (halves ? u[0][1] : u[1][0]) = make_uint2(q.x, q.y);
        u[1][1] = make_uint2(q.z, q.w);
        return;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const RowDims x = row_dims<HALVES>(row_unit<D, NEAR>(l, k), rotary_dim);
        u[k][0] = *reinterpret_cast<const uint2*>(src + x.a);
        u[k][1] = *reinterpret_cast<const uint2*>(src + x.b);
    }
}

template <int D, bool HALVES, bool ALL, bool NEAR>
__device__ __forceinline__ void row_store(uint16_t* dst, int l, int rotary_dim, bool wide, const uint2 (&u)[2][2])
{
    if (wide) {
        const RowDims x = row_dims<HALVES>(row_unit<D, NEAR>(l, 0), rotary_dim), y = row_dims<HALVES>(row_unit<D, NEAR>(l, 1), rotary_dim);
        const bool halves = HALVES && (ALL || 16 * l < rotary_dim);
        const uint2 second = halves ? u[1][0] : u[0][1], third = halves ? u[0][1] : u[1][0];
        *reinterpret_cast<uint4*>(dst + x.a) = make_uint4(u[0][0].x, u[0][0].y, second.x, second.y);
        *reinterpret_cast<uint4*>(dst + (halves ? x.b : y.a)) = make_uint4(third.x, third.y, u[1][1].x, u[1][1].y);
        return;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const RowDims x = row_dims<HALVES>(row_unit<D, NEAR>(l, k), rotary_dim);
        *reinterpret_cast<uint2*>(dst + x.a) = u[k][0];
        *reinterpret_cast<uint2*>(dst + x.b) = u[k][1];
    }
}

// row_load's reads as copies to the lane's places dst and dst + kRowsPlane, in row_load's order of words.
constexpr uint32_t kRowsPlane = 512;             // (a plane holds 16 bytes of every lane)

template <int D, bool HALVES, bool ALL, bool NEAR>
__device__ __forceinline__ void row_fetch(uint32_t dst, const uint16_t* src, int l, int rotary_dim, bool wide)
{
    const RowDims x = row_dims<HALVES>(row_unit<D, NEAR>(l, 0), rotary_dim), y = row_dims<HALVES>(row_unit<D, NEAR>(l, 1), rotary_dim);
    if (wide) {
        const bool halves = HALVES && (ALL || 16 * l < rotary_dim);
        rows_copy<16>(dst, src + x.a);
        rows_copy<16>(dst + kRowsPlane, src + (halves ? x.b : y.a));
        return;
    }
    rows_copy<8>(dst, src + x.a);
    rows_copy<8>(dst + 8, src + x.b);
    rows_copy<8>(dst + kRowsPlane, src + y.a);
    rows_copy<8>(dst + kRowsPlane + 8, src + y.b);
}

template <bool HALVES, bool ALL>
__device__ __forceinline__ void row_take(uint32_t at, int l, int rotary_dim, bool wide, uint2 (&u)[2][2])
{
    uint4 p, q;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(p.x), "=r"(p.y), "=r"(p.z), "=r"(p.w) : "r"(at));
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "r"(at + kRowsPlane));
    const bool halves = HALVES && wide && (ALL || 16 * l < rotary_dim);               // runs a of both units, then runs b
    const uint2 second = make_uint2(p.z, p.w), third = make_uint2(q.x, q.y);
    u[0][0] = make_uint2(p.x, p.y);
    u[0][1] = halves ? third : second;
    u[1][0] = halves ? second : third;
    u[1][1] = make_uint2(q.z, q.w);
}

// HALVES: pairs are (i, i + rotary_dim / 2); else neighbours, or nothing turns.
// ALL: all dims turn (rotary_dim is D).
template <int D, bool F16, bool PACKED, bool HALVES, bool ALL>
__global__ void __launch_bounds__(kRowsThreads, kRowsBlocks) decode_attn_rows_kernel(const RowsParams p)
{
    constexpr int L = D / 16;                                 // lanes of a head
    constexpr int HEADS = 32 / L;                             // heads of a task
    constexpr bool NEAR = HALVES || PACKED;
    extern __shared__ __align__(128) uint8_t smem[];
    pdl_launch_dependents();
    pdl_wait_primary();
    const int lane = threadIdx.x & 31, l = lane % L, group = lane / L;
    // the lane's places: tasks' planes, then four planes of angles for even and for odd rows of the warp
    const uint32_t ring = smem_u32(smem) + (threadIdx.x >> 5) * (32 * kRowsLane) + lane * 16;
    const uint32_t angles_at = ring + kRowsRing * 2 * kRowsPlane;
    const int rotary = ALL ? D : p.rotary_dim;
    const bool wide = !HALVES || ALL || rotary % 16 == 0;
    // tasks of HEADS heads, those of q first, then k, then v; work item id: row id / split, a share of its tasks
    const int tq = (p.n_q + HEADS - 1) / HEADS, tk = (p.n_k + HEADS - 1) / HEADS, tv = (p.n_v + HEADS - 1) / HEADS;
    const int tasks = tq + tk + tv;
    const unsigned split = p.split, stride = gridDim.x * (kRowsThreads / 32), items = (unsigned)p.rows * split;   // (below 2^31)
    const unsigned first_id = blockIdx.x * (kRowsThreads / 32) + (threadIdx.x >> 5);
    if (first_id >= items) return;
    auto row_of = [&](unsigned id) { return (int)(split == 1 ? id : id / split); };
    // the first task of share `part`
    auto cut_at = [&](unsigned part) { return split == 1 ? (part ? tasks : 0) : (int)((unsigned)tasks * part / split); };

    // ---- asking for tasks
    unsigned i_id = first_id;
    int i_row = row_of(i_id), i_task = cut_at(i_id - i_row * split), i_end = cut_at(i_id - i_row * split + 1);
    uint32_t i_slot = 0;
    auto ask = [&]() {
        if (i_id < items) {
            const uint32_t dst = ring + i_slot * (2 * kRowsPlane);
            if (i_task < tq) {
                const int h = i_task * HEADS + group;
                if (h < p.n_q) row_fetch<D, HALVES, ALL, NEAR>(dst, p.q + i_row * p.q_stride + h * D, l, rotary, wide);
            } else if (i_task < tq + tk) {
                const int h = (i_task - tq) * HEADS + group;
                if (h < p.n_k) row_fetch<D, HALVES, ALL, NEAR>(dst, p.k + i_row * p.k_stride + h * D, l, rotary, wide);
            } else {
                const int h = (i_task - tq - tk) * HEADS + group;
                if (h < p.n_v) row_fetch<D, false, ALL, NEAR>(dst, p.v + i_row * p.v_stride + h * D, l, 0, true);
            }
            if (++i_task == i_end) {
                i_id += stride;
                if (i_id < items) {
                    i_row = row_of(i_id);
                    i_task = cut_at(i_id - i_row * split);
                    i_end = cut_at(i_id - i_row * split + 1);
                }
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");  // (a group for every call: the waits below count them)
        i_slot = (i_slot + 1) % kRowsRing;
    };
    // positions and slots are read a row ahead, angles copied a row ahead of their use
    auto position = [&](unsigned id) { return p.positions != nullptr && id < items ? p.positions[row_of(id)] : 0; };
    auto slot_of = [&](unsigned id) {
        return p.k_cache != nullptr && id < items ? p.slots[row_of(id)] : -1;
    };
    auto copy_angles = [&](int pos, uint32_t to) {
        if (p.cos_sin == nullptr || pos < 0 || pos >= p.max_positions) return;
        const float* const angles = p.cos_sin + (int64_t)pos * rotary;
#pragma unroll
        for (int k = 0; k < 2; ++k) {                         // either way unit j's four pairs are 4 j .. 4 j + 3
            const int j = row_unit<D, NEAR>(l, k);
            if (!ALL && 8 * j >= rotary) continue;
            rows_copy<16>(to + (2 * k) * kRowsPlane, angles + 4 * j);
            rows_copy<16>(to + (2 * k + 1) * kRowsPlane, angles + (rotary >> 1) + 4 * j);
        }
    };
    int pos = position(first_id), next_pos = position(first_id + stride);
    int64_t slot = slot_of(first_id), next_slot = slot_of(first_id + stride);
    for (int i = 0; i < kRowsRing - 2; ++i) ask();
    copy_angles(pos, angles_at);
    ask();
    uint32_t t_slot = 0;
    bool odd = false;
    // The angles of a work item are asked for with the first task of the item before it, so the waits for tasks cover them where that
    // one had kRowsRing - 1 tasks or more (a row's shares differ by one, and a warp's next item may be another part); the first item's
    // were asked for with its own tasks.
    bool angles_late = true;

    for (unsigned id = first_id; id < items; id += stride) {
        const int row = row_of(id), begin = cut_at(id - row * split), end = cut_at(id - row * split + 1);
        const int after = position(id + 2 * stride);
        const int64_t after_slot = slot_of(id + 2 * stride);
        copy_angles(next_pos, angles_at + (odd ? 0 : 4) * kRowsPlane);
        const uint32_t angles = angles_at + (odd ? 4 : 0) * kRowsPlane;
        // padding, or a position behind the table: its tasks are taken from the ring and left alone
        bool skip = pos < 0;
        if (!skip && p.cos_sin != nullptr && pos >= p.max_positions) {
            if (lane == 0 && begin == 0 && p.status != nullptr) record_status(p.status, DA_ERR_STALE_PLAN);
            skip = true;
        }
        // the row's place in the cache (page < 0: none)
        int64_t page = slot >= 0 ? slot >> p.page_shift : -1;
        const int place = (int)(slot & ((1 << p.page_shift) - 1));
        if (page >= p.num_pages) {
            if (!skip && lane == 0 && begin == 0 && p.status != nullptr) record_status(p.status, DA_ERR_BAD_PAGE);
            page = -1;
        }

        // Tasks [first, last) of kind KIND (0 q, 1 k, 2 v), counted within the kind.
        auto walk = [&](auto kind_c, int first, int last) {
            constexpr int KIND = decltype(kind_c)::value;
            constexpr bool TURN = HALVES && KIND < 2;         // how the head's dims lie in the lanes
            const int n = KIND == 0 ? p.n_q : KIND == 1 ? p.n_k : p.n_v;
            const uint16_t* const w = KIND == 0 ? p.q_weight : KIND == 1 ? p.k_weight : nullptr;
            const int64_t w_stride = KIND == 0 ? p.q_weight_stride : p.k_weight_stride;
            const bool norm = KIND < 2 && w != nullptr, turn = KIND < 2 && p.cos_sin != nullptr;
            bool turned[2] = {false, false};
            // (a, b) <- r (m0 a - m1 b, m2 b + m3 a), r the root; pair e of unit k
            float m0[2][4], m1[2][4], m2[2][4], m3[2][4];
            bool fresh = true;                                // the matrices are still to be made
            for (int t = first; t < last; ++t) {
                asm volatile("cp.async.wait_group %0;" ::"n"(kRowsRing - 2) : "memory");
                uint2 raw[2][2];
                row_take<TURN, ALL>(ring + t_slot * (2 * kRowsPlane), l, rotary, wide, raw);
                t_slot = (t_slot + 1) % kRowsRing;
                ask();
                if (skip) continue;
                const int h = t * HEADS + group;
                const bool live = h < n;                      // (the whole warp stays: its lanes exchange values)
                if (norm || turn) {
                    if (fresh || (norm && w_stride != 0)) {
                        if (fresh && angles_late) asm volatile("cp.async.wait_group 0;" ::: "memory");
                        uint2 y[2][2];
                        y[0][0] = y[0][1] = y[1][0] = y[1][1] = make_uint2(0, 0);
                        if (norm && live) row_load<D, TURN, ALL, NEAR>(w + h * w_stride, l, rotary, wide || !TURN, y);
                        // (a lane without a head of its own here may have one in the next task: a shared weight is everybody's)
                        if (norm && !live && w_stride == 0) row_load<D, TURN, ALL, NEAR>(w, l, rotary, wide || !TURN, y);
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            float f[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
                            if (norm) {
#pragma unroll
                                for (int r = 0; r < 2; ++r) {
                                    const float2 lo = rows_pair<F16>(y[k][r].x), hi = rows_pair<F16>(y[k][r].y);
                                    f[4 * r] = lo.x; f[4 * r + 1] = lo.y; f[4 * r + 2] = hi.x; f[4 * r + 3] = hi.y;
                                }
                            }
                            const int j = row_unit<D, NEAR>(l, k);
                            float cs[4] = {1.f, 1.f, 1.f, 1.f}, sn[4] = {0.f, 0.f, 0.f, 0.f};
                            turned[k] = turn && (ALL || 8 * j < rotary);
                            if (turned[k]) {
                                asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(cs[0]), "=f"(cs[1]), "=f"(cs[2]), "=f"(cs[3]) : "r"(angles + (2 * k) * kRowsPlane));
                                asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(sn[0]), "=f"(sn[1]), "=f"(sn[2]), "=f"(sn[3]) : "r"(angles + (2 * k + 1) * kRowsPlane));
                            }
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const float wa = HALVES ? f[e] : f[2 * e], wb = HALVES ? f[4 + e] : f[2 * e + 1];
                                m0[k][e] = wa * cs[e];
                                m1[k][e] = wb * sn[e];
                                m2[k][e] = wb * cs[e];
                                m3[k][e] = wa * sn[e];
                            }
                        }
                        fresh = false;
                    }
                    float x[2][8], sum = 0.f, sum2 = 0.f;
#pragma unroll
                    for (int k = 0; k < 2; ++k)
#pragma unroll
                        for (int r = 0; r < 2; ++r) {
                            const float2 lo = rows_pair<F16>(raw[k][r].x), hi = rows_pair<F16>(raw[k][r].y);
                            x[k][4 * r] = lo.x; x[k][4 * r + 1] = lo.y; x[k][4 * r + 2] = hi.x; x[k][4 * r + 3] = hi.y;
                        }
                    float root = 1.f;
                    if (norm) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            sum = fmaf(x[0][e], x[0][e], sum);
                            sum2 = fmaf(x[1][e], x[1][e], sum2);
                        }
                        sum += sum2;
#pragma unroll
                        for (int off = L / 2; off >= 1; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
                        root = rsqrtf(sum * (1.0f / D) + p.eps);
                    }
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            float& a = HALVES ? x[k][e] : x[k][2 * e];
                            float& b = HALVES ? x[k][4 + e] : x[k][2 * e + 1];
                            const float a0 = a * m0[k][e], b0 = b * m2[k][e];
                            // (what does not turn stays clear of its neighbour, infinite ones included)
                            const float na = ALL || turned[k] ? fmaf(-b, m1[k][e], a0) : a0;
                            b = root * (ALL || turned[k] ? fmaf(a, m3[k][e], b0) : b0);
                            a = root * na;
                        }
#pragma unroll
                        for (int r = 0; r < 2; ++r)
                            raw[k][r] = make_uint2(rows_pack<F16>(x[k][4 * r], x[k][4 * r + 1]), rows_pack<F16>(x[k][4 * r + 2], x[k][4 * r + 3]));
                    }
                }
                uint16_t* const out = KIND == 0 ? p.q_out + row * p.q_out_stride : KIND == 1 && p.k_out != nullptr ? p.k_out + row * p.k_out_stride : nullptr;
                if (live && out != nullptr) row_store<D, TURN, ALL, NEAR>(out + h * D, l, rotary, wide || !TURN, raw);
                if (KIND == 0 || page < 0) continue;
                if (!PACKED) {
                    uint16_t* const pool = KIND == 1 ? static_cast<uint16_t*>(p.k_cache) + page * p.k_stride_page + place * p.k_stride_token
                                                     : static_cast<uint16_t*>(p.v_cache) + page * p.v_stride_page + place * p.v_stride_token;
                    if (live) row_store<D, TURN, ALL, NEAR>(pool + h * (KIND == 1 ? p.k_stride_head : p.v_stride_head), l, rotary, wide || !TURN, raw);
                } else {
                    // Sixteen neighbouring dims to a lane, runs 4 l .. 4 l + 3 of four: what the lane holds, but for K that was
                    // turned by halves, whose run g lies with unit g as its first (g < n, the units that turn) or with unit g - n
                    // as its second.
                    uint2 z[4] = {raw[0][0], raw[0][1], raw[1][0], raw[1][1]};
                    if (TURN) {
                        const int units = rotary >> 3;
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const int g = 4 * l + q;
                            const int unit = g < units ? g : g < 2 * units ? g - units : g >> 1;
                            const bool second = g < 2 * units ? g >= units : (g & 1);
#pragma unroll
                            for (int k = 0; k < 2; ++k)
#pragma unroll
                                for (int r = 0; r < 2; ++r) {
                                    if (ALL && k != (q & 1)) continue;        // (the number of units is even)
                                    const int from = (lane & ~(L - 1)) + (unit >> 1);
                                    const uint32_t lo = __shfl_sync(0xffffffffu, raw[k][r].x, from), hi = __shfl_sync(0xffffffffu, raw[k][r].y, from);
                                    if ((unit & 1) == k && second == (r == 1)) z[q] = make_uint2(lo, hi);
                                }
                        }
                    }
                    float y[2][8], amax = 0.f;
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const float2 lo = rows_pair<F16>(z[q].x), hi = rows_pair<F16>(z[q].y);
                        y[q >> 1][4 * (q & 1)] = lo.x; y[q >> 1][4 * (q & 1) + 1] = lo.y;
                        y[q >> 1][4 * (q & 1) + 2] = hi.x; y[q >> 1][4 * (q & 1) + 3] = hi.y;
                        amax = fmaxf(amax, fmaxf(fmaxf(fabsf(lo.x), fabsf(lo.y)), fmaxf(fabsf(hi.x), fabsf(hi.y))));
                    }
                    amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));      // the two lanes of a block of 32 dims
                    if (live) {
                        const __half scale = packed_scale(amax);
                        char* const tile = static_cast<char*>(p.k_cache) + page * p.k_stride_page + h * p.k_stride_head + (place >> 4) * packed_tile_bytes(D);
                        const int r = place & 15, block = l >> 1;
                        uint32_t* const codes = reinterpret_cast<uint32_t*>(tile + (KIND == 1 ? 0 : packed_v_codes(D)));
#pragma unroll
                        for (int k = 0; k < 2; ++k)
                            codes[KIND == 1 ? packed_k_word(D, r, 2 * l + k) : packed_v_word(D, r, 2 * l + k)] = packed_word(y[k], scale);
                        if ((l & 1) == 0) {
                            __half* const scales = reinterpret_cast<__half*>(tile + (KIND == 1 ? packed_k_scales(D) : packed_v_scales(D)));
                            scales[KIND == 1 ? packed_k_scale(D, r, block) : packed_v_scale(r, block)] = scale;
                        }
                    }
                }
            }
        };
        walk(std::integral_constant<int, 0>{}, begin, min(end, tq));
        walk(std::integral_constant<int, 1>{}, max(begin, tq) - tq, min(end, tq + tk) - tq);
        walk(std::integral_constant<int, 2>{}, max(begin, tq + tk) - tq - tk, end - tq - tk);
        pos = next_pos;
        slot = next_slot;
        next_pos = after;
        next_slot = after_slot;
        odd = !odd;
        angles_late = end - begin < kRowsRing - 1;
    }
}

}  // namespace da
