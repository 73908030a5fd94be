// Rows of new tokens: per-head norms, rotation and the cache write in one pass (decode_attn_prepare_rows).
//
// Bound by memory: a row's heads are read once and written once.  A group of D / 8 lanes owns one head of one row, eight
// dims a lane, held as two runs of four: for the rotation of halves a lane takes four dims of the first half and their
// partners of the second, so that a pair never leaves its lane; otherwise its eight dims are neighbours.  The mean of
// squares is a butterfly over the group's lanes.  A block takes one row; its warps walk the row's q, k and v heads.
#pragma once

#include "common.cuh"
#include "packed.cuh"

namespace da {

constexpr int kRowsThreads = 256;

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

// Where a lane's two runs of four dims begin.
struct RowDims {
    int a, b;
};

template <bool HALVES>
__device__ __forceinline__ RowDims row_dims(int l, int rotary_dim)
{
    if (!HALVES) return {8 * l, 8 * l + 4};
    const int n = rotary_dim >> 3;                            // lanes whose dims turn
    if (l < n) return {4 * l, (rotary_dim >> 1) + 4 * l};
    return {8 * l, 8 * l + 4};
}

// HALVES: pairs are (i, i + rotary_dim / 2); else neighbours, or nothing turns.
template <int D, bool F16, bool PACKED, bool HALVES>
__global__ void __launch_bounds__(kRowsThreads) decode_attn_rows_kernel(const RowsParams p)
{
    constexpr int L = D / 8;                                  // lanes of a head
    constexpr int GROUPS = kRowsThreads / L;
    pdl_launch_dependents();
    pdl_wait_primary();
    const int row = blockIdx.x;
    const int l = threadIdx.x % L, group = threadIdx.x / L;
    int pos = 0;
    if (p.positions != nullptr) {
        pos = __ldg(p.positions + row);
        if (pos < 0) return;
        if (p.cos_sin != nullptr && pos >= p.max_positions) {
            if (threadIdx.x == 0 && p.status != nullptr) record_status(p.status, DA_ERR_STALE_PLAN);
            return;
        }
    }
    // the row's place in the cache (page < 0: none)
    int64_t page = -1;
    int place = 0;
    if (p.k_cache != nullptr) {
        const int64_t slot = __ldg(reinterpret_cast<const long long*>(p.slots) + row);
        if (slot >= 0) {
            page = slot >> p.page_shift;
            place = (int)(slot & ((1 << p.page_shift) - 1));
            if (page >= p.num_pages) {
                if (threadIdx.x == 0 && p.status != nullptr) record_status(p.status, DA_ERR_BAD_PAGE);
                page = -1;
            }
        }
    }
    const RowDims turned = row_dims<HALVES>(l, p.rotary_dim);
    float c[8], s[8];                                         // HALVES: four pairs; else two of a run, twice
    const bool turns = p.cos_sin != nullptr && 8 * l < p.rotary_dim;
    if (turns) {
        const float* const t = p.cos_sin + (int64_t)pos * p.rotary_dim;
        // (either way the lane's four pairs are 4 l .. 4 l + 3)
        const float4 x = __ldg(reinterpret_cast<const float4*>(t) + l);
        const float4 y = __ldg(reinterpret_cast<const float4*>(t + (p.rotary_dim >> 1)) + l);
        c[0] = x.x; c[1] = x.y; c[2] = x.z; c[3] = x.w;
        s[0] = y.x; s[1] = y.y; s[2] = y.z; s[3] = y.w;
    }
    const int heads = p.n_q + p.n_k + p.n_v;
    for (int h0 = 0; h0 < heads; h0 += GROUPS) {
        const int h = h0 + group;
        const bool live = h < heads;                          // (the whole warp stays: its lanes exchange values)
        const int kind = h < p.n_q ? 0 : h < p.n_q + p.n_k ? 1 : 2;
        const int head = h - (kind == 0 ? 0 : kind == 1 ? p.n_q : p.n_q + p.n_k);
        const uint16_t* const src = (kind == 0 ? p.q + row * p.q_stride : kind == 1 ? p.k + row * p.k_stride : p.v + row * p.v_stride) + head * D;
        const uint16_t* const w = kind == 0 ? p.q_weight : kind == 1 ? p.k_weight : nullptr;
        const RowDims at = kind == 2 ? RowDims{8 * l, 8 * l + 4} : turned;
        uint2 u = make_uint2(0, 0), v = make_uint2(0, 0);
        if (live) {
            u = *reinterpret_cast<const uint2*>(src + at.a);
            v = *reinterpret_cast<const uint2*>(src + at.b);
        }
        float x[8];
        {
            const float2 a0 = rows_pair<F16>(u.x), a1 = rows_pair<F16>(u.y), b0 = rows_pair<F16>(v.x), b1 = rows_pair<F16>(v.y);
            x[0] = a0.x; x[1] = a0.y; x[2] = a1.x; x[3] = a1.y;
            x[4] = b0.x; x[5] = b0.y; x[6] = b1.x; x[7] = b1.y;
        }
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = fmaf(x[i], x[i], sum);
#pragma unroll
        for (int off = L / 2; off >= 1; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
        if (live && w != nullptr) {
            const uint16_t* const wr = w + head * (kind == 0 ? p.q_weight_stride : p.k_weight_stride);
            const uint2 wu = __ldg(reinterpret_cast<const uint2*>(wr + at.a)), wv = __ldg(reinterpret_cast<const uint2*>(wr + at.b));
            const float2 w0 = rows_pair<F16>(wu.x), w1 = rows_pair<F16>(wu.y), w2 = rows_pair<F16>(wv.x), w3 = rows_pair<F16>(wv.y);
            const float r = rsqrtf(sum * (1.0f / D) + p.eps);
            x[0] *= r * w0.x; x[1] *= r * w0.y; x[2] *= r * w1.x; x[3] *= r * w1.y;
            x[4] *= r * w2.x; x[5] *= r * w2.y; x[6] *= r * w3.x; x[7] *= r * w3.y;
        }
        if (turns && kind < 2) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float& a = HALVES ? x[i] : x[2 * i];
                float& b = HALVES ? x[4 + i] : x[2 * i + 1];
                const float na = a * c[i] - b * s[i];
                b = fmaf(b, c[i], a * s[i]);
                a = na;
            }
        }
        uint2 ya, yb;
        if (kind == 2) {
            ya = u;
            yb = v;
        } else {
            ya = make_uint2(rows_pack<F16>(x[0], x[1]), rows_pack<F16>(x[2], x[3]));
            yb = make_uint2(rows_pack<F16>(x[4], x[5]), rows_pack<F16>(x[6], x[7]));
        }
        uint16_t* const out = kind == 0   ? p.q_out + row * p.q_out_stride + head * D
                              : kind == 1 && p.k_out != nullptr ? p.k_out + row * p.k_out_stride + head * D
                                                                : nullptr;
        if (live && out != nullptr) {
            *reinterpret_cast<uint2*>(out + at.a) = ya;
            *reinterpret_cast<uint2*>(out + at.b) = yb;
        }
        if (!PACKED) {
            if (live && kind > 0 && page >= 0) {
                uint16_t* const pool = kind == 1 ? static_cast<uint16_t*>(p.k_cache) + page * p.k_stride_page + place * p.k_stride_token + head * p.k_stride_head
                                                 : static_cast<uint16_t*>(p.v_cache) + page * p.v_stride_page + place * p.v_stride_token + head * p.v_stride_head;
                *reinterpret_cast<uint2*>(pool + at.a) = ya;
                *reinterpret_cast<uint2*>(pool + at.b) = yb;
            }
        } else {
            // Eight neighbouring dims to a lane: run g of four dims lies with lane g (its first run), g - n (its second)
            // or, where nothing turns, lane g / 2.
            uint32_t z[4] = {ya.x, ya.y, yb.x, yb.y};
            if (HALVES) {
                const int n = p.rotary_dim >> 3, base = threadIdx.x & 31 & ~(L - 1);
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int g = 2 * l + half;
                    const int from = kind == 2 || g >= 2 * n ? g >> 1 : g < n ? g : g - n;
                    const bool second = kind == 2 || g >= 2 * n ? (g & 1) : g >= n;
                    const uint32_t a0 = __shfl_sync(0xffffffffu, ya.x, base + from), a1 = __shfl_sync(0xffffffffu, ya.y, base + from);
                    const uint32_t b0 = __shfl_sync(0xffffffffu, yb.x, base + from), b1 = __shfl_sync(0xffffffffu, yb.y, base + from);
                    z[2 * half] = second ? b0 : a0;
                    z[2 * half + 1] = second ? b1 : a1;
                }
            }
            float y[8], amax = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 f = rows_pair<F16>(z[i]);
                y[2 * i] = f.x;
                y[2 * i + 1] = f.y;
                amax = fmaxf(amax, fmaxf(fabsf(f.x), fabsf(f.y)));
            }
            amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));      // the four lanes of a block of 32 dims
            amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
            if (live && kind > 0 && page >= 0) {
                const __half scale = packed_scale(amax);
                char* const tile = static_cast<char*>(p.k_cache) + page * p.k_stride_page + head * p.k_stride_head +
                                   (place >> 4) * packed_tile_bytes(D);
                const int r = place & 15, block = l >> 2;
                uint32_t* const codes = reinterpret_cast<uint32_t*>(tile + (kind == 1 ? 0 : packed_v_codes(D)));
                codes[kind == 1 ? packed_k_word(D, r, l) : packed_v_word(D, r, l)] = packed_word(y, scale);
                if ((l & 3) == 0) {
                    __half* const scales = reinterpret_cast<__half*>(tile + (kind == 1 ? packed_k_scales(D) : packed_v_scales(D)));
                    scales[kind == 1 ? packed_k_scale(D, r, block) : packed_v_scale(r, block)] = scale;
                }
            }
        }
    }
}

}  // namespace da
