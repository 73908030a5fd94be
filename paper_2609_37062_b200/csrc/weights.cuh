// Running totals of attention weights.
//
// A plan that tracks weights leaves the logits x = scale * log2(e) * <q_h, k_t> of every visible token in
// the workspace, one [G][16] block per tile and KV head.  Once the log-sum-exp of the rows is known,
//   weights_out[b][g][t] = weights[b][g][t] + sum_{h in group g} 2^(x_ht - log2(e) * lse_h),
// the attention weight of token t summed over the query heads that share its K/V row.  A token the window
// hides adds nothing (its tile is not in the workspace, or its logit is -inf); so does a row that attended
// nothing (lse = -inf), whose logits may be from an earlier step.
//
// Bound by memory: 4 G + 8 bytes per token and KV head, a twentieth of the K/V bytes at group 4 and
// head_dim 128; recomputing the logits from K instead would read half of the K/V bytes once more.  A thread takes
// four consecutive tokens (16-byte loads of the logits, which lie head by head within a tile).
#pragma once

#include "common.cuh"

namespace da {

constexpr int kWeightsThreads = 256;
constexpr int kWeightsTokens = 4 * kWeightsThreads;   // of one (sequence, KV head) per block

struct WeightsParams {
    const float* logits;
    const float* lse;           // natural logarithm, [batch][Hq]
    const int32_t* seq_lens;
    const DevHeader* header;
    const SeqInfo* seq_info;
    const float* weights;
    float* weights_out;
    int64_t stride_seq, stride_head;
    int32_t* status;
    int32_t num_kv_heads, group, window, sinks;
    int32_t chunks;             // blocks per (sequence, KV head)
    int32_t vec;                // rows of the totals are 16-byte aligned
};

__global__ void __launch_bounds__(kWeightsThreads) decode_attn_weights_kernel(const WeightsParams p)
{
    pdl_launch_dependents();
    const int chunk = blockIdx.x % p.chunks, bg = blockIdx.x / p.chunks;
    const int b = bg / p.num_kv_heads, g = bg % p.num_kv_heads;
    const int G = p.group;
    const bool in_batch = b < p.header->batch;
    SeqInfo si;
    si.seq_len = 0;
    if (in_batch) si = p.seq_info[b];
    pdl_wait_primary();                                       // logits, log-sum-exps and totals are complete
    const int t = chunk * kWeightsTokens + 4 * (int)threadIdx.x;
    const int L = si.seq_len;
    if (t >= L) return;
    if (__ldg(p.seq_lens + b) != L) {                         // stale plan: nothing is added, reported
        if (threadIdx.x == 0) record_status(p.status, DA_ERR_STALE_PLAN);
        return;
    }
    const WindowCut cut = window_cut(L, p.window, p.sinks);
    const int tile = t >> 4;
    float a[4] = {0.f, 0.f, 0.f, 0.f};
    if (tile < cut.sink_tiles || tile >= cut.sink_tiles + cut.skip_tiles) {
        const int v = tile < cut.sink_tiles ? tile : tile - cut.skip_tiles;
        const int n_tiles = ((L + 15) >> 4) - cut.skip_tiles;
        const float* x = p.logits + logit_tile(si.tile_base, n_tiles, p.num_kv_heads, g, v, G) + (t & 15);
        const float* lse = p.lse + (int64_t)b * p.num_kv_heads * G + (int64_t)g * G;
        for (int h = 0; h < G; ++h) {
            const float e = __ldg(lse + h);
            if (e == -INFINITY) continue;
            const float4 l = __ldcg(reinterpret_cast<const float4*>(x + h * 16));
            const float e2 = e * kLog2e;
            a[0] += ex2f(l.x - e2);
            a[1] += ex2f(l.y - e2);
            a[2] += ex2f(l.z - e2);
            a[3] += ex2f(l.w - e2);
        }
    }
    const int64_t row = (int64_t)b * p.stride_seq + (int64_t)g * p.stride_head + t;
    const float* const w = p.weights + row;
    float* const o = p.weights_out + row;
    if (p.vec && t + 4 <= L) {
        float4 v = *reinterpret_cast<const float4*>(w);
        v.x += a[0]; v.y += a[1]; v.z += a[2]; v.w += a[3];
        *reinterpret_cast<float4*>(o) = v;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (t + i < L) o[i] = w[i] + a[i];
    }
}

inline int weights_launch(const WeightsParams& wp, unsigned blocks, cudaStream_t stream)
{
    cudaLaunchConfig_t cfg;
    cfg.gridDim = dim3(blocks, 1, 1);
    cfg.blockDim = dim3(kWeightsThreads, 1, 1);
    cfg.dynamicSmemBytes = 0;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, decode_attn_weights_kernel, wp) != cudaSuccess) {
        (void)cudaGetLastError();
        return DA_ERR_CUDA;
    }
    return DA_OK;
}

}  // namespace da
