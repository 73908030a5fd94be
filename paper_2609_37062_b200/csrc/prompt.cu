// Launches of the prompt kernels.
#include "prompt.cuh"
#include "prompt_launch.h"

namespace da {

namespace {

int launch(const void* fn, unsigned grid, int threads, size_t smem, void** args, cudaStream_t stream)
{
    cudaLaunchConfig_t cfg;
    cfg.gridDim = dim3(grid, 1, 1);
    cfg.blockDim = dim3(threads, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelExC(&cfg, fn, args) != cudaSuccess) {
        (void)cudaGetLastError();
        return DA_ERR_CUDA;
    }
    return DA_OK;
}

// 3-D map of q: [head_dim, query head, token]; a box is 64 dims of one group's heads of an MMA tile's tokens.
int make_q_map(CUtensorMap* map, const void* q, const decode_attn_shape_t& s, int64_t rows, int group, int tokens)
{
    const CUtensorMapDataType dt = s.q_dtype == DA_DTYPE_FP16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
    encode_tiled_fn enc = get_encode_tiled();
    if (!enc) return DA_ERR_CUDA;
    const cuuint64_t dims[3] = {(cuuint64_t)s.head_dim, (cuuint64_t)s.num_q_heads, (cuuint64_t)rows};
    const cuuint64_t strides[2] = {(cuuint64_t)s.head_dim * 2, (cuuint64_t)s.num_q_heads * s.head_dim * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)group, (cuuint32_t)tokens};
    const cuuint32_t estr[3] = {1, 1, 1};
    const CUresult r = enc(map, dt, 3, const_cast<void*>(q), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                           CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? DA_OK : DA_ERR_CUDA;
}

}  // namespace

int prompt_launch(const decode_attn_shape_t& s, const PromptCall& c, cudaStream_t stream)
{
    PromptParams p;
    p.v = static_cast<const __nv_bfloat16*>(c.v_cache);
    p.block_table = c.block_table;
    p.seq_lens = c.seq_lens;
    p.out = c.out;
    p.lse = c.lse;
    p.ws = c.ws;
    p.units = c.units;
    p.block_begin = c.block_begin;
    p.merges = c.merges;
    p.status = c.status;
    p.v_stride_page = s.v_stride_page; p.v_stride_token = s.v_stride_token; p.v_stride_head = s.v_stride_head;
    p.num_pages = s.num_pages;
    p.num_q_heads = s.num_q_heads;
    p.num_kv_heads = s.num_kv_heads;
    p.max_pages_per_seq = s.max_pages_per_seq;
    p.group = s.num_q_heads / s.num_kv_heads;
    p.tokens_per_tile = kPromptRows / p.group;
    p.window = c.window;
    p.sinks = c.sinks;
    p.tile_shift = 0;
    while ((16 << p.tile_shift) < s.page_size) ++p.tile_shift;
    p.out_kind = s.out_dtype == DA_DTYPE_BF16 ? 1 : s.out_dtype == DA_DTYPE_FP16 ? 2 : 0;
    p.scale_log2 = c.scale * kLog2e;
    CUtensorMap qmap, kmap, vmap;
    int rc = make_q_map(&qmap, c.q, s, c.q_rows, p.group, p.tokens_per_tile);
    if (rc != DA_OK) return rc;
    rc = make_pool_map(&kmap, c.k_cache, s, s.k_stride_page, s.k_stride_token, s.k_stride_head);
    if (rc != DA_OK) return rc;
    rc = make_pool_map(&vmap, c.v_cache, s, s.v_stride_page, s.v_stride_token, s.v_stride_head);
    if (rc != DA_OK) return rc;
    const bool f16 = s.kv_dtype == DA_DTYPE_FP16;
    const void* fn = s.head_dim == 128 ? (f16 ? (const void*)decode_attn_prompt_kernel<128, true> : (const void*)decode_attn_prompt_kernel<128, false>)
                                       : (f16 ? (const void*)decode_attn_prompt_kernel<64, true> : (const void*)decode_attn_prompt_kernel<64, false>);
    const int smem = s.head_dim == 128 ? PromptCfg<128>::kSmemBytes : PromptCfg<64>::kSmemBytes;
    if (cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) {
        (void)cudaGetLastError();
        return DA_ERR_CUDA;
    }
    void* args[] = {&p, &qmap, &kmap, &vmap};
    rc = launch(fn, c.n_blocks, kPromptThreads, (size_t)smem, args, stream);
    if (rc != DA_OK || c.n_merges == 0) return rc;
    const void* merge = s.head_dim == 128 ? (const void*)decode_attn_prompt_merge_kernel<128> : (const void*)decode_attn_prompt_merge_kernel<64>;
    void* merge_args[] = {&p};
    return launch(merge, c.n_merges * (unsigned)(kPromptTiles * kPromptRows * (s.head_dim / 4) / 256), 256, 0, merge_args, stream);
}

}  // namespace da
