// Host side of decode_attn_evict.
#include <algorithm>
#include <cstring>
#include <mutex>
#include <new>

#include "evict.cuh"
#include "planner.h"

using namespace da;

namespace {

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// The numbers of a call: what decode_attn_evict and decode_attn_validate_evict both ask of them.
int check_numbers(const decode_attn_shape_t& s, const decode_attn_evict_args_t& a)
{
    if (a.struct_size != sizeof(decode_attn_evict_args_t) || a.flags != 0) return DA_ERR_INVALID_ARG;
    if (a.budget_tokens < 1 || a.sink_tokens < 0 || a.recent_tokens < 0 ||
        (int64_t)a.sink_tokens + a.recent_tokens > a.budget_tokens)
        return DA_ERR_INVALID_ARG;
    if (a.dst_max_pages < 0 || (int64_t)a.dst_max_pages * s.page_size < a.budget_tokens) return DA_ERR_INVALID_ARG;
    return DA_OK;
}

// Blocks of a kernel that the current device holds at once, with the most shared memory its launches ask for (kept after the
// first query); 0 if that cannot be told.
int64_t resident_blocks(const void* fn, int threads, size_t smem)
{
    struct Entry {
        int device;
        const void* fn;
        int64_t blocks;
    };
    static std::mutex mu;
    static Entry known[64];                                   // (four kernels; nothing here may throw)
    static int n_known = 0;
    int dev = -1, per_sm = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) {
        (void)cudaGetLastError();
        return 0;
    }
    std::lock_guard<std::mutex> lock(mu);
    for (int i = 0; i < n_known; ++i)
        if (known[i].device == dev && known[i].fn == fn) return known[i].blocks;
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess ||
        cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, fn, threads, smem) != cudaSuccess) {
        (void)cudaGetLastError();
        return 0;
    }
    if (n_known < 64) known[n_known++] = {dev, fn, (int64_t)sms * per_sm};
    return (int64_t)sms * per_sm;
}

int launch(const void* fn, dim3 grid, int threads, size_t smem, EvictParams& ep, cudaStream_t stream)
{
    cudaLaunchConfig_t cfg;
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    void* args[] = {&ep};
    if (cudaLaunchKernelExC(&cfg, fn, args) != cudaSuccess) {
        (void)cudaGetLastError();
        return DA_ERR_CUDA;
    }
    return DA_OK;
}

}  // namespace

extern "C" int decode_attn_evict(const decode_attn_shape_t* shape, const decode_attn_evict_args_t* a, cudaStream_t stream)
{
    if (!shape || !a) return DA_ERR_INVALID_ARG;
    const decode_attn_shape_t& s = *shape;
    int rc = validate_shape(s);
    if (rc != DA_OK) return rc;
    rc = check_numbers(s, *a);
    if (rc != DA_OK) return rc;
    if (s.batch == 0) return DA_OK;
    if (!a->seq_lens || !a->block_table || !a->dst_block_table || !a->k_cache || !a->v_cache || !a->weights ||
        !a->weights_out || !a->kept || !a->seq_lens_out)
        return DA_ERR_INVALID_ARG;
    if (!aligned(a->k_cache, 16) || !aligned(a->v_cache, 16) || !aligned(a->weights, 4) || !aligned(a->weights_out, 4) ||
        !aligned(a->seq_lens, 4) || !aligned(a->block_table, 4) || !aligned(a->dst_block_table, 4) || !aligned(a->kept, 4) ||
        !aligned(a->seq_lens_out, 4) || !aligned(a->status, 4))
        return DA_ERR_INVALID_ARG;
    if (a->seq_lens_out == a->seq_lens) return DA_ERR_INVALID_ARG;   // the blocks of one row would see its new length
    if (a->weight_tokens < 1 || !totals_apart(a->weight_tokens, a->stride_seq, a->stride_head, s.batch, s.num_kv_heads))
        return DA_ERR_INVALID_ARG;

    EvictParams ep;
    ep.seq_lens = a->seq_lens;
    ep.block_table = a->block_table;
    ep.dst_block_table = a->dst_block_table;
    ep.k = static_cast<__nv_bfloat16*>(a->k_cache);
    ep.v = static_cast<__nv_bfloat16*>(a->v_cache);
    ep.weights = a->weights;
    ep.weights_out = a->weights_out;
    ep.kept = a->kept;
    ep.seq_lens_out = a->seq_lens_out;
    ep.status = a->status;
    ep.weight_tokens = a->weight_tokens;
    ep.stride_seq = a->stride_seq;
    ep.stride_head = a->stride_head;
    ep.k_stride_page = s.k_stride_page; ep.k_stride_token = s.k_stride_token; ep.k_stride_head = s.k_stride_head;
    ep.v_stride_page = s.v_stride_page; ep.v_stride_token = s.v_stride_token; ep.v_stride_head = s.v_stride_head;
    ep.num_pages = s.num_pages;
    ep.batch = s.batch;
    ep.num_kv_heads = s.num_kv_heads;
    ep.max_pages_per_seq = s.max_pages_per_seq;
    ep.dst_max_pages = a->dst_max_pages;
    ep.page_shift = 0;
    while ((1 << ep.page_shift) < s.page_size) ++ep.page_shift;
    ep.budget = a->budget_tokens;
    ep.sinks = a->sink_tokens;
    ep.recent = a->recent_tokens;

    // The longest row that the tables and the totals can hold sizes the select launch.
    const int64_t most = std::max<int64_t>(1, std::min<int64_t>((int64_t)s.max_pages_per_seq * s.page_size, a->weight_tokens));
    ep.chunk = (int32_t)std::min<int64_t>((most + 31) / 32 * 32, kEvictChunk);
    const size_t smem = (size_t)ep.chunk * sizeof(float);
    const int64_t rows = (int64_t)s.batch * s.num_kv_heads;
    const int64_t units = rows * ((ep.budget + kMoveTokens - 1) / kMoveTokens);
    const int64_t move_blocks = (units + kMoveThreads / 32 - 1) / (kMoveThreads / 32);
    if (rows > 0x7fffffffLL || move_blocks > 0x7fffffffLL) return DA_ERR_UNSUPPORTED;
    // up to 2,048 totals small blocks, several to an SM; up to 8,192 and 32,768 larger ones whose threads still hold all
    // keys (8 rows of 4,100 totals: 12.8 us with blocks of 512, 17.7 with the 1,024 that longer rows take)
    const int threads = most <= 2048 ? 256 : most <= 8192 ? 512 : 1024;
    // One launch where every warp of a block moves once (32 tokens) and all blocks are resident at once.  Rows of 1,500
    // totals, 256 tokens of 128 dims kept: 128 rows 15.0 us against 16.9 in two launches, 440 rows 23.1 against 25.8; 384
    // kept: 23.2 against 19.2.  Rows of 4,000, 512 kept: 128 rows 19.1 against 22.8, 256 rows (two waves) 43 against 33.
    // (Blocks of 1,024 threads have no registers to spare for it: 19 -> 24 us.)
    const bool wide = s.head_dim == 128;
    const void* const mover = most > 2048 ? (wide ? (const void*)decode_attn_evict_select_kernel<512, 1024, 16, 128>
                                                  : (const void*)decode_attn_evict_select_kernel<512, 1024, 16, 64>)
                                          : (wide ? (const void*)decode_attn_evict_select_kernel<256, 1024, 8, 128>
                                                  : (const void*)decode_attn_evict_select_kernel<256, 1024, 8, 64>);
    const bool one = most <= 8192 && ep.budget <= threads / 32 * kMoveTokens &&
                     rows <= resident_blocks(mover, threads, (most <= 2048 ? 2048 : 8192) * sizeof(float));
    const void* select = one           ? mover
                         : most > 8192 ? (const void*)decode_attn_evict_select_kernel<1024, 2048, 32, 0>
                         : most > 2048 ? (const void*)decode_attn_evict_select_kernel<512, 1024, 16, 0>
                                       : (const void*)decode_attn_evict_select_kernel<256, 1024, 8, 0>;
    const void* move = wide ? (const void*)decode_attn_evict_move_kernel<128> : (const void*)decode_attn_evict_move_kernel<64>;
    if (smem > 32 * 1024 &&
        cudaFuncSetAttribute(select, cudaFuncAttributeMaxDynamicSharedMemorySize, kEvictChunk * (int)sizeof(float)) != cudaSuccess) {
        (void)cudaGetLastError();
        return DA_ERR_CUDA;
    }
    rc = launch(select, dim3((unsigned)rows), threads, smem, ep, stream);
    if (rc != DA_OK || one) return rc;
    return launch(move, dim3((unsigned)move_blocks), kMoveThreads, 0, ep, stream);
}

extern "C" int decode_attn_validate_evict(const decode_attn_shape_t* shape, const decode_attn_evict_args_t* a,
                                          const int32_t* seq_lens_host, const int32_t* block_table_host,
                                          const int32_t* dst_block_table_host)
{
    if (!shape || !a) return DA_ERR_INVALID_ARG;
    const decode_attn_shape_t& s = *shape;
    int rc = validate_shape(s);
    if (rc != DA_OK) return rc;
    rc = check_numbers(s, *a);
    if (rc != DA_OK) return rc;
    if (s.batch > 0 && (!seq_lens_host || !block_table_host || !dst_block_table_host)) return DA_ERR_INVALID_ARG;
    unsigned char* const used = new (std::nothrow) unsigned char[(size_t)s.num_pages]();
    if (!used) return DA_ERR_UNSUPPORTED;
    for (int b = 0; b < s.batch && rc == DA_OK; ++b) {
        const int64_t pages = ((int64_t)seq_lens_host[b] + s.page_size - 1) / s.page_size;
        if (seq_lens_host[b] < 0 || pages > s.max_pages_per_seq) rc = DA_ERR_INVALID_ARG;
        for (int64_t i = 0; i < pages && rc == DA_OK; ++i) {
            const int32_t pg = block_table_host[(int64_t)b * s.max_pages_per_seq + i];
            if (pg < 0 || pg >= s.num_pages)
                rc = DA_ERR_BAD_PAGE;
            else
                used[pg] = 1;
        }
    }
    for (int b = 0; b < s.batch && rc == DA_OK; ++b) {
        if (seq_lens_host[b] <= a->budget_tokens) continue;
        const int64_t pages = ((int64_t)a->budget_tokens + s.page_size - 1) / s.page_size;
        for (int64_t i = 0; i < pages && rc == DA_OK; ++i) {
            const int32_t pg = dst_block_table_host[(int64_t)b * a->dst_max_pages + i];
            if (pg < 0 || pg >= s.num_pages || used[pg])
                rc = DA_ERR_BAD_PAGE;                          // outside the pool, read by a row, or given out twice
            else
                used[pg] = 1;
        }
    }
    delete[] used;
    return rc;
}
