// Launches of the tensor-core kernel: which variant serves a call.  Apart from the kernel itself, so that sources that
// share its device code do not compile every variant again.
#pragma once

#include "kernel_mma.cuh"

namespace da {

// f16: q, K and V are fp16 (attention mode); else bf16.
template <int MODE>
inline mma_kernel_t mma_kernel_for(int D, int G, bool prefix = false, bool f16 = false, bool masked = false)
{
    const bool dup = G <= 4;
    if (G > 8 && MODE == kModeAttend) {   // two tiles of heads; ordinary plans only
        if (prefix) return nullptr;
        if (D == 128)
            return f16 ? (masked ? decode_attn_mma_kernel<128, false, kModeAttend, false, true, true, true>
                                 : decode_attn_mma_kernel<128, false, kModeAttend, false, true, false, true>)
                       : (masked ? decode_attn_mma_kernel<128, false, kModeAttend, false, false, true, true>
                                 : decode_attn_mma_kernel<128, false, kModeAttend, false, false, false, true>);
        if (D == 64)
            return f16 ? (masked ? decode_attn_mma_kernel<64, false, kModeAttend, false, true, true, true>
                                 : decode_attn_mma_kernel<64, false, kModeAttend, false, true, false, true>)
                       : (masked ? decode_attn_mma_kernel<64, false, kModeAttend, false, false, true, true>
                                 : decode_attn_mma_kernel<64, false, kModeAttend, false, false, false, true>);
        return nullptr;
    }
    if (masked && MODE == kModeAttend && !prefix) {
        if (D == 128)
            return f16 ? (dup ? decode_attn_mma_kernel<128, true, kModeAttend, false, true, true>
                              : decode_attn_mma_kernel<128, false, kModeAttend, false, true, true>)
                       : (dup ? decode_attn_mma_kernel<128, true, kModeAttend, false, false, true>
                              : decode_attn_mma_kernel<128, false, kModeAttend, false, false, true>);
        if (D == 64)
            return f16 ? (dup ? decode_attn_mma_kernel<64, true, kModeAttend, false, true, true>
                              : decode_attn_mma_kernel<64, false, kModeAttend, false, true, true>)
                       : (dup ? decode_attn_mma_kernel<64, true, kModeAttend, false, false, true>
                              : decode_attn_mma_kernel<64, false, kModeAttend, false, false, true>);
        return nullptr;
    }
    if (f16) {
        if (MODE != kModeAttend) return nullptr;
        if (prefix) {
            if (!dup) return nullptr;
            if (D == 128) return decode_attn_mma_kernel<128, true, kModeAttend, true, true>;
            if (D == 64) return decode_attn_mma_kernel<64, true, kModeAttend, true, true>;
            return nullptr;
        }
        if (D == 128) return dup ? decode_attn_mma_kernel<128, true, kModeAttend, false, true>
                                 : decode_attn_mma_kernel<128, false, kModeAttend, false, true>;
        if (D == 64) return dup ? decode_attn_mma_kernel<64, true, kModeAttend, false, true>
                                : decode_attn_mma_kernel<64, false, kModeAttend, false, true>;
        return nullptr;
    }
    if (prefix) {   // shared-prefix plans: attention mode, groups of up to 4 heads
        if (MODE != kModeAttend || !dup) return nullptr;
        if (D == 128) return decode_attn_mma_kernel<128, true, kModeAttend, true>;
        if (D == 64) return decode_attn_mma_kernel<64, true, kModeAttend, true>;
        return nullptr;
    }
    if (D == 128) return dup ? decode_attn_mma_kernel<128, true, MODE, false> : decode_attn_mma_kernel<128, false, MODE, false>;
    if (D == 64) return dup ? decode_attn_mma_kernel<64, true, MODE, false> : decode_attn_mma_kernel<64, false, MODE, false>;
    return nullptr;
}

inline int mma_smem_bytes(int D, int G)
{
    const bool dup = G <= 4;
    if (D == 128) return dup ? MmaCfg<128, true>::kSmemBytes : MmaCfg<128, false>::kSmemBytes;
    return dup ? MmaCfg<64, true>::kSmemBytes : MmaCfg<64, false>::kSmemBytes;
}

template <int MODE>
inline int mma_prepare(int D, int G, mma_kernel_t* fn_out, bool prefix = false, bool f16 = false, bool masked = false,
                       bool ext = false)
{
    mma_kernel_t fn = ext ? mma_ext_kernel_for(D, G, f16, masked) : mma_kernel_for<MODE>(D, G, prefix, f16, masked);
    if (!fn) return DA_ERR_UNSUPPORTED;
    if (cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, mma_smem_bytes(D, G)) != cudaSuccess) {
        (void)cudaGetLastError();
        return DA_ERR_CUDA;
    }
    *fn_out = fn;
    return DA_OK;
}

inline int mma_query_occupancy(int D, int G, int* block_threads, int* dyn_smem, bool prefix = false, bool f16 = false,
                               bool ext = false)
{
    mma_kernel_t fn;
    if (mma_prepare<kModeAttend>(D, G, &fn, prefix, f16, false, ext) != DA_OK) return -1;
    *block_threads = kMmaThreads;
    *dyn_smem = mma_smem_bytes(D, G);
    int n = 0;
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, fn, kMmaThreads, mma_smem_bytes(D, G)) != cudaSuccess) {
        (void)cudaGetLastError();
        return -1;
    }
    return n;
}

template <int MODE>
inline int mma_launch_mode(const decode_attn_shape_t& s, int G, const KernelParams& kp, const MmaExtra& ex,
                           unsigned grid, cudaStream_t stream, bool prefix = false)
{
    mma_kernel_t fn;
    // (the probe and gather modes only move 16-bit words: one variant serves both input types)
    const bool masked = MODE == kModeAttend && !prefix && kp.run_mask != nullptr &&
                        (kp.grid_exit ? kp.may_rank != 0 : kp.n_ranked > 0);
    const bool ext = MODE == kModeAttend && (kp.window > 0 || kp.logits != nullptr);
    int rc = mma_prepare<MODE>(s.head_dim, G, &fn, prefix, MODE == kModeAttend && s.kv_dtype == DA_DTYPE_FP16, masked, ext);
    if (rc != DA_OK) return rc;
    CUtensorMap kmap, vmap;
    rc = make_pool_map(&kmap, kp.k, s, s.k_stride_page, s.k_stride_token, s.k_stride_head);
    if (rc != DA_OK) return rc;
    rc = make_pool_map(&vmap, kp.v, s, s.v_stride_page, s.v_stride_token, s.v_stride_head);
    if (rc != DA_OK) return rc;
    // programmatic dependency on the kernel launched before: this kernel's blocks may become
    // resident and run their prologue while that kernel drains (see pdl_wait_primary above)
    cudaLaunchConfig_t cfg;
    cfg.gridDim = dim3(grid, 1, 1);
    cfg.blockDim = dim3(kMmaThreads, 1, 1);
    cfg.dynamicSmemBytes = (size_t)mma_smem_bytes(s.head_dim, G);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, fn, kp, kmap, vmap, G, ex) != cudaSuccess) {
        (void)cudaGetLastError();
        return DA_ERR_CUDA;
    }
    return DA_OK;
}

inline int mma_launch(const decode_attn_shape_t& s, int G, const KernelParams& kp, unsigned grid, cudaStream_t stream,
                      bool prefix = false)
{
    MmaExtra ex = {nullptr, nullptr, nullptr, 0};
    return mma_launch_mode<kModeAttend>(s, G, kp, ex, grid, stream, prefix);
}

inline int mma_gather_probe(const decode_attn_shape_t& s, int G, const KernelParams& kp, uint32_t* checksum,
                            unsigned n_units, unsigned grid, cudaStream_t stream)
{
    if (cudaMemsetAsync(checksum, 0, sizeof(uint32_t) * n_units, stream) != cudaSuccess) {
        (void)cudaGetLastError();
        return DA_ERR_CUDA;
    }
    MmaExtra ex = {checksum, nullptr, nullptr, 0};
    return mma_launch_mode<kModeProbe>(s, G, kp, ex, grid, stream);
}

inline int mma_debug_gather(const decode_attn_shape_t& s, int G, const KernelParams& kp, int seq, void* k_out,
                            void* v_out, unsigned grid, cudaStream_t stream)
{
    MmaExtra ex = {nullptr, static_cast<__nv_bfloat16*>(k_out), static_cast<__nv_bfloat16*>(v_out), seq};
    return mma_launch_mode<kModeGather>(s, G, kp, ex, grid, stream);
}

}  // namespace da
