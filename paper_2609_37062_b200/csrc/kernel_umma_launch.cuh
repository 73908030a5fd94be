// Launch of the tcgen05 kernel for shared prefixes, apart from the kernel as kernel_mma_launch.cuh is.
#pragma once

#include "kernel_umma.cuh"

namespace da {

typedef void (*umma_kernel_t)(const KernelParams, const CUtensorMap, const CUtensorMap, const int, const int);

inline int umma_prepare(bool f16, umma_kernel_t* fn_out)
{
    umma_kernel_t fn = f16 ? decode_attn_umma_prefix_kernel<true> : decode_attn_umma_prefix_kernel<false>;
    *fn_out = fn;
    if (cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, kUmmaSmemBytes) != cudaSuccess) {
        (void)cudaGetLastError();
        return DA_ERR_CUDA;
    }
    return DA_OK;
}

// Units [0, n_prefix_units) of the plan's work list, dealt round-robin to `grid` blocks (at most one per SM).
inline int umma_prefix_launch(const decode_attn_shape_t& s, int G, const KernelParams& kp, unsigned n_prefix_units,
                              unsigned grid, cudaStream_t stream)
{
    if (n_prefix_units == 0) return DA_OK;
    umma_kernel_t fn;
    int rc = umma_prepare(s.kv_dtype == DA_DTYPE_FP16, &fn);
    if (rc != DA_OK) return rc;
    CUtensorMap kmap, vmap;
    rc = make_pool_map(&kmap, kp.k, s, s.k_stride_page, s.k_stride_token, s.k_stride_head);
    if (rc != DA_OK) return rc;
    rc = make_pool_map(&vmap, kp.v, s, s.v_stride_page, s.v_stride_token, s.v_stride_head);
    if (rc != DA_OK) return rc;
    cudaLaunchConfig_t cfg;
    cfg.gridDim = dim3(grid, 1, 1);
    cfg.blockDim = dim3(kUmmaThreads, 1, 1);
    cfg.dynamicSmemBytes = (size_t)kUmmaSmemBytes;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, fn, kp, kmap, vmap, G, (int)n_prefix_units) != cudaSuccess) {
        (void)cudaGetLastError();
        return DA_ERR_CUDA;
    }
    return DA_OK;
}

}  // namespace da
