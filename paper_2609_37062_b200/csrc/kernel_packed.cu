// Launches of the kernel for caches in 4 bits.
#include "kernel_packed.cuh"
#include "kernel_packed.h"

namespace da {

namespace {

typedef void (*packed_kernel_t)(const KernelParams, const int);

template <int D, bool F16>
packed_kernel_t for_group(int G, bool ext)
{
    if (G > 8) return ext ? decode_attn_packed_kernel<D, F16, true, true> : decode_attn_packed_kernel<D, F16, true, false>;
    return ext ? decode_attn_packed_kernel<D, F16, false, true> : decode_attn_packed_kernel<D, F16, false, false>;
}

packed_kernel_t kernel_for(int D, int G, bool f16, bool ext)
{
    if (D == 128) return f16 ? for_group<128, true>(G, ext) : for_group<128, false>(G, ext);
    return f16 ? for_group<64, true>(G, ext) : for_group<64, false>(G, ext);
}

int prepare(int D, int G, bool f16, bool ext, packed_kernel_t* fn)
{
    *fn = kernel_for(D, G, f16, ext);
    const int smem = D == 128 ? PackedCfg<128>::kSmem : PackedCfg<64>::kSmem;
    if (cudaFuncSetAttribute(*fn, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) {
        (void)cudaGetLastError();
        return -1;
    }
    return smem;
}

}  // namespace

int packed_query_occupancy(int D, int G, bool ext, int* block_threads, int* dyn_smem)
{
    packed_kernel_t fn;
    const int smem = prepare(D, G, false, ext, &fn);
    if (smem < 0) return -1;
    int n = 0;
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, fn, kPackedThreads, smem) != cudaSuccess) {
        (void)cudaGetLastError();
        return -1;
    }
    *block_threads = kPackedThreads;
    *dyn_smem = smem;
    return n;
}

int packed_launch(const decode_attn_shape_t& s, int G, const KernelParams& kp, unsigned grid, cudaStream_t stream)
{
    packed_kernel_t fn;
    const int smem = prepare(s.head_dim, G, s.kv_dtype == DA_DTYPE_FP16, kp.window > 0, &fn);
    if (smem < 0) return DA_ERR_CUDA;
    cudaLaunchConfig_t cfg;
    cfg.gridDim = dim3(grid, 1, 1);
    cfg.blockDim = dim3(kPackedThreads, 1, 1);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, fn, kp, G) != cudaSuccess) {
        (void)cudaGetLastError();
        return DA_ERR_CUDA;
    }
    return DA_OK;
}

}  // namespace da
