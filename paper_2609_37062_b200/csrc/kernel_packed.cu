// Launches of the kernel for caches in 4 bits.
#include "kernel_packed.cuh"
#include "kernel_packed.h"
#include "opt_in.h"

namespace da {

namespace {

typedef void (*packed_kernel_t)(const KernelParams, const int);

struct PackedVariant {
    packed_kernel_t fn;
    int threads, smem;
};

template <int D, bool F16, bool EXT, int W, int NT>
PackedVariant variant(bool dup)
{
    using Cfg = PackedCfg<D, W, NT>;
    return {dup ? decode_attn_packed_kernel<D, F16, F16 && NT == 1, EXT, W, NT> : decode_attn_packed_kernel<D, F16, false, EXT, W, NT>,
            Cfg::kThreads, Cfg::kSmem};
}

template <int D, bool F16, bool EXT>
PackedVariant for_group(int G, bool big)
{
    if (G > 8) return variant<D, F16, EXT, 4, 2>(false);
    return big ? variant<D, F16, EXT, 8, 1>(F16 && G <= 4) : variant<D, F16, EXT, 4, 1>(F16 && G <= 4);
}

template <int D>
PackedVariant for_type(int G, bool f16, bool ext, bool big)
{
    if (ext) return f16 ? for_group<D, true, true>(G, big) : for_group<D, false, true>(G, big);
    return f16 ? for_group<D, true, false>(G, big) : for_group<D, false, false>(G, big);
}

// The variant of a plan, opted in to its shared memory.
int prepare(int D, int G, bool f16, bool ext, bool big, PackedVariant* v)
{
    *v = D == 128 ? for_type<128>(G, f16, ext, big) : for_type<64>(G, f16, ext, big);
    return opt_in_shared_memory((const void*)v->fn, v->smem);
}

}  // namespace

int packed_query_occupancy(int D, int G, bool ext, bool big, int* block_threads, int* dyn_smem)
{
    PackedVariant v;
    if (prepare(D, G, false, ext, big, &v) != DA_OK) return -1;
    int n = 0;
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, v.fn, v.threads, v.smem) != cudaSuccess) {
        (void)cudaGetLastError();
        return -1;
    }
    *block_threads = v.threads;
    *dyn_smem = v.smem;
    return n;
}

int packed_launch(const decode_attn_shape_t& s, int G, bool big, const KernelParams& kp, unsigned grid, cudaStream_t stream)
{
    PackedVariant v;
    const int rc = prepare(s.head_dim, G, s.kv_dtype == DA_DTYPE_FP16, kp.window > 0, big, &v);
    if (rc != DA_OK) return rc;
    cudaLaunchConfig_t cfg;
    cfg.gridDim = dim3(grid, 1, 1);
    cfg.blockDim = dim3(v.threads, 1, 1);
    cfg.dynamicSmemBytes = (size_t)v.smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, v.fn, kp, G) != cudaSuccess) {
        (void)cudaGetLastError();
        return DA_ERR_CUDA;
    }
    return DA_OK;
}

}  // namespace da
