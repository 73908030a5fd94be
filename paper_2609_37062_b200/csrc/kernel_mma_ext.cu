// The tensor-core kernel's variants for windowed plans and plans that track attention weights, in a
// translation unit of their own so that the library compiles in parallel.
#include "kernel_mma.cuh"

namespace da {

template <int D, bool F16, bool MASKED>
static mma_kernel_t for_group(int G)
{
    if (G > 8) return decode_attn_mma_kernel<D, false, kModeAttend, false, F16, MASKED, true, true>;
    return G <= 4 ? decode_attn_mma_kernel<D, true, kModeAttend, false, F16, MASKED, false, true>
                  : decode_attn_mma_kernel<D, false, kModeAttend, false, F16, MASKED, false, true>;
}

template <int D>
static mma_kernel_t for_type(int G, bool f16, bool masked)
{
    if (masked) return f16 ? for_group<D, true, true>(G) : for_group<D, false, true>(G);
    return f16 ? for_group<D, true, false>(G) : for_group<D, false, false>(G);
}

mma_kernel_t mma_ext_kernel_for(int D, int G, bool f16, bool masked)
{
    if (!mma_supports(D, G)) return nullptr;
    return D == 128 ? for_type<128>(G, f16, masked) : for_type<64>(G, f16, masked);
}

}  // namespace da
