// The tensor-core kernel's variants for windowed plans and plans that track attention weights, in a
// translation unit of their own so that the library compiles in parallel.
#include "kernel_mma.cuh"

namespace da {

template <int D, bool F16>
static mma_kernel_t for_group(int G)
{
    if (G > 8) return decode_attn_mma_kernel<D, false, kModeAttend, false, F16, false, true, true>;
    return G <= 4 ? decode_attn_mma_kernel<D, true, kModeAttend, false, F16, false, false, true>
                  : decode_attn_mma_kernel<D, false, kModeAttend, false, F16, false, false, true>;
}

mma_kernel_t mma_ext_kernel_for(int D, int G, bool f16)
{
    if (!mma_supports(D, G)) return nullptr;
    if (D == 128) return f16 ? for_group<128, true>(G) : for_group<128, false>(G);
    return f16 ? for_group<64, true>(G) : for_group<64, false>(G);
}

}  // namespace da
