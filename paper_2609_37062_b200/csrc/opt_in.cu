#include "opt_in.h"

#include <mutex>

#include "decode_attn.h"

namespace da {

int opt_in_shared_memory(const void* kernel, int bytes)
{
    struct Entry {
        int device;
        const void* kernel;
    };
    static std::mutex mu;
    static Entry known[512];                                  // (an array: nothing here may throw)
    static int n_known = 0;
    int device = -1;
    if (cudaGetDevice(&device) != cudaSuccess) {
        (void)cudaGetLastError();
        return DA_ERR_CUDA;
    }
    std::lock_guard<std::mutex> lock(mu);
    for (int i = 0; i < n_known; ++i)
        if (known[i].kernel == kernel && known[i].device == device) return DA_OK;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) {
        (void)cudaGetLastError();
        return DA_ERR_CUDA;
    }
    if (n_known < 512) known[n_known++] = {device, kernel};
    return DA_OK;
}

}  // namespace da
