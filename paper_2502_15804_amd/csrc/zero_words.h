// Clears memory with a fill kernel, not a memset: a caller may record the call into a HIP graph, where memset nodes are best avoided.
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstddef>
#include <cstdint>

namespace fairkv {

static __global__ __launch_bounds__(256) void fairkv_zero_words_kernel(uint32_t *p, size_t n_words)
{
    for (size_t i = static_cast<size_t>(blockIdx.x) * 256 + threadIdx.x; i < n_words; i += static_cast<size_t>(gridDim.x) * 256)
        p[i] = 0u;
}
inline void zero_words(void *p, size_t n_words, hipStream_t st)
{
    const unsigned blocks = static_cast<unsigned>(std::min<size_t>((n_words + 255) / 256, 1024));
    hipLaunchKernelGGL(fairkv_zero_words_kernel, dim3(blocks), dim3(256), 0, st, static_cast<uint32_t *>(p), n_words);
}

}  // namespace fairkv
