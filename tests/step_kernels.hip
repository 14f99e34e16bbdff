// Instantiations of the kernels of a step over a growing cache, and the helper that fetches their tiles behind the least favourable
// instruction in front of it (a vector instruction that wrote its base).  Compiled to assembly by test_step_assembly.py.
#include "append_rotated.h"
#include "decode_tree.h"
template __global__ void fairkv::fairkv_decode_tree_kernel<128, false, 1, 4, 2, 2>(fairkv::TreeArgs);
template __global__ void fairkv::fairkv_decode_tree_kernel<64, true, 1, 4, 2, 3>(fairkv::TreeArgs);
template __global__ void fairkv::fairkv_decode_tree_kernel<128, false, 2, 4, 2, 3>(fairkv::TreeArgs);
template __global__ void fairkv::fairkv_decode_tree_kernel<128, false, 4, 2, 3, 1>(fairkv::TreeArgs);
template __global__ void fairkv::fairkv_decode_tree_kernel<128, true, 8, 1, 4, 1>(fairkv::TreeArgs);
template __global__ void fairkv::fairkv_append_rotated_kernel<uint16_t, uint16_t, 128>(fairkv::RotateArgs);
template __global__ void fairkv::fairkv_append_rotated_kernel<uint16_t, uint8_t, 64>(fairkv::RotateArgs);
template __global__ void fairkv::fairkv_append_rotated_kernel<float, float, 128>(fairkv::RotateArgs);
template __global__ void fairkv::fairkv_accept_kernel<256>(fairkv::AcceptArgs);

template <int N>
__device__ __forceinline__ void chunks(const float *const *bases, float *out)
{
    __shared__ __attribute__((aligned(1024))) char lds[N * 1040];
    const uint32_t at = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(FAIRKV_LDS_PTR(lds)));
    uint32_t off[N];
    for (int i = 0; i < N; ++i) off[i] = 48 + threadIdx.x * 16 - 16 * i;
    fairkv::load_chunks_to_lds<N, 1040>(fairkv::uniform_ptr(bases[threadIdx.x / 64]), off, at);
    fairkv::wait_vmcnt<0>();
    out[threadIdx.x] = reinterpret_cast<const float *>(lds)[threadIdx.x];
}
extern "C" __global__ void chunks2(const float *const *bases, float *out) { chunks<2>(bases, out); }
extern "C" __global__ void chunks4(const float *const *bases, float *out) { chunks<4>(bases, out); }
