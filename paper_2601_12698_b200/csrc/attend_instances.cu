// Instances of the attention kernels for one element type (RT_UNIT_T) and one cache format (RT_UNIT_FMT); the build
// script compiles this file once per combination.
#include "attend_host.h"
#include "attend_keys_kernel.cuh"
#include "attend_merge_kernel.cuh"
#include "attend_prefix_kernel.cuh"

#define RT_CONCAT_(a, b) a##b
#define RT_CONCAT(a, b) RT_CONCAT_(a, b)

namespace {

template <int DP>
rt::AttendKernels kernels()
{
    using namespace rt;
    using T = RT_UNIT_T;
    constexpr int FMT = RT_UNIT_FMT;
    AttendKernels a;
    if constexpr (DP <= 128)  // heads of 256 leave tensor memory no room for two streams
        a.k[kPrefixTiles] = {(const void*)attend_prefix_kernel<T, FMT, DP>, PrefixShape<FMT, DP>::kSmem};
    a.k[kKeys16] = {(const void*)attend_keys_kernel<T, FMT, DP, 16>, KeysShape<FMT, DP, 16>::kSmem};
    a.k[kKeys64] = {(const void*)attend_keys_kernel<T, FMT, DP, 64>, KeysShape<FMT, DP, 64>::kSmem};
    a.k[kMergeParts] = {(const void*)merge_parts_kernel<T, DP>, 0};
    return a;
}

}  // namespace

rt::AttendKernels RT_CONCAT(rt_attend_kernels_, RT_UNIT_NAME)(int padded_dim)
{
    return padded_dim == 64 ? kernels<64>() : padded_dim == 128 ? kernels<128>() : kernels<256>();
}
