// Instances of the attention kernels for one element type (RT_UNIT_T) and one cache format (RT_UNIT_FMT); the build
// script compiles this file once per combination.
#include "attend_prefix_kernel.cuh"
#include "attend_rows_kernel.cuh"
#include "attend_host.h"

#define RT_CONCAT_(a, b) a##b
#define RT_CONCAT(a, b) RT_CONCAT_(a, b)

namespace {
template <int DP>
void tensor_core_kernel(rt::AttendKernels* k)
{
    if constexpr (DP <= 128) {  // heads of 256 leave tensor memory no room for two streams
        k->prefix_tc = (const void*)rt::attend_prefix_kernel<RT_UNIT_T, RT_UNIT_FMT, DP>;
        k->tc_smem = rt::PrefixShape<RT_UNIT_FMT, DP>::kSmem;
    }
}
}  // namespace

rt::AttendKernels RT_CONCAT(rt_attend_kernels_, RT_UNIT_NAME)(int padded_dim)
{
    using namespace rt;
    AttendKernels k;
    switch (padded_dim) {
#define RT_CASE(DP)                                                                                          \
    case DP:                                                                                                 \
        k.prefix_rows = (const void*)attend_rows_kernel<RT_UNIT_T, RT_UNIT_FMT, DP, true>;                   \
        k.suffix_rows = (const void*)attend_rows_kernel<RT_UNIT_T, RT_UNIT_FMT, DP, false>;                  \
        k.rows_smem = RowsShape<RT_UNIT_FMT, DP>::kSmem;                                                     \
        k.merge = (const void*)merge_parts_kernel<RT_UNIT_T, DP>;                                            \
        tensor_core_kernel<DP>(&k);                                                                          \
        break;
        RT_CASE(64)
        RT_CASE(128)
        RT_CASE(256)
#undef RT_CASE
    }
    return k;
}
