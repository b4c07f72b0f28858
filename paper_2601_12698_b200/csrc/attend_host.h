// Host-side declarations of the attention kernels' instances.
#pragma once

#include <stddef.h>

namespace rt {

struct AttendKernels {
    const void* prefix_rows = nullptr;
    const void* suffix_rows = nullptr;
    const void* merge = nullptr;
    size_t rows_smem = 0;
    const void* prefix_tc = nullptr;  // tensor-core form of the prefix; NULL for heads that it does not serve
    size_t tc_smem = 0;
};

}  // namespace rt

#define RT_ATTEND_UNITS(X) X(bf16_plain) X(bf16_e4m3) X(bf16_int8) X(fp16_plain) X(fp16_e4m3) X(fp16_int8)
#define RT_DECLARE(name) rt::AttendKernels rt_attend_kernels_##name(int padded_dim);
RT_ATTEND_UNITS(RT_DECLARE)
#undef RT_DECLARE
