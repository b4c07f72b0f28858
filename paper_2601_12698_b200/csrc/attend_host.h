// Host-side declarations of the attention kernels' instances.
#pragma once

#include <stddef.h>

namespace rt {

// One form of a kernel and the dynamic shared memory it is launched with.
struct AttendKernel {
    const void* fn = nullptr;
    size_t smem = 0;
};
enum { kPrefixTiles = 0, kKeys16 = 1, kKeys64 = 2, kMergeParts = 3, kAttendKernels = 4 };
struct AttendKernels {
    AttendKernel k[kAttendKernels];  // fn == NULL: the form does not serve heads of that size
};

}  // namespace rt

#define RT_ATTEND_UNITS(X) X(bf16_plain) X(bf16_e4m3) X(bf16_int8) X(fp16_plain) X(fp16_e4m3) X(fp16_int8)
#define RT_DECLARE(name) rt::AttendKernels rt_attend_kernels_##name(int padded_dim);
RT_ATTEND_UNITS(RT_DECLARE)
#undef RT_DECLARE
