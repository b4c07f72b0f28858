// What the instances of the prompt attention's kernels (prompt_instances.cu) tell its entry point.
#pragma once

#include <stddef.h>

namespace rt {

struct PromptKernels {
    const void* attention[3];  // heads up to 64, 128, 256
    size_t smem[3];
    const void* merge;
};
PromptKernels prompt_kernels_bf16();
PromptKernels prompt_kernels_fp16();

}  // namespace rt
