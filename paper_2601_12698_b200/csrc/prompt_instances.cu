// The prompt attention's kernels for one element type.
#include "prompt_host.h"
#include "prompt_kernel.cuh"

#define RT_JOIN2(a, b) a##b
#define RT_JOIN(a, b) RT_JOIN2(a, b)

namespace rt {

PromptKernels RT_JOIN(prompt_kernels_, RT_UNIT_NAME)()
{
    PromptKernels k;
    k.attention[0] = (const void*)prompt_attention_kernel<RT_UNIT_T, 64>;
    k.attention[1] = (const void*)prompt_attention_kernel<RT_UNIT_T, 128>;
    k.attention[2] = (const void*)prompt_attention_kernel<RT_UNIT_T, 256>;
    k.smem[0] = PromptShape<64>::kSmem;
    k.smem[1] = PromptShape<128>::kSmem;
    k.smem[2] = PromptShape<256>::kSmem;
    k.merge = (const void*)prompt_merge_kernel<RT_UNIT_T>;
    return k;
}

}  // namespace rt
