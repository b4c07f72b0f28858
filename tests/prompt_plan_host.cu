// The entry point of the attention over packed prompts with the device below it replaced by stand-ins, so that its plan can be looked
// at without a GPU (see test_prompt_plan_host.py).
#include "../paper_2601_12698_b200/csrc/prompt_attention.cu"

namespace {
int g_status = 0;
}

namespace rt {

void set_error(const char*, ...) {}
unsigned wait_poll_limit() { return kMbarrierPollLimit; }
int drop_copies() { return 0; }
int* device_status_word() { return &g_status; }
int current_device_index(int* index) { *index = 0; return RT_OK; }
int current_limits(rt_limits* out)
{
    memset(out, 0, sizeof(*out));
    out->sm_count = 148;
    return RT_OK;
}
int launch_kernel(const void*, dim3, dim3, size_t, cudaStream_t, void**) { return RT_OK; }
PromptKernels prompt_kernels_bf16() { return {}; }
PromptKernels prompt_kernels_fp16() { return {}; }

}  // namespace rt

extern "C" unsigned harness_more_waits(int64_t k_tokens, int64_t n_seqs) { return rt::prompt_more_waits(k_tokens, n_seqs); }
