// The entry point of the attention over a shared prefix with everything below it replaced by stand-ins, so that its plan
// and the arguments of its launches can be looked at without a GPU (see test_attention_plan_host.py).
#include "../paper_2601_12698_b200/csrc/shared_prefix_attention.cu"

struct Launch {
    int32_t kernel;  // kPrefixTiles, kKeys16, kKeys64, kMergeParts
    int32_t threads;
    int64_t ctas;
    int32_t prefix_parts, suffix_parts, prefix_ctas, run;
    int64_t part_out, part_lse;  // 0: NULL
};

namespace {

Launch g_launches[8];
int g_n = 0, g_status = 0, g_sm_count = 148;

rt::AttendKernels stand_ins()
{
    rt::AttendKernels a;
    for (int i = 0; i < rt::kAttendKernels; ++i) a.k[i].fn = (const void*)(uintptr_t)(i + 1);
    return a;
}

}  // namespace

#define RT_DEFINE(name) rt::AttendKernels rt_attend_kernels_##name(int) { return stand_ins(); }
RT_ATTEND_UNITS(RT_DEFINE)

namespace rt {

void set_error(const char*, ...) {}
int check_cache(const rt_kv_cache*, bool) { return RT_OK; }
int log2_or_minus1(unsigned) { return -1; }
unsigned wait_poll_limit() { return kMbarrierPollLimit; }
int drop_copies() { return 0; }
int* device_status_word() { return &g_status; }
int current_device_index(int* index) { *index = 0; return RT_OK; }
int current_limits(rt_limits* out)
{
    memset(out, 0, sizeof(*out));
    out->sm_count = g_sm_count;
    return RT_OK;
}
int launch_kernel(const void* fn, dim3 grid, dim3 block, size_t, cudaStream_t, void** params)
{
    const AttendArgs& a = *(const AttendArgs*)params[0];
    Launch& l = g_launches[g_n++];
    l.kernel = (int)(uintptr_t)fn - 1;
    l.threads = (int)block.x;
    l.ctas = grid.x;
    l.prefix_parts = a.prefix_parts;
    l.suffix_parts = a.suffix_parts;
    l.prefix_ctas = l.kernel == kKeys16 || l.kernel == kKeys64 ? *(const int*)params[1] : 0;
    l.run = l.kernel == kPrefixTiles || l.kernel == kMergeParts ? ((const PrefixSplit*)params[1])->run : 0;
    l.part_out = (int64_t)(uintptr_t)a.part_out;
    l.part_lse = (int64_t)(uintptr_t)a.part_lse;
    return RT_OK;
}

}  // namespace rt

extern "C" {
void harness_reset(int sm_count) { g_n = 0; g_sm_count = sm_count; }
int harness_launches(Launch* out)
{
    for (int i = 0; i < g_n; ++i) out[i] = g_launches[i];
    return g_n;
}
}
