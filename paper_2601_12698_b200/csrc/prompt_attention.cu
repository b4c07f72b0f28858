// Entry point of the attention over packed prompts: argument checks, the split of the work, tensor maps, the launches.
#include <string.h>

#include <algorithm>
#include <atomic>

#include "prompt_host.h"
#include "prompt_kernel.cuh"
#include "tuner_internal.h"

namespace rt {
namespace {

constexpr int64_t kMaxRows = 1LL << 30;
constexpr int kMaxGroup = 128;

struct PromptPlan {
    int form;  // index of the kernel: heads up to 64, 128, 256
    int group, stream_tokens, block_tokens, parts;
    long long ctas;
    int64_t workspace;
};

long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

int check_geometry(const rt_prompt_batch* b, int q_heads, int kv_heads, int dim)
{
    if (!b) {
        set_error("batch is NULL");
        return RT_ERR_NULL;
    }
    if (b->n_seqs < 0 || b->n_seqs > (1LL << 24) || b->q_tokens < 0 || b->q_tokens > kMaxRows || b->k_tokens < 0 || b->k_tokens > kMaxRows ||
        b->max_q_len < 0 || b->max_k_len < 0) {
        set_error("n_seqs=%lld q_tokens=%lld k_tokens=%lld or a length out of range", (long long)b->n_seqs, (long long)b->q_tokens, (long long)b->k_tokens);
        return RT_ERR_SHAPE;
    }
    if (kv_heads < 1 || kv_heads > 65535 || q_heads < kv_heads || q_heads % kv_heads || q_heads / kv_heads > kMaxGroup) {
        set_error("q_heads=%d is not 1 .. %d times kv_heads=%d", q_heads, kMaxGroup, kv_heads);
        return RT_ERR_SHAPE;
    }
    if (dim < 8 || dim > RT_KV_MAX_HEAD_DIM || dim % 8) {
        set_error("head_dim=%d is not a multiple of 8 up to %d", dim, RT_KV_MAX_HEAD_DIM);
        return RT_ERR_SHAPE;
    }
    return RT_OK;
}

int make_prompt_plan(const rt_prompt_batch* b, int q_heads, int kv_heads, int dim, PromptPlan* p)
{
    rt_limits L;
    const int st = current_limits(&L);
    if (st != RT_OK) return st;
    memset(p, 0, sizeof(*p));
    p->form = dim <= 64 ? 0 : dim <= 128 ? 1 : 2;
    p->group = q_heads / kv_heads;
    p->stream_tokens = kPromptTile / p->group;
    p->block_tokens = p->form == 2 ? p->stream_tokens : 2 * p->stream_tokens;
    // (no sequence is longer than the tensors, whatever the batch says)
    const long long max_q_len = std::min(b->max_q_len, b->q_tokens), max_k_len = std::min(b->max_k_len, b->k_tokens);
    // Blocks: as many as there are full ones, and a ragged one of each sequence.
    const long long blocks = b->q_tokens / p->block_tokens + b->n_seqs;
    const long long expected = std::min(blocks, b->n_seqs * ceil_div(max_q_len, p->block_tokens)) * kv_heads, tiles = ceil_div(max_k_len, kPromptTile);
    // Blocks that do not fill the device evenly, against many keys: the keys are cut into parts, as many as end first by a model of whole
    // waves of items: a key tile takes 1.7 us (2.3 with heads of more than 128), beginning and ending an item 3, joining the parts 3 and
    // the time to write and read them at 5 TB/s.  512 tokens behind 16000, 40 heads on 8 of 128, 88 blocks: 242 us in one part, 215 in three (237 and 189 on another card).
    // Blocks of two waves and more are left whole: their order evens them out.
    p->parts = 1;
    if (expected > 0 && expected < 2LL * L.sm_count && b->q_tokens / p->block_tokens * kv_heads < 2LL * L.sm_count && tiles >= 8) {
        const double tile_us = p->form == 2 ? 2.3 : 1.7, part_us = (double)b->q_tokens * q_heads * dim * 8 / 5e6;
        double best = 0;
        for (int parts = 1; parts <= std::min<long long>(kPromptMaxParts, tiles / 2); ++parts) {
            const double time = (double)ceil_div(expected * parts, L.sm_count) * (ceil_div(tiles, parts) * tile_us + 3) + (parts > 1 ? 3 + parts * part_us : 0);
            if (parts == 1 || time < best * 0.95) {
                best = time;
                p->parts = parts;
            }
        }
    }
    p->ctas = std::min<long long>(L.sm_count, blocks * kv_heads * p->parts);
    const int64_t rows = b->q_tokens * q_heads;
    if (p->parts > 1) p->workspace = (int64_t)p->parts * rows * dim * 4 + ((int64_t)p->parts * rows * 4 + 4 + 15) / 16 * 16;  // results, logarithms, a flag
    return RT_OK;
}

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled()
{
    static const EncodeTiled fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) p = nullptr;
        return (EncodeTiled)p;
    }();
    return fn;
}

// [tokens, heads, dim] with the strides in elements; a box is 64 dims of `box_heads` heads of `box_tokens` tokens, in the 128-byte swizzle.
int make_map(CUtensorMap* map, const void* data, int dtype, int dim, int heads, long long tokens, long long head_stride, long long token_stride,
             int box_heads, int box_tokens)
{
    const EncodeTiled encode = encode_tiled();
    if (!encode) {
        set_error("the driver has no cuTensorMapEncodeTiled");
        return RT_ERR_CUDA;
    }
    const cuuint64_t row = (cuuint64_t)(dim * 2 + 15) / 16 * 16;  // (of an axis with one entry the stride says nothing)
    const cuuint64_t sizes[3] = {(cuuint64_t)dim, (cuuint64_t)heads, (cuuint64_t)tokens};
    const cuuint64_t strides[2] = {heads > 1 ? (cuuint64_t)head_stride * 2 : row, tokens > 1 ? (cuuint64_t)token_stride * 2 : row * heads};
    const cuuint32_t box[3] = {64, (cuuint32_t)box_heads, (cuuint32_t)box_tokens}, steps[3] = {1, 1, 1};
    const CUresult r = encode(map, dtype == RT_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(data), sizes, strides,
                              box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) {
        set_error("no tensor map for head_dim=%d heads=%d tokens=%lld, strides %lld and %lld (driver error %d)", dim, heads, tokens, head_stride, token_stride, (int)r);
        return RT_ERR_CUDA;
    }
    return RT_OK;
}

// Shared memory beyond the default limit is asked for once per device and kernel.
int allow_smem(const PromptKernels& k, int dtype, int form)
{
    static std::atomic<unsigned char> done[kDeviceSlots][2][3];
    int device;
    const int st = current_device_index(&device);
    if (st != RT_OK) return st;
    if (!done[device][dtype][form].load(std::memory_order_acquire)) {
        RT_CUDA_OK(cudaFuncSetAttribute(k.attention[form], cudaFuncAttributeMaxDynamicSharedMemorySize, (int)k.smem[form]));
        done[device][dtype][form].store(1, std::memory_order_release);
    }
    return RT_OK;
}

}  // namespace
}  // namespace rt

extern "C" {

int64_t prompt_attention_workspace_bytes(const rt_prompt_batch* batch, int32_t q_heads, int32_t kv_heads, int32_t head_dim)
{
    rt::PromptPlan p;
    if (rt::check_geometry(batch, q_heads, kv_heads, head_dim) != RT_OK || rt::make_prompt_plan(batch, q_heads, kv_heads, head_dim, &p) != RT_OK) return -1;
    return p.workspace;
}

int prompt_attention_launch(const rt_prompt_batch* b, const void* q, int64_t q_token_stride, int64_t q_head_stride, int32_t q_heads, const void* k,
                            int64_t k_token_stride, int64_t k_head_stride, const void* v, int64_t v_token_stride, int64_t v_head_stride,
                            int32_t kv_heads, int32_t head_dim, void* out, float* lse, float softmax_scale, int dtype, void* workspace,
                            int64_t workspace_bytes, void* stream)
{
    using namespace rt;
    if (dtype != RT_BF16 && dtype != RT_FP16) {
        set_error("dtype %d is not bf16 or fp16", dtype);
        return RT_ERR_DTYPE;
    }
    int st = check_geometry(b, q_heads, kv_heads, head_dim);
    if (st != RT_OK) return st;
    if (!(softmax_scale >= 0.f) || !(softmax_scale < INFINITY)) {
        set_error("softmax_scale=%g is not finite or negative", (double)softmax_scale);
        return RT_ERR_SHAPE;
    }
    if (b->q_tokens == 0 || b->n_seqs == 0) return RT_OK;
    if (!q || !out || !b->q_starts || !b->k_starts || (b->k_tokens > 0 && (!k || !v))) {
        set_error("a tensor pointer is NULL");
        return RT_ERR_NULL;
    }
    const int64_t strides[6] = {b->q_tokens > 1 ? q_token_stride : 8, q_heads > 1 ? q_head_stride : 8, b->k_tokens > 1 ? k_token_stride : 8,
                                kv_heads > 1 ? k_head_stride : 8, b->k_tokens > 1 ? v_token_stride : 8, kv_heads > 1 ? v_head_stride : 8};
    for (int64_t s : strides) {
        if (s <= 0 || s >= (1LL << 39)) {
            set_error("a stride of %lld elements is out of range", (long long)s);
            return RT_ERR_SHAPE;
        }
        if (s % 8) {
            set_error("a stride of %lld elements is not a multiple of 16 bytes", (long long)s);
            return RT_ERR_ALIGN;
        }
    }
    const uintptr_t kv = b->k_tokens > 0 ? (uintptr_t)k | (uintptr_t)v : 0;
    if ((((uintptr_t)q | kv | (uintptr_t)out | (uintptr_t)workspace) & 15u) || (((uintptr_t)lse | (uintptr_t)b->q_starts | (uintptr_t)b->k_starts) & 3u)) {
        set_error("q, k, v, out and workspace must be multiples of 16 bytes, the other tensors of 4");
        return RT_ERR_ALIGN;
    }
    if (b->k_tokens > 0 && (out == k || out == v)) {  // (some rows' keys and values would be other rows' results)
        set_error("out overlaps k or v");
        return RT_ERR_SHAPE;
    }
    PromptPlan p;
    if ((st = make_prompt_plan(b, q_heads, kv_heads, head_dim, &p)) != RT_OK) return st;
    if (p.workspace > 0 && !workspace) {
        set_error("workspace is NULL");
        return RT_ERR_NULL;
    }
    if (workspace_bytes < p.workspace) {
        set_error("workspace of %lld bytes, %lld are needed", (long long)workspace_bytes, (long long)p.workspace);
        return RT_ERR_CAPACITY;
    }
    PromptArgs a;
    memset(&a, 0, sizeof(a));
    a.q_starts = b->q_starts;
    a.k_starts = b->k_starts;
    a.n_seqs = (int)b->n_seqs;
    a.q_tokens = (int)b->q_tokens;
    a.k_tokens = (int)b->k_tokens;
    a.causal = b->causal != 0;
    a.kv_heads = kv_heads;
    a.group = p.group;
    a.group_inverse = (65536 + p.group - 1) / p.group;
    a.dim = head_dim;
    a.stream_tokens = p.stream_tokens;
    a.block_tokens = p.block_tokens;
    a.parts = p.parts;
    a.score_scale = softmax_scale * 1.4426950408889634f;
    a.v = (const unsigned char*)v;
    a.v_token_stride = v_token_stride * 2;
    a.v_head_stride = kv_heads > 1 ? v_head_stride * 2 : 0;
    a.out = out;
    a.lse = lse;
    if (p.parts > 1) {
        a.part_out = (float*)workspace;
        a.part_lse = a.part_out + (int64_t)p.parts * b->q_tokens * q_heads * head_dim;
        a.part_ready = (int*)(a.part_lse + (int64_t)p.parts * b->q_tokens * q_heads);
    }
    // (binary32 parts of heads that are multiples of 8 are)
    a.wide_rows = p.parts > 1 ? (uintptr_t)workspace % 32 == 0 : head_dim % 16 == 0 && (uintptr_t)out % 32 == 0;
    a.status = device_status_word();
    if (!a.status) return RT_ERR_NO_DEVICE;
    a.wait_polls = wait_poll_limit();
    a.more_waits = prompt_more_waits(b->k_tokens, b->n_seqs);
    a.drop_copies = drop_copies();
    const PromptKernels kernels = dtype == RT_BF16 ? prompt_kernels_bf16() : prompt_kernels_fp16();
    if ((st = allow_smem(kernels, dtype, p.form)) != RT_OK) return st;
    CUtensorMap q_map, k_map, v_map;
    memset(&k_map, 0, sizeof(k_map));
    memset(&v_map, 0, sizeof(v_map));
    if ((st = make_map(&q_map, q, dtype, head_dim, q_heads, b->q_tokens, q_head_stride, q_token_stride, p.group, p.stream_tokens)) != RT_OK) return st;
    if (b->k_tokens > 0) {  // (without keys no tile is fetched)
        if ((st = make_map(&k_map, k, dtype, head_dim, kv_heads, b->k_tokens, k_head_stride, k_token_stride, 1, kPromptTile)) != RT_OK) return st;
        if ((st = make_map(&v_map, v, dtype, head_dim, kv_heads, b->k_tokens, v_head_stride, v_token_stride, 1, p.form == 2 ? PromptShape<256>::kValueRows : kPromptTile)) != RT_OK) return st;
    }
    void* params[] = {&q_map, &k_map, &v_map, &a};
    st = launch_kernel(kernels.attention[p.form], dim3((unsigned)p.ctas), dim3(kPromptThreads), kernels.smem[p.form], (cudaStream_t)stream, params);
    if (st != RT_OK || p.parts == 1) return st;
    const long long merge_ctas = ceil_div(b->q_tokens * q_heads, kPromptMergeThreads / 32);
    void* merge_params[] = {&a};
    return launch_kernel(kernels.merge, dim3((unsigned)merge_ctas), dim3(kPromptMergeThreads), 0, (cudaStream_t)stream, merge_params);
}

}  // extern "C"
