// Entry points of the paged key/value cache: argument checks, the launch rule and the kernels' instances.
#include <string.h>

#include "kv_cache_kernels.cuh"
#include "tuner_internal.h"

namespace rt {

// What every call on a cache may rely on.  `pointers`: also check that the tensors are there.
int check_cache(const rt_kv_cache* c, bool pointers)
{
    if (!c) {
        set_error("cache is NULL");
        return RT_ERR_NULL;
    }
    if (c->format < RT_KV_PLAIN || c->format > RT_KV_INT8) {
        set_error("cache format %d is not an rt_kv_format", (int)c->format);
        return RT_ERR_DTYPE;
    }
    if (c->format == RT_KV_PLAIN && (c->dtype < RT_BF16 || c->dtype > RT_FP32)) {
        set_error("cache dtype %d is not an rt_dtype", (int)c->dtype);
        return RT_ERR_DTYPE;
    }
    if (c->n_pages < 0 || c->n_pages > (1LL << 31) - 1 || c->page_size < 1 || c->page_size > 65536 || c->kv_heads < 1 ||
        c->kv_heads > 65535 || c->head_dim < 1 || c->head_dim > RT_KV_MAX_HEAD_DIM) {
        set_error("n_pages=%lld page_size=%d kv_heads=%d head_dim=%d out of range", (long long)c->n_pages, (int)c->page_size,
                  (int)c->kv_heads, (int)c->head_dim);
        return RT_ERR_SHAPE;
    }
    if (c->page_stride < 0 || c->token_stride < 0 || c->head_stride < 0 || c->scale_page_stride < 0 || c->scale_token_stride < 0 ||
        c->scale_head_stride < 0) {
        set_error("negative cache stride");
        return RT_ERR_SHAPE;
    }
    if (!pointers || c->n_pages == 0) return RT_OK;
    if (!c->k || !c->v || (c->format != RT_KV_PLAIN && (!c->k_scale || !c->v_scale))) {
        set_error("a cache pointer is NULL");
        return RT_ERR_NULL;
    }
    const uintptr_t mask = c->format != RT_KV_PLAIN ? 0u : (uintptr_t)elem_bytes_of(c->dtype) - 1u;
    if ((((uintptr_t)c->k | (uintptr_t)c->v) & mask) ||
        (c->format != RT_KV_PLAIN && (((uintptr_t)c->k_scale | (uintptr_t)c->v_scale) & 3u))) {
        set_error("a cache tensor is not aligned to its element size");
        return RT_ERR_ALIGN;
    }
    return RT_OK;
}

int log2_or_minus1(unsigned v)
{
    if (v == 0 || (v & (v - 1)) != 0) return -1;
    int s = 0;
    while ((1u << s) < v) ++s;
    return s;
}

namespace {

typedef void (*CacheKernel)(CacheArgs);

// Launch shape of one call: elements per lane, elements per access, lanes per vector.
template <bool WRITE, typename T, int FMT, int E, int AL, int LANES>
int launch_shape(const CacheArgs& args, cudaStream_t stream)
{
    CacheArgs a = args;
    constexpr int GROUPS = kCacheThreads / LANES;
    constexpr int U = 2;
    // A CTA takes as many tokens as fill its groups: once over while the device has SMs to spare, U times once it is
    // covered (the vectors of one batch are then in flight together).
    const int per_token = 2 * a.heads;
    rt_limits L;
    int st = current_limits(&L);
    if (st != RT_OK) return st;
    const long long groups_wanted = a.n_tokens * per_token;
    const bool deep = groups_wanted > (long long)L.sm_count * 4 * GROUPS;
    const int want = GROUPS * (deep ? U : 1);
    a.tokens_per_cta = std::max(1, want / per_token);
    const long long ctas = (a.n_tokens + a.tokens_per_cta - 1) / a.tokens_per_cta;
    if (ctas > 0x7fffffffLL) {
        set_error("n_tokens=%lld needs too many CTAs", (long long)a.n_tokens);
        return RT_ERR_SHAPE;
    }
    const CacheKernel fn = WRITE ? (deep ? (CacheKernel)kv_cache_write_kernel<T, FMT, E, AL, LANES, U>
                                         : (CacheKernel)kv_cache_write_kernel<T, FMT, E, AL, LANES, 1>)
                                 : (deep ? (CacheKernel)kv_cache_read_kernel<T, FMT, E, AL, LANES, U>
                                         : (CacheKernel)kv_cache_read_kernel<T, FMT, E, AL, LANES, 1>);
    void* params[] = {&a};
    return launch_kernel((const void*)fn, dim3((unsigned)ctas), dim3(kCacheThreads), 0, stream, params);
}

// Sixteen elements to a lane (the kernels are bound by instructions, and those that find a vector's places are shared by more
// elements: 16384 x 8 x 128 bf16 to e4m3 took 30 us with eight, 20 with sixteen), in accesses as wide as sizes, strides and
// pointers allow.  Accesses that are less than a lane's share go round the lanes (16384 x 8 x 100 bf16, plain: 17 us, 30 with
// a lane's accesses side by side).  Places that are not even multiples of four elements (odd head sizes): accesses of one
// element, eight to a lane (16384 x 8 x 33 bf16 to e4m3: 19 us, 83 with one to a lane).
template <bool WRITE, typename T, int FMT, int AL>
int launch_aligned(const CacheArgs& a, cudaStream_t stream)
{
    if (a.dim <= 64) return launch_shape<WRITE, T, FMT, 16, AL, 4>(a, stream);
    if (a.dim <= 128) return launch_shape<WRITE, T, FMT, 16, AL, 8>(a, stream);
    return launch_shape<WRITE, T, FMT, 16, AL, 16>(a, stream);
}
template <bool WRITE, typename T, int FMT>
int launch_typed(const CacheArgs& a, int align_elems, cudaStream_t stream)
{
    if (align_elems >= 16) return launch_aligned<WRITE, T, FMT, 16>(a, stream);
    if constexpr (sizeof(T) < 4) {
        if (align_elems >= 8) return launch_aligned<WRITE, T, FMT, 8>(a, stream);
    }
    if (align_elems >= 4) return launch_aligned<WRITE, T, FMT, 4>(a, stream);
    if (a.dim <= 64) return launch_shape<WRITE, T, FMT, 8, 1, 8>(a, stream);
    if (a.dim <= 128) return launch_shape<WRITE, T, FMT, 8, 1, 16>(a, stream);
    return launch_shape<WRITE, T, FMT, 8, 1, 32>(a, stream);
}

template <bool WRITE, typename T>
int launch_format(int format, const CacheArgs& a, int align_elems, cudaStream_t stream)
{
    switch (format) {
        case RT_KV_PLAIN: return launch_typed<WRITE, T, kKvPlain>(a, align_elems, stream);
        case RT_KV_E4M3: return launch_typed<WRITE, T, kKvE4m3>(a, align_elems, stream);
        default: return launch_typed<WRITE, T, kKvInt8>(a, align_elems, stream);
    }
}

// Largest of 16, 8, 4, 1 such that accesses of that many elements are aligned everywhere: those to token tensors want
// min(16, elements * size) bytes, those to the cache min(16, elements * held size).
int shared_alignment(const rt_kv_cache* c, const void* key, long long kts, long long khs, const void* value, long long vts,
                     long long vhs, int dtype, long long n_tokens)
{
    const long long size = elem_bytes_of(dtype), held = c->format == RT_KV_PLAIN ? size : 1;
    for (int e = 16; e > 2; e >>= 1) {
        const long long tok = std::min<long long>(16, e * size), kv = std::min<long long>(16, e * held);
        bool ok = c->head_dim % e == 0;
        ok = ok && (uintptr_t)key % tok == 0 && (uintptr_t)value % tok == 0 && (uintptr_t)c->k % kv == 0 && (uintptr_t)c->v % kv == 0;
        if (n_tokens > 1) ok = ok && kts * size % tok == 0 && vts * size % tok == 0;
        if (c->kv_heads > 1) ok = ok && khs * size % tok == 0 && vhs * size % tok == 0 && c->head_stride * held % kv == 0;
        if (c->page_size > 1) ok = ok && c->token_stride * held % kv == 0;
        if (c->n_pages > 1) ok = ok && c->page_stride * held % kv == 0;
        if (ok) return e;
    }
    return 1;
}

template <bool WRITE>
int cache_launch(const rt_kv_cache* c, const void* key, int64_t kts, int64_t khs, const void* value, int64_t vts, int64_t vhs,
                 const int64_t* slots, int64_t n_tokens, int dtype, void* stream)
{
    int st = check_cache(c, n_tokens > 0);
    if (st != RT_OK) return st;
    if (dtype < RT_BF16 || dtype > RT_FP32) {
        set_error("dtype %d is not an rt_dtype", dtype);
        return RT_ERR_DTYPE;
    }
    if (c->format == RT_KV_PLAIN && c->dtype != dtype) {
        set_error("a plain cache of dtype %d does not hold dtype %d", (int)c->dtype, dtype);
        return RT_ERR_DTYPE;
    }
    if (n_tokens < 0 || kts < 0 || khs < 0 || vts < 0 || vhs < 0) {
        set_error("n_tokens=%lld or a stride is negative", (long long)n_tokens);
        return RT_ERR_SHAPE;
    }
    if (n_tokens == 0) return RT_OK;
    if (!key || !value || !slots) {
        set_error("a tensor pointer is NULL");
        return RT_ERR_NULL;
    }
    const uintptr_t elem_mask = (uintptr_t)elem_bytes_of(dtype) - 1u;
    if ((((uintptr_t)key | (uintptr_t)value) & elem_mask) || ((uintptr_t)slots & 7u)) {
        set_error("key, value or slots is not aligned to its element size");
        return RT_ERR_ALIGN;
    }
    CacheArgs a;
    memset(&a, 0, sizeof(a));
    a.side[0] = (unsigned char*)c->k;
    a.side[1] = (unsigned char*)c->v;
    a.scale[0] = c->k_scale;
    a.scale[1] = c->v_scale;
    a.tokens[0] = (unsigned char*)const_cast<void*>(key);
    a.tokens[1] = (unsigned char*)const_cast<void*>(value);
    a.token_stride[0] = kts;
    a.token_stride[1] = vts;
    a.token_head_stride[0] = khs;
    a.token_head_stride[1] = vhs;
    a.slots = (const long long*)slots;
    a.n_tokens = n_tokens;
    a.n_slots = c->n_pages * c->page_size;
    a.page_stride = c->page_stride;
    a.entry_stride = c->token_stride;
    a.head_stride = c->head_stride;
    a.scale_page_stride = c->scale_page_stride;
    a.scale_entry_stride = c->scale_token_stride;
    a.scale_head_stride = c->scale_head_stride;
    a.page_size = (unsigned)c->page_size;
    a.page_shift = log2_or_minus1((unsigned)c->page_size);
    a.vec_shift = log2_or_minus1(2u * (unsigned)c->kv_heads);
    a.heads = c->kv_heads;
    a.dim = c->head_dim;
    a.status = device_status_word();
    if (!a.status) return RT_ERR_NO_DEVICE;
    const int e = shared_alignment(c, key, kts, khs, value, vts, vhs, dtype, n_tokens);
    switch (dtype) {
        case RT_BF16: return launch_format<WRITE, __nv_bfloat16>(c->format, a, e, (cudaStream_t)stream);
        case RT_FP16: return launch_format<WRITE, __half>(c->format, a, e, (cudaStream_t)stream);
        default: return launch_format<WRITE, float>(c->format, a, e, (cudaStream_t)stream);
    }
}

}  // namespace
}  // namespace rt

extern "C" {

int kv_cache_write_launch(const rt_kv_cache* cache, const void* key, int64_t key_token_stride, int64_t key_head_stride,
                          const void* value, int64_t value_token_stride, int64_t value_head_stride, const int64_t* slots,
                          int64_t n_tokens, int dtype, void* stream)
{
    return rt::cache_launch<true>(cache, key, key_token_stride, key_head_stride, value, value_token_stride, value_head_stride,
                                  slots, n_tokens, dtype, stream);
}

int kv_cache_read_launch(const rt_kv_cache* cache, const int64_t* slots, int64_t n_tokens, void* key_out,
                         int64_t key_token_stride, int64_t key_head_stride, void* value_out, int64_t value_token_stride,
                         int64_t value_head_stride, int dtype, void* stream)
{
    return rt::cache_launch<false>(cache, key_out, key_token_stride, key_head_stride, value_out, value_token_stride,
                                   value_head_stride, slots, n_tokens, dtype, stream);
}

}  // extern "C"
