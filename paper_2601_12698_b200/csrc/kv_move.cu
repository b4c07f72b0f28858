// Entry points of the moves inside a paged cache: argument checks, launch rules and the kernels' instances.
#include <stddef.h>
#include <string.h>

#include <atomic>

#include "kv_move_kernels.cuh"
#include "tuner_internal.h"

namespace rt {

int check_cache(const rt_kv_cache* c, bool pointers);
int log2_or_minus1(unsigned v);

static_assert(kMaxLayers == RT_MAX_LAYERS, "the kernels' argument arrays hold RT_MAX_LAYERS caches");

namespace {

int64_t held_bytes(const rt_kv_cache& c) { return c.format == RT_KV_PLAIN ? elem_bytes_of(c.dtype) : 1; }

// The caches' pointers and their common geometry.
int gather_caches(const rt_kv_cache* caches, int n, MoveArgs* m)
{
    if (!caches) {
        set_error("caches is NULL");
        return RT_ERR_NULL;
    }
    if (n < 1 || n > RT_MAX_LAYERS) {
        set_error("n_caches=%d is not 1 .. %d", n, RT_MAX_LAYERS);
        return RT_ERR_SHAPE;
    }
    const rt_kv_cache& c = caches[0];
    const bool quantised = c.format != RT_KV_PLAIN;
    for (int i = 0; i < n; ++i) {
        const rt_kv_cache& x = caches[i];
        const int st = check_cache(&x, true);
        if (st != RT_OK) return st;
        // (shape, format and the elements' strides lie side by side, so do the scales' strides)
        if (memcmp(&x.n_pages, &c.n_pages, offsetof(rt_kv_cache, dtype) - offsetof(rt_kv_cache, n_pages)) || (!quantised && x.dtype != c.dtype) ||
            memcmp(&x.page_stride, &c.page_stride, 3 * sizeof(int64_t)) ||
            (quantised && memcmp(&x.scale_page_stride, &c.scale_page_stride, 3 * sizeof(int64_t)))) {
            set_error("cache %d is not like the first", i);
            return RT_ERR_SHAPE;
        }
        m->base[0][2 * i] = (unsigned char*)x.k;
        m->base[0][2 * i + 1] = (unsigned char*)x.v;
        m->base[1][2 * i] = quantised ? (unsigned char*)x.k_scale : nullptr;
        m->base[1][2 * i + 1] = quantised ? (unsigned char*)x.v_scale : nullptr;
    }
    const int64_t es = held_bytes(c);
    m->kind[0] = {c.page_stride * es, c.token_stride * es, c.head_stride * es, (int)(c.head_dim * es)};
    m->kind[1] = {c.scale_page_stride * 4, c.scale_token_stride * 4, c.scale_head_stride * 4, 4};
    m->sides = 2 * n;
    m->kinds = quantised ? 2 : 1;
    m->n_pages = c.n_pages;
    m->page_size = c.page_size;
    m->heads = c.kv_heads;
    return RT_OK;
}

// The runs of a page of this kind (see PageRuns), axes of one entry joined with anything.
PageRuns runs_of(const MoveKind& k, int page_size, int heads)
{
    const long long row = k.row_bytes;
    const bool heads_joined = heads == 1 || k.head_stride == row;                                      // a token's heads in one run
    const bool tokens_joined = page_size == 1 || k.token_stride == (heads_joined ? heads * row : row);  // one run behind another
    PageRuns r = {0, 0, (int)row, 1, 0, 0};
    if (heads_joined && tokens_joined) {
        r.run_bytes = (int)(heads * row);
        r.run_tokens = 1;
        r.outer_fixed = 1;
    } else if (heads_joined) {
        r.run_bytes = (int)(heads * row);
        r.outer_stride = k.token_stride;
    } else if (page_size == 1 || k.token_stride == row) {
        r.run_tokens = 1;
        r.outer_fixed = heads;
        r.outer_stride = k.head_stride;
    } else {
        r.outer_stride = k.token_stride;
        r.inner = heads;
        r.inner_stride = k.head_stride;
    }
    return r;
}

// Widest access, up to `most` bytes, that starts and ends of runs allow everywhere.
int access_width(const MoveArgs& m, int kind, long long run_bytes, int most)
{
    const MoveKind& k = m.kind[kind];
    uint64_t places = (uint64_t)run_bytes | (uint64_t)most;
    if (m.n_pages > 1) places |= (uint64_t)k.page_stride;
    if (m.page_size > 1) places |= (uint64_t)k.token_stride;
    if (m.heads > 1) places |= (uint64_t)k.head_stride;
    for (int i = 0; i < m.sides; ++i) places |= (uint64_t)(uintptr_t)m.base[kind][i];
    return (int)(places & (~places + 1));
}

typedef void (*CopyKernel)(CopyPagesArgs);
template <int SVB>
CopyKernel copy_kernel(int vb)
{
    switch (vb) {
        case 32: return kv_copy_pages_kernel<32, SVB>;
        case 16: return kv_copy_pages_kernel<16, SVB>;
        case 8: return kv_copy_pages_kernel<8, SVB>;
        case 4: return kv_copy_pages_kernel<4, SVB>;
        default: return kv_copy_pages_kernel<1, SVB>;
    }
}

typedef void (*CompactKernel)(CompactArgs);
template <int VB, int STAGES>
CompactKernel compact_kernel(int lanes)
{
    if constexpr (VB < 4) return kv_compact_kernel<VB, 32, STAGES>;
    else
        return lanes == 4    ? kv_compact_kernel<VB, 4, STAGES>
               : lanes == 8  ? kv_compact_kernel<VB, 8, STAGES>
               : lanes == 16 ? kv_compact_kernel<VB, 16, STAGES>
                             : kv_compact_kernel<VB, 32, STAGES>;
}
template <int VB>
CompactKernel compact_kernel(int lanes, bool deep)
{
    if constexpr (VB < 4) return compact_kernel<VB, kMoveStages>(lanes);
    else return deep ? compact_kernel<VB, kMoveDeepStages>(lanes) : compact_kernel<VB, kMoveStages>(lanes);
}

// The kernel for accesses of `width` bytes, `lanes` of them side by side.  Shared memory beyond the default limit is asked for once per
// device and kernel.
int find_compact_kernel(int width, int lanes, bool deep, int smem, CompactKernel* fn)
{
    static std::atomic<unsigned char> done[kDeviceSlots][5][6][2];
    switch (width) {
        case 16: *fn = compact_kernel<16>(lanes, deep); break;
        case 8: *fn = compact_kernel<8>(lanes, deep); break;
        case 4: *fn = compact_kernel<4>(lanes, deep); break;
        case 2: *fn = compact_kernel<2>(lanes, deep); break;
        default: *fn = compact_kernel<1>(lanes, deep); break;
    }
    if (smem <= 48 * 1024) return RT_OK;
    int device;
    const int st = current_device_index(&device);
    if (st != RT_OK) return st;
    std::atomic<unsigned char>& mine = done[device][log2_or_minus1((unsigned)width)][log2_or_minus1((unsigned)lanes)][deep];
    if (!mine.load(std::memory_order_acquire)) {
        RT_CUDA_OK(cudaFuncSetAttribute((const void*)*fn, cudaFuncAttributeMaxDynamicSharedMemorySize, compact_smem(2, width, deep ? kMoveDeepStages : kMoveStages)));
        mine.store(1, std::memory_order_release);
    }
    return RT_OK;
}

}  // namespace
}  // namespace rt

extern "C" {

int kv_cache_copy_pages_launch(const rt_kv_cache* caches, int32_t n_caches, const int32_t* src, const int32_t* dst, const int32_t* tokens,
                               int64_t n_pages, void* stream)
{
    using namespace rt;
    CopyPagesArgs a;
    memset(&a, 0, sizeof(a));
    int st = gather_caches(caches, n_caches, &a.m);
    if (st != RT_OK) return st;
    if (n_pages < 0 || n_pages > (1LL << 30)) {
        set_error("n_pages=%lld out of range", (long long)n_pages);
        return RT_ERR_SHAPE;
    }
    if (n_pages == 0) return RT_OK;
    if (!src || !dst) {
        set_error("src or dst is NULL");
        return RT_ERR_NULL;
    }
    if (((uintptr_t)src | (uintptr_t)dst | (uintptr_t)tokens) & 3u) {
        set_error("src, dst or tokens is not aligned to its element size");
        return RT_ERR_ALIGN;
    }
    const long long largest = (long long)a.m.page_size * a.m.heads * std::max(a.m.kind[0].row_bytes, a.m.kind[1].row_bytes);
    if (largest > (1LL << 30)) {  // places inside a page are ints
        set_error("a page of %lld bytes is too large", largest);
        return RT_ERR_SHAPE;
    }
    a.m.status = device_status_word();
    if (!a.m.status) return RT_ERR_NO_DEVICE;
    a.src = src;
    a.dst = dst;
    a.tokens = tokens;
    a.n = n_pages;
    int width[2] = {0, 0};
    long long ctas = 1;
    for (int kind = 0; kind < a.m.kinds; ++kind) {
        a.runs[kind] = runs_of(a.m.kind[kind], a.m.page_size, a.m.heads);
        const PageRuns& r = a.runs[kind];
        width[kind] = access_width(a.m, kind, r.run_bytes, 32);
        if (width[kind] == 2) width[kind] = 1;
        const long long page_bytes = (long long)a.m.page_size * a.m.heads * a.m.kind[kind].row_bytes;
        const long long vectors = (page_bytes + width[kind] - 1) / width[kind];
        int threads = 1;
        while (threads < kMoveThreads && threads * 4 < vectors) threads *= 2;
        a.threads_per_pair[kind] = threads;
        a.chunks[kind] = (int)std::min<long long>(1024, std::max<long long>(1, vectors / (kMoveThreads * 4)));
        const long long pairs_per_cta = kMoveThreads / threads;
        ctas = std::max(ctas, (n_pages + pairs_per_cta - 1) / pairs_per_cta * a.chunks[kind]);
    }
    if (ctas > 0x7fffffffLL) {
        set_error("n_pages=%lld needs too many CTAs", (long long)n_pages);
        return RT_ERR_SHAPE;
    }
    const CopyKernel fn = a.m.kinds == 1 ? copy_kernel<0>(width[0]) : width[1] >= 16 ? copy_kernel<16>(width[0]) : copy_kernel<4>(width[0]);
    void* params[] = {&a};
    return launch_kernel((const void*)fn, dim3((unsigned)ctas, (unsigned)(a.m.sides * a.m.kinds)), dim3(kMoveThreads), 0, (cudaStream_t)stream, params);
}

int kv_cache_compact_launch(const rt_kv_cache* caches, int32_t n_caches, const rt_compact_batch* b, void* stream)
{
    using namespace rt;
    CompactArgs a;
    memset(&a, 0, sizeof(a));
    if (!b) {
        set_error("batch is NULL");
        return RT_ERR_NULL;
    }
    int st = gather_caches(caches, n_caches, &a.m);
    if (st != RT_OK) return st;
    if (b->n_seqs < 0 || b->n_seqs > (1LL << 24) || b->window < 0 || b->window > (1LL << 30) || b->page_table_width < 0 ||
        b->page_table_width > 0x7fffffffLL || b->page_table_stride < 0 || b->keep_stride < 0) {
        set_error("n_seqs=%lld window=%lld or a width or stride out of range", (long long)b->n_seqs, (long long)b->window);
        return RT_ERR_SHAPE;
    }
    if (b->n_seqs == 0) return RT_OK;
    if (!b->starts || !b->lens || !b->new_lens || (b->page_table_width > 0 && !b->page_table) || (b->window > 0 && !b->keep)) {
        set_error("a tensor pointer is NULL");
        return RT_ERR_NULL;
    }
    if (((uintptr_t)b->page_table | (uintptr_t)b->starts | (uintptr_t)b->lens | (uintptr_t)b->new_lens) & 3u) {
        set_error("page_table, starts, lens or new_lens is not aligned to its element size");
        return RT_ERR_ALIGN;
    }
    // (every CTA of a sequence reads its start and length, one writes the new length)
    const uint64_t own = (uint64_t)b->n_seqs * 4, to_lens = (uintptr_t)b->new_lens - (uintptr_t)b->lens, to_starts = (uintptr_t)b->new_lens - (uintptr_t)b->starts;
    if (to_lens < own || 0 - to_lens < own || to_starts < own || 0 - to_starts < own) {
        set_error("new_lens must not overlap the inputs");
        return RT_ERR_SHAPE;
    }
    a.m.status = device_status_word();
    if (!a.m.status) return RT_ERR_NO_DEVICE;
    a.page_table = b->page_table;
    a.page_table_stride = b->page_table_stride;
    a.page_table_width = (int)b->page_table_width;
    a.page_shift = log2_or_minus1((unsigned)a.m.page_size);
    a.starts = b->starts;
    a.lens = b->lens;
    a.keep = b->keep;
    a.keep_stride = b->keep_stride;
    a.window = (int)b->window;
    a.new_lens = b->new_lens;
    a.n_seqs = (int)b->n_seqs;
    const long long n_seqs = b->n_seqs;
    rt_limits L;
    if ((st = current_limits(&L)) != RT_OK) return st;
    // A task is a side of a layer, a head and a piece of its rows: whole rows, or where that leaves SMs without a CTA, pieces down to 64 bytes.
    // Tasks of a sequence to one CTA: few enough that two CTAs to an SM cover the device, and no fewer than its warps.  With no more CTAs than
    // SMs each has more under way.  (40 sequences x 32 layers x 8 heads, two or three rows each: 7.1 us in a graph with two CTAs to an SM,
    // 8.8 with four.  Rows in halves, for more CTAs than SMs, were slower: 12 sequences x 8 layers: 164 us, then 145 without.  One sequence of
    // 100000 tokens x 4 layers x 8 heads of 128 bf16: 581 us, 1439 with whole rows and three items under way; 24000 x 32 layers: 421 and 590.)
    const int width = access_width(a.m, 0, a.m.kind[0].row_bytes, 16), row_vectors = a.m.kind[0].row_bytes / width;
    int lanes = 32;
    while (width >= 4 && lanes > 4 && lanes / 2 >= row_vectors) lanes /= 2;
    long long tasks, ctas;
    for (;; lanes /= 2) {
        a.pieces = (row_vectors + lanes - 1) / lanes;
        tasks = (long long)a.m.sides * a.m.heads * a.pieces;
        a.tasks_per_cta = (int)std::min<long long>(128, std::max<long long>(8, tasks * n_seqs / (L.sm_count * 2LL) / 8 * 8));
        a.ctas_per_seq = (int)((tasks + a.tasks_per_cta - 1) / a.tasks_per_cta);
        ctas = (long long)a.ctas_per_seq * n_seqs;
        if (ctas * 2 > L.sm_count || width < 4 || lanes == 4 || lanes * width <= 64) break;
    }
    if (ctas > 0x7fffffffLL) {
        set_error("n_seqs=%lld needs too many CTAs", n_seqs);
        return RT_ERR_SHAPE;
    }
    const bool deep = width >= 4 && ctas <= L.sm_count;
    const int smem = compact_smem(a.m.kinds, width, deep ? kMoveDeepStages : kMoveStages);
    CompactKernel fn;
    if ((st = find_compact_kernel(width, lanes, deep, smem, &fn)) != RT_OK) return st;
    void* params[] = {&a};
    return launch_kernel((const void*)fn, dim3((unsigned)ctas), dim3(kMoveThreads), (size_t)smem, (cudaStream_t)stream, params);
}

}  // extern "C"
