// Entry point of the attention over a shared prefix: argument checks, the split of the work into parts, the launches.
#include <string.h>

#include <atomic>

#include "attend_common.cuh"
#include "attend_host.h"
#include "attend_keys_kernel.cuh"
#include "attend_merge_kernel.cuh"
#include "attend_prefix_kernel.cuh"
#include "attend_split.h"
#include "tuner_internal.h"

namespace rt {

int check_cache(const rt_kv_cache* c, bool pointers);
int log2_or_minus1(unsigned v);

namespace {

constexpr int kMaxLen = 1 << 30;
constexpr int kMaxParts = 64;  // of a suffix, and of a prefix that is not dealt out by tiles

struct AttendPlan {
    int padded_dim;
    int group;
    long long tokens;
    int prefix_form, suffix_form;  // kPrefixTiles, kKeys16, kKeys64; -1: no keys
    int prefix_parts, prefix_keys, suffix_parts, suffix_keys;
    PrefixSplit split;  // run > 0: the prefix is dealt out by tiles
    long long prefix_ctas, suffix_ctas;
    bool joined;  // results lie in parts, which merge_parts_kernel joins; otherwise the only part is the result
    int64_t workspace;
};

AttendKernels kernels_of(int dtype, int format, int padded_dim)
{
    typedef AttendKernels (*Get)(int);
    static const Get get[2][3] = {{rt_attend_kernels_bf16_plain, rt_attend_kernels_bf16_e4m3, rt_attend_kernels_bf16_int8},
                                  {rt_attend_kernels_fp16_plain, rt_attend_kernels_fp16_e4m3, rt_attend_kernels_fp16_int8}};
    return get[dtype][format](padded_dim);
}

// Shared memory beyond the default limit is asked for once per device and kernel.
int launch_form(const AttendKernels& kernels, int form, int dtype, int format, int padded_dim, long long ctas, int threads,
                cudaStream_t stream, void** params)
{
    static std::atomic<unsigned char> done[kDeviceSlots][2][3][3][kAttendKernels];
    const AttendKernel& k = kernels.k[form];
    if (k.smem > 48 * 1024) {
        int device;
        const int st = current_device_index(&device);
        if (st != RT_OK) return st;
        std::atomic<unsigned char>& flag = done[device][dtype][format][padded_dim / 128][form];
        if (!flag.load(std::memory_order_acquire)) {
            RT_CUDA_OK(cudaFuncSetAttribute(k.fn, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)k.smem));
            flag.store(1, std::memory_order_release);
        }
    }
    return launch_kernel(k.fn, dim3((unsigned)ctas), dim3(threads), k.smem, stream, params);
}

long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

// Parts of `keys` keys such that `tiles` tiles times the parts give about `want` CTAs, none of fewer than `least` keys.
void split_keys(long long keys, long long tiles, long long want, int least, int* parts, int* part_keys)
{
    long long n = std::max<long long>(1, want / std::max<long long>(1, tiles));
    n = std::min<long long>(n, std::min<long long>(kMaxParts, ceil_div(keys, least)));
    const long long each = ceil_div(ceil_div(keys, n), least) * least;
    *part_keys = (int)std::min<long long>(each, kMaxLen);
    *parts = (int)ceil_div(keys, each);
}

// Geometry checks and the split.  The same for the workspace query and the launch.
int make_attend_plan(const rt_kv_cache* c, const rt_prefix_batch* b, int q_heads, AttendPlan* p)
{
    int st = check_cache(c, false);
    if (st != RT_OK) return st;
    if (!b) {
        set_error("batch is NULL");
        return RT_ERR_NULL;
    }
    const int step = c->format == RT_KV_PLAIN ? 8 : 16;
    if (c->head_dim % step != 0) {
        set_error("head_dim=%d is not a multiple of %d", (int)c->head_dim, step);
        return RT_ERR_SHAPE;
    }
    if (q_heads < 1 || q_heads % c->kv_heads != 0) {
        set_error("q_heads=%d is not a multiple of kv_heads=%d", q_heads, (int)c->kv_heads);
        return RT_ERR_SHAPE;
    }
    if (b->q_len < 1 || b->q_len > RT_MAX_QUERY_LEN) {
        set_error("q_len=%d outside 1..%d", (int)b->q_len, RT_MAX_QUERY_LEN);
        return RT_ERR_SHAPE;
    }
    if (b->n_seqs < 0 || b->prefix_len < 0 || b->prefix_len > kMaxLen || b->max_suffix_len < 0 || b->max_suffix_len > kMaxLen ||
        b->page_table_width < 0 || b->page_table_stride < 0 || b->n_prefix_pages < 0) {
        set_error("n_seqs=%lld prefix_len=%lld max_suffix_len=%lld or a page table size out of range", (long long)b->n_seqs,
                  (long long)b->prefix_len, (long long)b->max_suffix_len);
        return RT_ERR_SHAPE;
    }
    if (b->n_seqs > 0x7fffffffLL / ((long long)b->q_len * q_heads)) {
        set_error("n_seqs=%lld times q_len times q_heads exceeds 2^31 - 1", (long long)b->n_seqs);
        return RT_ERR_SHAPE;
    }
    if ((long long)b->n_prefix_pages * c->page_size < b->prefix_len) {
        set_error("%d prefix pages of %d tokens do not hold %lld", (int)b->n_prefix_pages, (int)c->page_size, (long long)b->prefix_len);
        return RT_ERR_SHAPE;
    }
    if ((long long)b->page_table_width * c->page_size < b->max_suffix_len) {
        set_error("%d pages of %d tokens do not hold %lld", (int)b->page_table_width, (int)c->page_size, (long long)b->max_suffix_len);
        return RT_ERR_SHAPE;
    }
    rt_limits L;
    st = current_limits(&L);
    if (st != RT_OK) return st;
    memset(p, 0, sizeof(*p));
    p->padded_dim = c->head_dim <= 64 ? 64 : c->head_dim <= 128 ? 128 : 256;
    p->group = q_heads / c->kv_heads;
    p->tokens = b->n_seqs * b->q_len;
    if (p->tokens == 0) return RT_OK;
    p->prefix_form = p->suffix_form = -1;
    const long long prefix_rows = p->tokens * p->group, suffix_rows = (long long)b->q_len * p->group;
    if (b->prefix_len > 0) {
        // Heads up to 128: 16 rows to a CTA and one launch with the suffixes up to 64 rows (64 rows, prefix 8192, int8: 31 us, 37 with
        // the tiles kernel, 34 with 64 rows to a CTA; 96 rows: 42, 37 and 46).  Heads of 256: 64 rows to a CTA (128 rows, prefix 8192:
        // 57 us, 103 with 16), but for few rows and keys (32 rows, prefix 600: 12.1 us with 16, 14.4 with 64; prefix 8192: 37.4 and 31.4).
        if (p->padded_dim == 256) p->prefix_form = prefix_rows <= 32 && b->prefix_len <= 2048 ? kKeys16 : kKeys64;
        else p->prefix_form = prefix_rows <= 64 ? kKeys16 : kPrefixTiles;
        if (p->prefix_form == kPrefixTiles) {
            PrefixSplit& s = p->split;
            s.tiles = (int)ceil_div(b->prefix_len, kTcTile);
            s.rows = (int)prefix_rows;
            s.blocks = (int)ceil_div(prefix_rows, kTcBlockRows);
            const long long units = (long long)s.blocks * c->kv_heads;
            // The two kernels run side by side, one CTA of this one taking a whole SM, where its CTAs are no more than the SMs (with
            // more, the suffix kernel starts in their last wave, and the model is only a bound on the runs): it gets the share of the
            // SMs that its share of the work asks for.  The unit is what a tile of 128 keys costs the suffix kernel on one SM (1.4 us plain, 1.7
            // quantised); a tile for 256 rows costs the prefix kernel 1.6 of that, beginning and ending a run about 7.  Suffixes are
            // taken to be half as long as they may be: a max_suffix_len far above the lengths leaves the prefix too few SMs (64
            // sequences of up to 100 keys, prefix 8192: 50 us where it is 100, 71 at 2048, 150 at 8192).
            const double prefix_work = (double)units * (s.tiles * 1.6 + 7), tiles_per_suffix = 0.5 * (double)ceil_div(b->max_suffix_len, 128);
            const double suffix_work = tiles_per_suffix * (double)ceil_div(suffix_rows, 16) * c->kv_heads * (double)b->n_seqs;
            long long sms = (long long)(L.sm_count * prefix_work / (prefix_work + suffix_work) + 0.5);
            sms = std::max<long long>(1, std::min<long long>(sms, L.sm_count));
            // The number of runs that ends first on that many SMs: whole waves of CTAs, each as long as its run.
            double best = 0;
            s.run = s.tiles;
            for (int runs = 1; runs <= std::min(s.tiles, kMaxParts); ++runs) {
                const int run = (int)ceil_div(s.tiles, runs);
                const double time = (double)ceil_div(units * ceil_div(s.tiles, run), sms) * (run * 1.6 + 7);
                if (runs == 1 || time < best * 0.97) {
                    best = time;
                    s.run = run;
                }
            }
            s.runs = (int)ceil_div(s.tiles, s.run);
            p->prefix_ctas = units * s.runs;
            p->prefix_parts = s.runs * (narrow_block(s, s.blocks - 1) ? 2 : 1);
        } else {
            const int nr = p->prefix_form == kKeys16 ? 16 : 64;
            const long long tiles = ceil_div(prefix_rows, nr) * c->kv_heads;
            split_keys(b->prefix_len, tiles, (long long)L.sm_count * (nr == 16 ? 2 : 1), 128, &p->prefix_parts, &p->prefix_keys);
            p->prefix_ctas = tiles * p->prefix_parts;
        }
    }
    if (b->max_suffix_len > 0) {
        // Of the prefix's form, and then in its launch, where that is keys first.  Otherwise 16 rows to a CTA up to three times that
        // many (heads of 128, 40 suffixes of 1 .. 700 keys: 48 rows 72 us, 68 with 64 to a CTA; in int8 68 and 74; 64 rows 93 and
        // 81), for heads of 256 up to 16 (20 rows: 110 us, 73 with 64).
        if (p->prefix_form > kPrefixTiles) p->suffix_form = p->prefix_form;
        else p->suffix_form = suffix_rows <= (p->padded_dim == 256 ? 16 : 48) ? kKeys16 : kKeys64;
        const int nr = p->suffix_form == kKeys16 ? 16 : 64;
        const long long tiles = ceil_div(suffix_rows, nr) * c->kv_heads * b->n_seqs;
        // Two CTAs of 16 rows share an SM; beside the tiles kernel, which takes SMs of its own, fewer and longer parts are better
        // (17 sequences x 8 heads of 64, 5 query tokens: 19.7 us with one part, 23.5 with two).
        const bool pairs = nr == 16 && p->prefix_form != kPrefixTiles;
        split_keys(b->max_suffix_len, tiles, (long long)L.sm_count * (pairs ? 2 : 1), 128, &p->suffix_parts, &p->suffix_keys);
        p->suffix_ctas = tiles * p->suffix_parts;
    }
    if (p->prefix_ctas + p->suffix_ctas > 0x7fffffffLL) {
        set_error("the batch needs too many CTAs");
        return RT_ERR_SHAPE;
    }
    const int parts = p->prefix_parts + p->suffix_parts;
    const int64_t rows = p->tokens * q_heads;
    // Without any part the merge kernel writes the empty result.  The tiles kernel leaves parts even where it leaves only one.
    p->joined = parts != 1 || p->prefix_form == kPrefixTiles;
    if (p->joined && parts > 0) p->workspace = (int64_t)parts * rows * c->head_dim * 4 + ((int64_t)parts * rows * 4 + 15) / 16 * 16;
    return RT_OK;
}

}  // namespace
}  // namespace rt

extern "C" {

int64_t shared_prefix_attention_workspace_bytes(const rt_kv_cache* cache, const rt_prefix_batch* batch, int32_t q_heads)
{
    rt::AttendPlan p;
    if (rt::make_attend_plan(cache, batch, q_heads, &p) != RT_OK) return -1;
    return p.workspace;
}

int shared_prefix_attention_launch(const rt_kv_cache* c, const rt_prefix_batch* b, const void* q, int64_t q_token_stride,
                                   int64_t q_head_stride, int32_t q_heads, void* out, float* lse, float softmax_scale, int dtype,
                                   void* workspace, int64_t workspace_bytes, void* stream)
{
    using namespace rt;
    if (dtype != RT_BF16 && dtype != RT_FP16) {
        set_error("dtype %d is not bf16 or fp16", dtype);
        return RT_ERR_DTYPE;
    }
    AttendPlan p;
    int st = make_attend_plan(c, b, q_heads, &p);
    if (st != RT_OK) return st;
    if (c->format == RT_KV_PLAIN && c->dtype != dtype) {
        set_error("a plain cache of dtype %d does not serve queries of dtype %d", (int)c->dtype, dtype);
        return RT_ERR_DTYPE;
    }
    if (p.tokens == 0) return RT_OK;
    const int parts = p.prefix_parts + p.suffix_parts;
    if (!q || !out || !b->suffix_lens || (b->prefix_len > 0 && !b->prefix_pages) || (b->max_suffix_len > 0 && !b->page_table) ||
        (p.workspace > 0 && !workspace)) {
        set_error("a tensor pointer is NULL");
        return RT_ERR_NULL;
    }
    if (parts > 0 && (st = check_cache(c, true)) != RT_OK) return st;
    if (parts > 0 && c->n_pages == 0) {
        set_error("a cache without pages holds neither prefix nor suffix");
        return RT_ERR_SHAPE;
    }
    if (workspace_bytes < p.workspace) {
        set_error("workspace of %lld bytes, %lld are needed", (long long)workspace_bytes, (long long)p.workspace);
        return RT_ERR_CAPACITY;
    }
    if (q_token_stride < 0 || q_head_stride < 0) {
        set_error("negative q stride");
        return RT_ERR_SHAPE;
    }
    const int64_t es = c->format == RT_KV_PLAIN ? 2 : 1;
    const int64_t strides = (c->n_pages > 1 ? c->page_stride * es : 0) | (c->page_size > 1 ? c->token_stride * es : 0) |
                            (c->kv_heads > 1 ? c->head_stride * es : 0) | (p.tokens > 1 ? q_token_stride * 2 : 0) |
                            (q_heads > 1 ? q_head_stride * 2 : 0);
    if ((((uintptr_t)c->k | (uintptr_t)c->v | (uintptr_t)q | (uintptr_t)out | (uintptr_t)workspace) & 15u) || (strides & 15) ||
        (((uintptr_t)lse | (uintptr_t)b->suffix_lens | (uintptr_t)b->page_table | (uintptr_t)b->prefix_pages) & 3u)) {
        set_error("k, v, q, out, workspace and their strides must be multiples of 16 bytes, the other tensors of 4");
        return RT_ERR_ALIGN;
    }
    AttendArgs a;
    memset(&a, 0, sizeof(a));
    a.k = (const unsigned char*)c->k;
    a.v = (const unsigned char*)c->v;
    a.k_scale = c->k_scale;
    a.v_scale = c->v_scale;
    a.page_stride = c->page_stride;
    a.token_stride = c->token_stride;
    a.head_stride = c->head_stride;
    a.scale_page_stride = c->scale_page_stride;
    a.scale_token_stride = c->scale_token_stride;
    a.scale_head_stride = c->scale_head_stride;
    a.n_pages = c->n_pages;
    a.page_size = (unsigned)c->page_size;
    a.page_shift = log2_or_minus1((unsigned)c->page_size);
    a.prefix_pages = b->prefix_pages;
    a.page_table = b->page_table;
    a.suffix_lens = b->suffix_lens;
    a.page_table_stride = b->page_table_stride;
    a.page_table_width = b->page_table_width;
    a.prefix_len = (int)b->prefix_len;
    a.max_suffix_len = (int)b->max_suffix_len;
    a.n_seqs = (int)b->n_seqs;
    a.q_len = b->q_len;
    a.kv_heads = c->kv_heads;
    a.group = p.group;
    a.dim = c->head_dim;
    a.q = (const unsigned char*)q;
    a.q_token_stride = q_token_stride;
    a.q_head_stride = q_head_stride;
    a.score_scale = softmax_scale * 1.4426950408889634f;
    a.prefix_parts = p.prefix_parts;
    a.prefix_keys = p.prefix_keys;
    a.suffix_parts = p.suffix_parts;
    a.suffix_keys = p.suffix_keys;
    a.part_out = (float*)workspace;
    a.part_lse = p.workspace > 0 ? (float*)workspace + (int64_t)parts * p.tokens * q_heads * c->head_dim : nullptr;
    a.out = out;
    a.lse = lse;
    a.status = device_status_word();
    if (!a.status) return RT_ERR_NO_DEVICE;
    a.wait_polls = wait_poll_limit();
    a.drop_copies = drop_copies();
    const AttendKernels k = kernels_of(dtype, c->format, p.padded_dim);
    const cudaStream_t s = (cudaStream_t)stream;
    const auto launch = [&](int form, long long ctas, int threads, void* second) {
        void* params[] = {&a, second};
        return launch_form(k, form, dtype, c->format, p.padded_dim, ctas, threads, s, params);
    };
    int prefix_ctas = p.prefix_form > kPrefixTiles ? (int)p.prefix_ctas : 0;
    if (p.prefix_form == kPrefixTiles) {
        a.before_suffix = a.after_prefix = p.suffix_form >= 0;
        st = launch(kPrefixTiles, p.prefix_ctas, kTcThreads, &p.split);
        if (st != RT_OK) return st;
    }
    const int keys_form = p.suffix_form >= 0 ? p.suffix_form : prefix_ctas > 0 ? p.prefix_form : -1;
    if (keys_form >= 0) {  // suffixes, and the prefix where it takes the same form
        st = launch(keys_form, prefix_ctas + p.suffix_ctas, kKeysThreads, &prefix_ctas);
        if (st != RT_OK) return st;
    }
    if (p.joined) st = launch(kMergeParts, ceil_div(p.tokens * q_heads * (p.padded_dim == 256 ? 2 : 1), kMergePartsThreads / 32), kMergePartsThreads, &p.split);
    return st;
}

}  // extern "C"
