// Entries of a paged cache moved inside it (sm_100a): whole pages copied, and the gaps of given-up tokens closed, in all layers
// of a model with one launch.  Bound by HBM: every byte that moves is read and written once.
#pragma once

#include "add_rmsnorm_kernel.cuh"
#include "kv_cache_kernels.cuh"

namespace rt {

constexpr int kMoveThreads = 256;
constexpr int kMaxLayers = 128;  // RT_MAX_LAYERS

// One kind of entry: the elements (k and v), or the scales.
struct MoveKind {
    long long page_stride, token_stride, head_stride;  // bytes
    int row_bytes;                                     // of one token and head
};
struct MoveArgs {
    unsigned char* base[2][2 * kMaxLayers];  // [kind][2 * layer + side]
    MoveKind kind[2];
    int sides;      // 2 * layers
    int kinds;      // 2 when there are scales
    long long n_pages;
    int page_size;
    int heads;
    int* status;
};

// Vectors of VB bytes, single bytes too (layouts that no wider access divides).
template <int VB>
__device__ __forceinline__ Vec<VB> ld_move(const unsigned char* p)
{
    if constexpr (VB == 1) {
        Vec<1> v;
        uint32_t x;
        asm volatile("ld.global.L1::no_allocate.u8 %0, [%1];" : "=r"(x) : "l"(p));
        v.w[0] = x;
        return v;
    } else {
        return ld_stream<VB>(p);
    }
}
template <int VB>
__device__ __forceinline__ void st_move(unsigned char* p, const Vec<VB>& v)
{
    if constexpr (VB == 1) *p = (unsigned char)v.w[0];
    else st_stream<VB>(p, v);
}

// ---- pages ----------------------------------------------------------------------------------------------------

// What the first `tokens` entries of a page are made of: `outer` x `inner` runs of `bytes` bytes.  Axes that lie behind one another
// without gaps are joined, so that a page is one run where the layout allows it.
struct PageRuns {
    long long outer_stride, inner_stride;
    int run_bytes;         // of a run, times the tokens when run_tokens
    int inner;             // runs behind one another at inner_stride
    int outer_fixed;       // number of outer runs, 0: the tokens
    int run_tokens;        // a run holds all tokens of a head (or of the page)
};
struct CopyPagesArgs {
    MoveArgs m;
    PageRuns runs[2];
    const int32_t* src;
    const int32_t* dst;
    const int32_t* tokens;
    long long n;
    int threads_per_pair[2];  // a power of two up to kMoveThreads
    int chunks[2];            // CTAs side by side on one page
};

// A group of threads takes a pair of pages of one side of one layer: blockIdx.y names the side (the scales' sides follow the
// elements'), blockIdx.x pairs and, for pages of more than kMoveThreads * U vectors, pieces of them.  U vectors of a thread are
// in flight at once.
template <int VB, int U>
__device__ __forceinline__ void copy_pages(const CopyPagesArgs& a, const PageRuns& runs, int kind, int side)
{
    const int per_pair = a.threads_per_pair[kind], chunks = a.chunks[kind];
    const int pairs_per_cta = kMoveThreads / per_pair;
    const long long block = blockIdx.x / (unsigned)chunks;
    const int chunk = (int)(blockIdx.x - (unsigned)(block * chunks));
    const long long pair = block * pairs_per_cta + threadIdx.x / per_pair;
    if (pair >= a.n) return;
    const int src = __ldg(a.src + pair), dst = __ldg(a.dst + pair);
    int tokens = a.tokens ? __ldg(a.tokens + pair) : a.m.page_size;
    if (src < 0 || dst < 0) return;
    if (src >= a.m.n_pages || dst >= a.m.n_pages || tokens < 0 || tokens > a.m.page_size) {
        atomicExch(a.m.status, kDeviceIndexCode);
        if (src >= a.m.n_pages || dst >= a.m.n_pages) return;
        tokens = min(max(tokens, 0), a.m.page_size);
    }
    const MoveKind& k = a.m.kind[kind];
    const unsigned char* from = a.m.base[kind][side] + (long long)src * k.page_stride;
    unsigned char* to = a.m.base[kind][side] + (long long)dst * k.page_stride;
    const int run = (runs.run_tokens ? runs.run_bytes * tokens : runs.run_bytes) / VB;  // vectors of a run
    const int outer = runs.outer_fixed > 0 ? runs.outer_fixed : tokens;
    const int total = outer * runs.inner * run;
    const bool single = outer * runs.inner == 1;
    const auto place = [&](int i) -> long long {
        if (single) return (long long)i * VB;
        const int r = (int)((unsigned)i / (unsigned)run), o = (int)((unsigned)r / (unsigned)runs.inner);
        return o * runs.outer_stride + (r - o * runs.inner) * runs.inner_stride + (long long)(i - r * run) * VB;
    };
    const int step = per_pair * chunks;
    for (int i0 = chunk * per_pair + threadIdx.x % per_pair; i0 < total; i0 += U * step) {
        Vec<VB> x[U];
        long long at[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            at[u] = i0 + u * step < total ? place(i0 + u * step) : -1;
            if (at[u] >= 0) x[u] = ld_move<VB>(from + at[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (at[u] >= 0) st_move<VB>(to + at[u], x[u]);
    }
}
template <int VB, int SVB>
__global__ void __launch_bounds__(kMoveThreads) kv_copy_pages_kernel(const __grid_constant__ CopyPagesArgs a)
{
    wait_for_previous_kernel();
    if ((int)blockIdx.y < a.m.sides) copy_pages<VB, 4>(a, a.runs[0], 0, (int)blockIdx.y);
    else if (SVB > 0) copy_pages<SVB == 0 ? 4 : SVB, 4>(a, a.runs[1], 1, (int)blockIdx.y - a.m.sides);
}

// ---- gaps -----------------------------------------------------------------------------------------------------

struct CompactArgs {
    MoveArgs m;
    const int32_t* page_table;
    long long page_table_stride;
    int page_table_width;
    int page_shift;  // log2(page_size), or -1
    const int32_t* starts;
    const int32_t* lens;
    const unsigned char* keep;
    long long keep_stride;
    int window;
    int32_t* new_lens;
    int n_seqs;
    int tasks_per_cta;  // of the sides x heads of a sequence
    int ctas_per_seq;
};

// Moves rows of the list, in order, for one warp's tasks.  The list ascends and a row never moves up, so nothing that a
// store overwrites is still to be read once all loads of its own batch and of those before it are done: the batch's loads
// come first, then its stores, and no other warp touches the same rows.
struct MoveList {
    long long src[kMoveThreads], dst[kMoveThreads];
};

// CTA: one sequence, some of its tasks (a side of a layer and a head each).  The window goes by in chunks of 256 tokens: who is
// kept and where it goes is found with two votes and a scan, the places of those that move are listed, and every warp moves
// the list's rows of its tasks, U accesses of a lane in flight.
template <int VB, int LANES, int U>
__global__ void __launch_bounds__(kMoveThreads) kv_compact_kernel(const __grid_constant__ CompactArgs a)
{
    __shared__ MoveList list[2];
    __shared__ int warp_kept[kMoveThreads / 32], warp_moved[kMoveThreads / 32];
    constexpr int WARPS = kMoveThreads / 32, ROWS = 32 / LANES;
    const int seq = (int)(blockIdx.x / (unsigned)a.ctas_per_seq), part = (int)(blockIdx.x - (unsigned)(seq * a.ctas_per_seq));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    wait_for_previous_kernel();
    const int start = __ldg(a.starts + seq), len = __ldg(a.lens + seq);
    const int n = start >= 0 && start <= len ? len - start : 0;
    bool fits = true;
    if (len >= 0) {
        const long long pages = ((long long)len + a.m.page_size - 1) / a.m.page_size;
        fits = start >= 0 && start <= len && n <= a.window && pages <= a.page_table_width;
    }
    if (len < 0 || !fits) {
        if (part == 0 && threadIdx.x == 0) {
            a.new_lens[seq] = len;
            if (!fits) atomicExch(a.m.status, kDeviceIndexCode);
        }
        return;
    }
    const unsigned char* keep = a.keep + (long long)seq * a.keep_stride;
    const int32_t* pages = a.page_table + (long long)seq * a.page_table_stride;
    const int first_task = part * a.tasks_per_cta, tasks = min(a.tasks_per_cta, a.m.sides * a.m.heads - first_task);
    const int row_vectors = a.m.kind[0].row_bytes / VB;
    const int turns = (row_vectors + LANES - 1) / LANES;  // accesses of a lane to one row
    int kept_before = 0;
    for (int c0 = 0; c0 < n; c0 += kMoveThreads) {
        const int i = c0 + (int)threadIdx.x;
        const bool kept = i < n && __ldg(keep + i) != 0;
        const unsigned kept_vote = __ballot_sync(0xFFFFFFFFu, kept);
        if (lane == 0) warp_kept[warp] = __popc(kept_vote);
        __syncthreads();  // (and the list of the chunk before is done with)
        int rank = kept_before + __popc(kept_vote & ((1u << lane) - 1u)), chunk_kept = 0;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            if (w < warp) rank += warp_kept[w];
            chunk_kept += warp_kept[w];
        }
        bool moved = kept && rank != i;
        unsigned src_page = 0, dst_page = 0, src_in = 0, dst_in = 0;
        if (moved) {
            const unsigned src = (unsigned)(start + i), dst = (unsigned)(start + rank);
            const unsigned sp = a.page_shift >= 0 ? src >> a.page_shift : src / (unsigned)a.m.page_size;
            const unsigned dp = a.page_shift >= 0 ? dst >> a.page_shift : dst / (unsigned)a.m.page_size;
            src_in = src - sp * (unsigned)a.m.page_size;
            dst_in = dst - dp * (unsigned)a.m.page_size;
            src_page = (unsigned)__ldg(pages + sp);
            dst_page = (unsigned)__ldg(pages + dp);
            if (src_page >= a.m.n_pages || dst_page >= a.m.n_pages) {  // (a negative number is a large one)
                atomicExch(a.m.status, kDeviceIndexCode);
                moved = false;
            }
        }
        const unsigned moved_vote = __ballot_sync(0xFFFFFFFFu, moved);
        if (lane == 0) warp_moved[warp] = __popc(moved_vote);
        __syncthreads();
        int at = __popc(moved_vote & ((1u << lane) - 1u)), rows = 0;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            if (w < warp) at += warp_moved[w];
            rows += warp_moved[w];
        }
        if (moved) {
#pragma unroll
            for (int kind = 0; kind < 2; ++kind) {
                list[kind].src[at] = (long long)src_page * a.m.kind[kind].page_stride + (long long)src_in * a.m.kind[kind].token_stride;
                list[kind].dst[at] = (long long)dst_page * a.m.kind[kind].page_stride + (long long)dst_in * a.m.kind[kind].token_stride;
            }
        }
        kept_before += chunk_kept;
        __syncthreads();
        if (rows == 0) continue;

        // Elements: the warp's tasks one behind another, each in batches of ROWS rows and `turns` accesses.
        const int batches = (rows + ROWS - 1) / ROWS, per_task = batches * turns;
        const int mine = (tasks - warp + WARPS - 1) / WARPS;  // tasks warp, warp + WARPS, ...
        int task = 0, batch = 0, turn = 0;
        for (int g0 = 0; g0 < mine * per_task; g0 += U) {
            Vec<VB> x[U];
            unsigned char* to[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                to[u] = nullptr;
                if (task < mine) {
                    const int row = batch * ROWS + lane / LANES, v = turn * LANES + lane % LANES;
                    if (row < rows && v < row_vectors) {
                        const int t = first_task + warp + task * WARPS, side = t / a.m.heads, head = t - side * a.m.heads;
                        unsigned char* base = a.m.base[0][side] + (long long)head * a.m.kind[0].head_stride + v * VB;
                        x[u] = ld_move<VB>(base + list[0].src[row]);
                        to[u] = base + list[0].dst[row];
                    }
                    if (++turn == turns) {
                        turn = 0;
                        if (++batch == batches) {
                            batch = 0;
                            ++task;
                        }
                    }
                }
            }
            __syncwarp();
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (to[u]) st_move<VB>(to[u], x[u]);
            __syncwarp();
        }
        // Scales: a side's are moved by the CTA that has its head 0, all heads by one warp.
        if (a.m.kinds == 2) {
            const int first_side = (first_task + a.m.heads - 1) / a.m.heads, last_side = (first_task + tasks - 1) / a.m.heads;
            for (int side = first_side + warp; side <= last_side; side += WARPS) {
                unsigned char* base = a.m.base[1][side];
                const int values = rows * a.m.heads;
                for (int g0 = 0; g0 < values; g0 += 32 * 4) {
                    uint32_t x[4];
                    long long to[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const int g = g0 + u * 32 + lane;
                        to[u] = -1;
                        if (g < values) {
                            const int row = g / a.m.heads;
                            const long long head = (long long)(g - row * a.m.heads) * a.m.kind[1].head_stride;
                            x[u] = ld_stream<4>(base + list[1].src[row] + head).w[0];
                            to[u] = list[1].dst[row] + head;
                        }
                    }
                    __syncwarp();
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        if (to[u] >= 0) *reinterpret_cast<uint32_t*>(base + to[u]) = x[u];
                    __syncwarp();
                }
            }
        }
    }
    if (part == 0 && threadIdx.x == 0) a.new_lens[seq] = start + kept_before;
}

}  // namespace rt
