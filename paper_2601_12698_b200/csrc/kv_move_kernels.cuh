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
// in flight at once.  Measured: 500 pages of 64 x 8 x 128 e4m3 in 16 layers, 2.16 GB: 283 us, 7.6 TB/s (a third of the sources is
// read twice, out of L2); 12 partly filled pages of 16 x 8 x 128 bf16 in 32 layers: 5.2 us in a graph.
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
    int pieces;         // of a row, each a task of its own
    int tasks_per_cta;  // of the sides x heads x pieces of a sequence
    int ctas_per_seq;
};

// Where a row that moves lies and where it goes, in bytes.
struct MoveRow {
    long long src, dst;
};
constexpr int kMoveTurns = 4;  // tokens of a thread that are looked at together
constexpr int kMoveChunk = kMoveThreads * kMoveTurns;

constexpr int kMoveStages = 3, kMoveDeepStages = 10;  // items of a warp under way, with two CTAs to an SM and with one
constexpr int kMoveAccesses = 4;  // accesses of a lane in an item
constexpr int kMoveScales = 16;   // scales of a thread under way

// Shared memory of a CTA: the lists, of elements and of scales, and the items under way.
inline int compact_smem(int kinds, int vector_bytes, int stages)
{
    return kinds * kMoveChunk * (int)sizeof(MoveRow) + (vector_bytes >= 4 ? kMoveThreads * stages * kMoveAccesses * vector_bytes : 0);
}

template <int VB>
__device__ __forceinline__ void cp_async(uint32_t to, const unsigned char* from)
{
    if constexpr (VB == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to), "l"(from), "n"(VB) : "memory");
}
template <int VB>
__device__ __forceinline__ Vec<VB> ld_slot(uint32_t at)
{
    Vec<VB> v;
    if constexpr (VB == 16) asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.w[0]), "=r"(v.w[1]), "=r"(v.w[2]), "=r"(v.w[3]) : "r"(at) : "memory");
    else if constexpr (VB == 8) asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(v.w[0]), "=r"(v.w[1]) : "r"(at) : "memory");
    else asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v.w[0]) : "r"(at) : "memory");
    return v;
}
// CTA: one sequence, some of its tasks (a side of a layer, a head and a piece of its rows each).  The window goes by in chunks of 1024 tokens: who is
// kept and where it goes is found with votes and a scan, the places of those that move are listed, and every warp moves the list's
// rows of its tasks, through shared memory (accesses narrower than 4 bytes: through registers).
//
// The list ascends and a row never moves up, so nothing that a store overwrites is still to be read once its own item and those before
// it are loaded: loads go ahead, stores never do.  No other warp touches a task's rows.
//
// Bound by HBM with many rows, where what counts is how much is under way and how little is worked out per access: a row's places are
// bytes in the list, a task's base is found once, a chunk's first scales are loaded ahead of its elements.  Measured: 12 sequences x 8
// layers x 8 heads of 128 int8, 1500 rows of each, 608 MB: 124 us, 4.9 TB/s, 0.76 of the copy bandwidth (145 with two items of a warp under
// way, in registers; 305 with every access's place worked out from page numbers and the scales moved by one warp; chunks of 512 tokens
// 131, of 2048 139; CTAs of 4 warps 141, of 16 141).  What is left: beginnings and ends of chunks, and sequences of unequal lengths.
// 40 sequences x 32 layers, two or three rows each: 7.1 us in a graph.
template <int VB, int LANES, int STAGES>
__global__ void __launch_bounds__(kMoveThreads, 2) kv_compact_kernel(const __grid_constant__ CompactArgs a)
{
    constexpr int WARPS = kMoveThreads / 32, ROWS = 32 / LANES, U = kMoveAccesses;
    __shared__ int warp_count[kMoveTurns][WARPS];
    extern __shared__ __align__(16) unsigned char shared[];
    MoveRow(*const list)[kMoveChunk] = reinterpret_cast<MoveRow(*)[kMoveChunk]>(shared);  // of elements, and of scales
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(shared) + (uint32_t)(a.m.kinds * sizeof(MoveRow) * kMoveChunk) +
                          (threadIdx.x >> 5) * (STAGES * U * 32 * VB) + (threadIdx.x & 31) * VB;
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
    const int per_side = a.m.heads * a.pieces, first_task = part * a.tasks_per_cta, tasks = min(a.tasks_per_cta, a.m.sides * per_side - first_task);
    const int row_vectors = a.m.kind[0].row_bytes / VB;
    // Place of a thread's j-th token among those of the chunk for which `mine` holds, and their number.
    const auto scan = [&](const bool (&mine)[kMoveTurns], int (&at)[kMoveTurns]) -> int {
#pragma unroll
        for (int j = 0; j < kMoveTurns; ++j) {
            const unsigned vote = __ballot_sync(0xFFFFFFFFu, mine[j]);
            at[j] = __popc(vote & ((1u << lane) - 1u));
            if (lane == 0) warp_count[j][warp] = __popc(vote);
        }
        __syncthreads();
        int total = 0;
#pragma unroll
        for (int j = 0; j < kMoveTurns; ++j)
#pragma unroll
            for (int w = 0; w < WARPS; ++w) {
                if (w == warp) at[j] += total;
                total += warp_count[j][w];
            }
        __syncthreads();
        return total;
    };
    int kept_before = 0;
    for (int c0 = 0; c0 < n; c0 += kMoveChunk) {
        bool mine[kMoveTurns];
        int rank[kMoveTurns], at[kMoveTurns];
#pragma unroll
        for (int j = 0; j < kMoveTurns; ++j) {
            const int i = c0 + j * kMoveThreads + (int)threadIdx.x;
            mine[j] = i < n && __ldg(keep + i) != 0;
        }
        const int chunk_kept = scan(mine, rank);
        unsigned src_page[kMoveTurns], src_in[kMoveTurns], dst_page[kMoveTurns], dst_in[kMoveTurns];
#pragma unroll
        for (int j = 0; j < kMoveTurns; ++j) {
            const int i = c0 + j * kMoveThreads + (int)threadIdx.x;
            rank[j] += kept_before;
            mine[j] = mine[j] && rank[j] != i;
            if (mine[j]) {
                const unsigned src = (unsigned)(start + i), dst = (unsigned)(start + rank[j]);
                const unsigned sp = a.page_shift >= 0 ? src >> a.page_shift : src / (unsigned)a.m.page_size;
                const unsigned dp = a.page_shift >= 0 ? dst >> a.page_shift : dst / (unsigned)a.m.page_size;
                src_page[j] = (unsigned)__ldg(pages + sp);
                dst_page[j] = (unsigned)__ldg(pages + dp);
                src_in[j] = src - sp * (unsigned)a.m.page_size;
                dst_in[j] = dst - dp * (unsigned)a.m.page_size;
                if (src_page[j] >= a.m.n_pages || dst_page[j] >= a.m.n_pages) {  // (a negative number is a large one)
                    atomicExch(a.m.status, kDeviceIndexCode);
                    mine[j] = false;
                }
            }
        }
        const int rows = scan(mine, at);
#pragma unroll
        for (int j = 0; j < kMoveTurns; ++j)
            if (mine[j]) {
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    if (k < a.m.kinds)
                        list[k][at[j]] = {(long long)(times(src_page[j], a.m.kind[k].page_stride) + times(src_in[j], a.m.kind[k].token_stride)),
                                          (long long)(times(dst_page[j], a.m.kind[k].page_stride) + times(dst_in[j], a.m.kind[k].token_stride))};
            }
        kept_before += chunk_kept;
        __syncthreads();

        // Elements: many rows one task at a time, few rows U tasks at a time.  An item is U accesses of a lane: TU tasks, BU batches of ROWS
        // rows.  A warp goes through its items in order, STAGES under way.
        const auto move = [&](auto tasks_at_once) {
            constexpr int TU = decltype(tasks_at_once)::value, BU = U / TU;
            const int batches = (rows + ROWS * BU - 1) / (ROWS * BU);
            struct Cursor {
                int task, batch;
                unsigned char* base[TU];
            };
            const auto place = [&](Cursor& c) {
#pragma unroll
                for (int i = 0; i < TU; ++i) {
                    const int t = first_task + c.task + i * WARPS, side = t / per_side, rest = t - side * per_side;
                    int head = rest, v = lane % LANES;
                    if (a.pieces > 1) {
                        head = rest / a.pieces;
                        v += (rest - head * a.pieces) * LANES;
                    }
                    c.base[i] = c.task + i * WARPS < tasks && v < row_vectors ? a.m.base[0][side] + (long long)head * a.m.kind[0].head_stride + v * VB : nullptr;
                }
            };
            const auto next = [&](Cursor& c) {
                if (++c.batch < batches) return;
                c.batch = 0;
                c.task += TU * WARPS;
                place(c);
            };
            const int items = warp < tasks ? (tasks - warp + TU * WARPS - 1) / (TU * WARPS) * batches : 0;
            Cursor to = {warp, 0, {}};
            place(to);
            if constexpr (VB >= 4) {
                Cursor from = to;
                int fetched = 0, slot = 0;
                const auto fetch = [&](int stage) {
                    if (fetched < items) {
#pragma unroll
                        for (int u = 0; u < U; ++u) {
                            const int r = (from.batch * BU + u / TU) * ROWS + lane / LANES;
                            if (from.base[u % TU] && r < rows) cp_async<VB>(ring + (stage * U + u) * 32 * VB, from.base[u % TU] + list[0][r].src);
                        }
                        ++fetched;
                        next(from);
                    }
                    asm volatile("cp.async.commit_group;" ::: "memory");
                };
#pragma unroll
                for (int s = 0; s < STAGES; ++s) fetch(s);
                for (int n = 0; n < items; ++n) {
                    asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
                    __syncwarp();
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const int r = (to.batch * BU + u / TU) * ROWS + lane / LANES;
                        if (to.base[u % TU] && r < rows) st_move<VB>(to.base[u % TU] + list[0][r].dst, ld_slot<VB>(ring + (slot * U + u) * 32 * VB));
                    }
                    next(to);
                    fetch(slot);
                    slot = slot + 1 == STAGES ? 0 : slot + 1;
                }
            } else {
                for (int n = 0; n < items; ++n, next(to)) {
                    Vec<VB> x[U];
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const int r = (to.batch * BU + u / TU) * ROWS + lane / LANES;
                        if (to.base[u % TU] && r < rows) x[u] = ld_move<VB>(to.base[u % TU] + list[0][r].src);
                    }
                    __syncwarp();
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const int r = (to.batch * BU + u / TU) * ROWS + lane / LANES;
                        if (to.base[u % TU] && r < rows) st_move<VB>(to.base[u % TU] + list[0][r].dst, x[u]);
                    }
                    __syncwarp();
                }
            }
        };
        // Scales: a side's are moved by the CTA that has its first task, all heads by all warps, a batch's loads ahead of its stores; the
        // first batch's ahead of the elements, which cover their wait.
        const int values = a.m.kinds == 2 ? rows * a.m.heads : 0;
        const int first_side = (first_task + per_side - 1) / per_side, last_side = (first_task + tasks - 1) / per_side;
        uint32_t y[kMoveScales];
        const auto scale_place = [&](int g, bool to) -> long long {
            const int r = (int)((unsigned)g / (unsigned)a.m.heads);
            return (to ? list[1][r].dst : list[1][r].src) + (long long)(g - r * a.m.heads) * a.m.kind[1].head_stride;
        };
        const auto fetch_scales = [&](int side, int g0) {
#pragma unroll
            for (int e = 0; e < kMoveScales; ++e) {
                const int g = g0 + e * kMoveThreads + (int)threadIdx.x;
                if (g < values) y[e] = ld_stream<4>(a.m.base[1][side] + scale_place(g, false)).w[0];
            }
        };
        const auto store_scales = [&](int side, int g0) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < kMoveScales; ++e) {
                const int g = g0 + e * kMoveThreads + (int)threadIdx.x;
                if (g < values) *reinterpret_cast<uint32_t*>(a.m.base[1][side] + scale_place(g, true)) = y[e];
            }
        };
        if (values > 0 && first_side <= last_side) fetch_scales(first_side, 0);
        if (rows > 2 * ROWS) move(std::integral_constant<int, 1>());
        else if (rows > 0) move(std::integral_constant<int, U>());
        for (int side = first_side; side <= last_side; ++side)
            for (int g0 = 0; g0 < values; g0 += kMoveThreads * kMoveScales) {
                if (side != first_side || g0 != 0) fetch_scales(side, g0);
                store_scales(side, g0);
            }
    }
    if (part == 0 && threadIdx.x == 0) a.new_lens[seq] = start + kept_before;
}

}  // namespace rt
