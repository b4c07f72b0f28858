// Attention of whole prompts on the fifth-generation tensor cores (sm_100a, tcgen05 + tensor memory + TMA).
//
//     S = Q K^T,  W = 2^(score_scale S - m),  O = W V      in one pass over the keys, a running reference m and sum per row.
//
// A "row" is one query head of one query token.  The rows of one key/value head are packed token by token, its `group` query heads
// side by side, so that a tile of 128 rows is 128 / group tokens: short sequences and single tokens fill tiles as well as the
// grouping lets them, and a causal block spans few keys.  An item of work is a block of 256 rows (two tiles, one for each softmax
// stream) of one sequence and key/value head, and a range of its key tiles of 128.
//
// One CTA to an SM, 16 warps, each CTA working through items:
//   warps 0-3, 4-7   two softmax streams of 128 rows, one row to a thread (tensor memory lane = row): scores from tensor memory, m and
//                    the sum in registers, the weights back over the scores as the 16-bit left operand of the second product;
//   warps 8-11       look through the values of tiles that not every row sees (see below);
//   warps 12, 13     issue the products, each for its stream (heads of more than 128: one the outputs', one the scores');
//   warp 14          fetches queries, keys and values with TMA into rings of 128-byte-swizzled tiles;
//   warp 15          works out the items.
// The streams share keys and values and take turns on the tensor cores: while one's scores are exponentiated the other's products
// run.  The queries and first tiles of the next item are fetched, and its first scores computed, while this one's results leave.
//
// Heads of more than 128 (DP = 256): tensor memory has no room for two outputs of 256, so both streams take the same 128 rows and one output,
// the first the first 64 keys of every tile and the second the others.  What is left of tensor memory holds the scores of two tiles: the
// next tile's are computed while this one's are exponentiated.
//
// The reference m is moved only when a score exceeds it by 8, as in the prefix kernel: weights reach 2^8 of its own.  Streams that share rows share
// the reference, as if the second's keys came behind the first's: a stream works with the reference that it knows, and before it
// announces its weights it waits until the other has announced those that come before, looks whether the reference has been moved, and
// if so works again.
//
// fp16 weights are taken 2^7 times as large, up to 2^15, so that those far below the reference keep their bits: they are rounded to multiples
// of 2^-31 of the reference's weight at the least, off by 2^-32 of it.  (Without the factor, weights e^-18 of the first key's became zeros.)
//
// Values that a row does not see meet a weight of zero in the product, and 0 * inf is NaN.  Where a tile has such values (the diagonal, the
// sequence's end), warps 8-11 replace infinities and NaN among the keys that not all rows see by zeros before the product, and
// the rows that do see them add them when they are written.
//
// Bounds: 4 * 128 * 128 * dim flops and 128 * 128 exponentials per tile and stream; at dim 128 the tensor cores need 1024
// cycles for that and the SM's 16 exponentials a cycle 1024 as well.  Products read their operands from shared memory at 128 bytes a
// cycle: 128 x 64 x 16 take 48 cycles instead of 32, 128 x 128 x 16 the 64 that they should, and with the left operand in tensor memory both
// do.  So at dim 128 a stream's products take 768 + 512 cycles, both streams' 2560 of the 3120 that a tile takes: operands first, then the chain
// from scores to weights; the power limit decides how long a cycle is.  Scores 64 keys at a time, which let the tensor cores go on while the other half is
// exponentiated, are worth that at dims up to 128 (one product of 128 keys: 563 us, not 440).
//
// Measured (TFLOP/s of the causal pairs; the clock drops to 1.64 GHz under the power limit in the long ones):
//   8192 tokens, 32 heads on 8 of 128: 440 us, 1250; the tensor cores busy in 64 % of the cycles, the special function unit in 64 %;
//   16384 tokens: 1700 .. 2060 us, 1290 .. 1070 by the card; heads of 64, 8192 tokens: 355 us, special function unit 74 %;
//   32 heads on 4 of 256, 4096 tokens: 248 us, 1110; shared memory: 2560 cycles of a tile's 3600 go to operands and to what TMA writes;
//   100 tokens: 9.9 us, one CTA's chain: beginning 0.4, item 1.2, first copies 0.7, products and softmax 3, results 1.2, launch.
#pragma once

#include <cuda.h>

#include "attend_common.cuh"
#include "tensor_core.cuh"

namespace rt {

constexpr int kPromptThreads = 512;
constexpr int kPromptTile = 128;  // keys of a tile, rows of a stream
constexpr int kPromptItems = 4;   // ring of items
constexpr int kPromptLanded = 8;  // masked tiles whose values can be under way: more than the ring holds
constexpr int kPromptMaxParts = 32;

struct PromptArgs {
    const int32_t* q_starts;
    const int32_t* k_starts;
    int n_seqs;
    int q_tokens, k_tokens;
    int causal;
    int kv_heads, group, dim;
    int group_inverse;  // 2^16 / group, rounded up: i / group is (i * group_inverse) >> 16 for i < 128
    int stream_tokens;  // tokens of a stream's 128 rows
    int block_tokens;   // tokens of an item
    int parts;          // ranges of key tiles that every block is cut into
    float score_scale;  // softmax_scale * log2(e)
    const unsigned char* v;
    long long v_token_stride, v_head_stride;  // bytes
    void* out;        // [token][head][dim]
    float* lse;       // [token][head] or NULL
    float* part_out;  // parts > 1: [part][token][head][dim], normalised
    float* part_lse;  // [part][token][head], base 2
    int* part_ready;  // parts > 1: set to 1 when the starts are sound, or to 0, and then nothing is written
    int wide_rows;    // rows of out, or of part_out, are multiples of 32 bytes
    int* status;
    unsigned wait_polls;
    unsigned more_waits;  // what a wait for an item is given beyond the second of every wait: see prompt_more_waits
    int drop_copies;
};

// A warp may have to wait for an item from its beginning to its end, or until it is found.  That may take 16384 cycles for each key tile (one
// takes 2500 to 6000, by the heads' size and where it is read from) and 1024 for each sequence (they are gone through 32 at a time, up
// to 32 times, at about 800 cycles): as many more waits, of kMbarrierCycleLimit each.  None up to 15 million keys and 1.9 million sequences.  (With
// a single one, 2^24 sequences whose blocks' costs lie in more than five powers of two ended as if a wait had been without hope.)
inline unsigned prompt_more_waits(long long k_tokens, long long n_seqs)
{
    return (unsigned)((k_tokens / kPromptTile * 16384 + n_seqs * 1024) / kMbarrierCycleLimit);
}

struct PromptItem {
    int valid;
    int q_row, tokens;    // first query row and number of query tokens
    int k_row;            // first key row of the sequence
    int last_key;         // last key that the first token sees (may be negative)
    int key_step;         // 1: every further token sees one key more (causal)
    int end_key;          // keys of the sequence
    int tile0, tile1;     // this part's key tiles
    int masked_from;      // first tile with keys that not every row sees
    int kv_head, part;
    int turned;           // 1: the first stream takes the rows behind, the second those in front
    int bad_values;       // infinities or NaN were taken out of the masked tiles' values
};

template <int DP>
struct PromptShape {
    static constexpr int kBlocks = DP / 64;               // column blocks of a tile of queries, keys or values
    static constexpr bool kSharedRows = DP == 256;        // both streams take the same rows
    static constexpr int kCols = DP == 256 ? 128 : DP;    // dims that a stream writes
    static constexpr int kValueRows = kSharedRows ? kPromptTile / 2 : kPromptTile;  // keys of a box of values: those of a stream
    static constexpr int kBlockBytes = kPromptTile * 128;
    // The ring: 160 KB, a block to a slot, or both of heads of 128.  (Heads of 128, 8192 tokens: 435 us with two, 445 with one.)
    static constexpr int kSlotBlocks = DP == 128 ? 2 : 1;
    static constexpr int kUnits = kBlocks / kSlotBlocks;  // slots of a tile
    static constexpr int kSlotBytes = kSlotBlocks * kBlockBytes;
    static constexpr int kSlots = 10 / kSlotBlocks;
    // Streams that share rows: a ring of its own for the keys, a tile of them, and one for the values, two slots to a stream's of a tile.  (Keys
    // are done with long before the values fetched ahead of them.  One ring for both, 4096 tokens, 32 heads on 4 of 256: 248 us.)
    static constexpr int kKeySlots = kBlocks, kValuePairs = (kSlots - kKeySlots) / 2;
    static constexpr int kQueryBytes = kBlocks * kBlockBytes;  // of one stream
    static constexpr int kQueries = kSharedRows ? 1 : 2;
    static constexpr size_t kRingAt = (size_t)kQueries * kQueryBytes;
    static constexpr size_t kSmem = kRingAt + (size_t)kSlots * kSlotBytes + 1024;  // 1024: alignment of the tiles
    static constexpr int kSoftmaxRegs = 160;  // of 2 * 128 for a softmax thread and one of another role
};

// log2 of the factor that weights and their sum are held with.  (bf16 has binary32's range and needs none.)
template <typename T>
__device__ constexpr float kPromptWeightShift = std::is_same<T, __half>::value ? 7.f : 0.f;

__device__ __forceinline__ void tma_load_3d(void* dst, const CUtensorMap* map, int x, int y, int z, uint64_t* bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(smem_u32(dst)),
                 "l"(map), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z) : "memory");
}

// 32 bytes of a row, of `columns` columns from `col` on, in one access or, where places are multiples of 16 bytes only, in two.
template <int WORDS>
__device__ __forceinline__ void store_row(unsigned char* to, const uint32_t* x, int col, int columns, const PromptArgs& a)
{
    if (a.wide_rows) {
        Vec<32> v;
#pragma unroll
        for (int k = 0; k < WORDS; ++k) v.w[k] = x[k];
        if (col < a.dim) st_stream<32>(to, v);
    } else {
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (col + h * columns / 2 < a.dim) *reinterpret_cast<uint4*>(to + h * 16) = make_uint4(x[4 * h], x[4 * h + 1], x[4 * h + 2], x[4 * h + 3]);
    }
}

// A sequence as the items see it.  `sound`: its starts do not descend and lie in the tensors; otherwise it has no rows.
struct PromptSequence {
    int q_row, q_len, k_row, k_len;
    bool sound;
};
__device__ __forceinline__ PromptSequence prompt_sequence(const PromptArgs& a, int i)
{
    const int q0 = __ldg(a.q_starts + i), q1 = __ldg(a.q_starts + i + 1), k0 = __ldg(a.k_starts + i), k1 = __ldg(a.k_starts + i + 1);
    const bool sound = 0 <= q0 && q0 <= q1 && q1 <= a.q_tokens && 0 <= k0 && k0 <= k1 && k1 <= a.k_tokens;
    return {sound ? q0 : 0, sound ? q1 - q0 : 0, sound ? k0 : 0, sound ? k1 - k0 : 0, sound};
}

// The order in which blocks are taken, whole warps: the most expensive first, so that the CTAs end together.  (17 sequences of up to 1500
// tokens, 8 heads of 64: 42.8 us, 61.1 in the sequences' order.)  A block's cost is counted in blocks of keys: causal blocks of a sequence cost base, base + 1, ...; otherwise all the same.
// Up to 128 sequences are kept in registers and the order is exact.  More are gone through 32 at a time, once for each power of two of the
// cost that occurs, and a CTA's ranks ascend, so that it goes through them once in all (looked up for every block instead: 1000 sequences
// of 16 tokens, 32 heads on 8 of 128, 854 us; 4000: 12.9 ms).
struct PromptOrder {
    static constexpr int kKept = 4;  // sequences that a lane keeps in registers
    const PromptArgs& a;
    int blocks[kKept], base[kKept];
    long long total;
    int cost;              // the cost found last: no further block costs more
    long long dearer;      // blocks that cost more than `cost`
    long long not_cheaper; // blocks that cost `cost` or more

    __device__ __forceinline__ bool shape(int i, int& n, int& first) const
    {
        const PromptSequence s = prompt_sequence(a, i);
        n = (s.q_len + a.block_tokens - 1) / a.block_tokens;
        first = a.causal ? max(s.k_len - s.q_len, 0) / a.block_tokens : s.k_len / a.block_tokens;
        return s.sound;
    }
    __device__ __forceinline__ int count(int n, int first, int c) const  // blocks that cost c or more
    {
        return a.causal ? min(max(first + n - c, 0), n) : (first >= c ? n : 0);
    }
    template <typename F>
    __device__ __forceinline__ void each(F f) const  // f(sequence, blocks, base); up to 32 * kKept sequences, 32 lanes' at a time
    {
        const int lane = threadIdx.x & 31;
#pragma unroll
        for (int j = 0; j < kKept; ++j)
            if (j * 32 < a.n_seqs) f(j * 32 + lane, blocks[j], base[j]);
    }
    __device__ __forceinline__ long long all(int c) const
    {
        long long sum = 0;
        each([&](int, int n, int first) { sum += __reduce_add_sync(0xFFFFFFFFu, (unsigned)count(n, first, c)); });
        return sum;
    }
    static __device__ __forceinline__ int cost_class(int c) { return 32 - __clz(c); }  // 0: 0, 1: 1, 2: 2 and 3, 3: 4 .. 7, ...
    bool sound;        // all sequences are; otherwise there are no blocks
    unsigned classes;  // more than 32 * kKept sequences: those of the costs that occur
    int at_class, at_group, at_blocks, at_base;
    long long passed;  // blocks of dearer classes and, in this one, of the groups before
    __device__ __forceinline__ explicit PromptOrder(const PromptArgs& args) : a(args)
    {
        const int lane = threadIdx.x & 31;
        bool mine = true;
#pragma unroll
        for (int j = 0; j < kKept; ++j) {
            blocks[j] = base[j] = 0;
            if (j * 32 + lane < a.n_seqs) mine = shape(j * 32 + lane, blocks[j], base[j]) && mine;
        }
        long long sum = 0;
#pragma unroll
        for (int j = 0; j < kKept; ++j) sum += __reduce_add_sync(0xFFFFFFFFu, (unsigned)blocks[j]);
        if (a.n_seqs > kKept * 32) {
            unsigned occur = 0;
            const auto note = [&](int n, int first) {
                if (n > 0) occur |= (0xFFFFFFFFu >> (31 - cost_class(first + (a.causal ? n - 1 : 0)))) & (0xFFFFFFFFu << cost_class(first));
            };
#pragma unroll
            for (int j = 0; j < kKept; ++j) note(blocks[j], base[j]);
#pragma unroll 4
            for (int i0 = kKept * 32; i0 < a.n_seqs; i0 += 32) {
                int n = 0, first = 0;
                if (i0 + lane < a.n_seqs) mine = shape(i0 + lane, n, first) && mine;
                note(n, first);
                sum += __reduce_add_sync(0xFFFFFFFFu, (unsigned)n);
            }
            classes = __reduce_or_sync(0xFFFFFFFFu, occur);
            at_class = cost_class((int)classes) - 1;
            at_group = 0;
            at_blocks = blocks[0];
            at_base = base[0];
            passed = 0;
        }
        sound = __all_sync(0xFFFFFFFFu, mine);
        total = sound ? sum : 0;
        cost = -1;
        dearer = not_cheaper = 0;
    }
    // Many sequences: sequence and block of place `rank` (ranks ascend from call to call); -1: the starts have changed meanwhile.
    __device__ __forceinline__ void find_among_many(long long rank, int& seq, int& block)
    {
        const int lane = threadIdx.x & 31;
        seq = -1;
        block = 0;
        while (at_class >= 0) {
            const int low = at_class == 0 ? 0 : 1 << (at_class - 1);
            const int dearer_here = at_class == 31 ? 0 : count(at_blocks, at_base, 1 << at_class), here = count(at_blocks, at_base, low) - dearer_here;
            int upto = here;
#pragma unroll
            for (int s = 1; s < 32; s <<= 1) {
                const int x = __shfl_up_sync(0xFFFFFFFFu, upto, s);
                if (lane >= s) upto += x;
            }
            const unsigned mine = __ballot_sync(0xFFFFFFFFu, rank < passed + upto);
            if (mine) {
                const int from = __ffs(mine) - 1;
                seq = at_group * 32 + from;
                const int i = (int)(rank - passed) - __shfl_sync(0xFFFFFFFFu, upto - here, from);  // of the sequence's blocks in this class
                const int n = __shfl_sync(0xFFFFFFFFu, at_blocks, from);
                block = a.causal ? n - 1 - __shfl_sync(0xFFFFFFFFu, dearer_here, from) - i : i;
                return;
            }
            passed += __shfl_sync(0xFFFFFFFFu, upto, 31);
            if (++at_group * 32 >= a.n_seqs) {
                at_group = 0;
                at_class = cost_class((int)(classes & ((1u << at_class) - 1))) - 1;
            }
            at_blocks = at_base = 0;
            if (at_group * 32 + lane < a.n_seqs) shape(at_group * 32 + lane, at_blocks, at_base);
        }
    }
    // The same without an order, for a grid that takes all blocks at once.
    __device__ __forceinline__ void find_any(long long rank, int& seq, int& block) const
    {
        long long before = 0;
        seq = -1;
        each([&](int i, int n, int) {
            int upto = n;
#pragma unroll
            for (int s = 1; s < 32; s <<= 1) {
                const int x = __shfl_up_sync(0xFFFFFFFFu, upto, s);
                if ((int)(threadIdx.x & 31) >= s) upto += x;
            }
            const unsigned mine = __ballot_sync(0xFFFFFFFFu, seq < 0 && rank < before + upto);
            if (mine && seq < 0) {
                const int from = __ffs(mine) - 1;
                block = (int)(rank - before) - __shfl_sync(0xFFFFFFFFu, upto - n, from);
                seq = __shfl_sync(0xFFFFFFFFu, i, from);
            }
            before += __shfl_sync(0xFFFFFFFFu, upto, 31);
        });
    }
    // Sequence and block of place `rank`; ranks ascend from call to call.
    __device__ __forceinline__ void find(long long rank, int& seq, int& block)
    {
        if (cost < 0) {
            int top = 0;
            each([&](int, int n, int first) { top = max(top, first + (a.causal ? n : 0)); });
            cost = (int)__reduce_max_sync(0xFFFFFFFFu, (unsigned)top);
            not_cheaper = all(cost);
        }
        if (rank >= not_cheaper) {
            // the largest cost with more than `rank` blocks that cost it or more: mostly the next one down
            int lo = 0, hi = cost;  // all(lo) > rank >= all(hi)
            int step = 1;
            while (hi - step > 0) {
                if (all(hi - step) > rank) {
                    lo = hi - step;
                    break;
                }
                hi -= step;
                step *= 2;
            }
            while (hi - lo > 1) {
                const int mid = (lo + hi) / 2;
                if (all(mid) > rank) lo = mid;
                else hi = mid;
            }
            cost = lo;
            dearer = all(lo + 1);
            not_cheaper = all(lo);
        }
        int left = (int)(rank - dearer);
        int found_seq = -1, found_block = 0;
        each([&](int i, int n, int first) {
            // blocks of this sequence that cost exactly `cost`
            const int here = count(n, first, cost) - count(n, first, cost + 1);
            int before = here;
#pragma unroll
            for (int s = 1; s < 32; s <<= 1) {
                const int x = __shfl_up_sync(0xFFFFFFFFu, before, s);
                if ((int)(threadIdx.x & 31) >= s) before += x;
            }
            const int sum = __shfl_sync(0xFFFFFFFFu, before, 31);
            before -= here;
            const unsigned mine = __ballot_sync(0xFFFFFFFFu, found_seq < 0 && left >= before && left < before + here);
            if (mine) {
                const int from = __ffs(mine) - 1;
                found_seq = __shfl_sync(0xFFFFFFFFu, i, from);
                found_block = __shfl_sync(0xFFFFFFFFu, a.causal ? cost - first : left - before, from);
            } else if (found_seq < 0) {
                left -= sum;
            }
        });
        seq = found_seq;
        block = found_block;
    }
};

template <typename T, int DP>
__global__ void __launch_bounds__(kPromptThreads, 1) prompt_attention_kernel(const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map,
                                                                            const __grid_constant__ CUtensorMap v_map, const __grid_constant__ PromptArgs a)
{
    using S = PromptShape<DP>;
    constexpr bool kSharedRows = S::kSharedRows;
    constexpr int kHalves = kSharedRows ? 1 : 2;  // halves of a tile that a stream takes
    constexpr int kBlocks = S::kBlocks, kSlotBlocks = S::kSlotBlocks, kUnits = S::kUnits;
    constexpr uint32_t kScoreIdesc = tc_instruction<T>(kSharedRows ? kPromptTile : kPromptTile / 2, false, false);
    constexpr uint32_t kColO = 2 * kPromptTile, kBufferCols = kSharedRows ? kPromptTile : 64;  // columns of a buffer of scores, of both streams where they share rows

    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    unsigned char* ring = smem + S::kRingAt;
    __shared__ __align__(8) uint64_t full[S::kSlots], empty[S::kSlots], item_full[kPromptItems], item_free[kPromptItems], landed[kPromptLanded], q_full, q_free, s_full[2][2],
        p_full[2][2], o_done[2][2], o_full[2], sums_full[2], results_read, drained[2];
    __shared__ PromptItem items[kPromptItems];
    __shared__ uint32_t tmem_base;
    __shared__ float row_reference[kSharedRows ? kPromptTile : 1], row_sum[kSharedRows ? kPromptTile : 1];  // what streams that share rows tell one another

    const int tid = threadIdx.x, warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0), lane = tid & 31;
    if (tid < S::kSlots) {
        mbarrier_init(&full[tid], 1);
        mbarrier_init(&empty[tid], kSharedRows ? 1 : 2);
    } else if (tid >= 32 && tid < 32 + kPromptItems) {
        mbarrier_init(&item_full[tid - 32], 1);
        mbarrier_init(&item_free[tid - 32], 15);  // warps that read it: 8 softmax, 4 looking, 2 issuing, 1 fetching
        items[tid - 32].valid = 0;
    } else if (tid >= 64 && tid < 66) {
        const int i = tid - 64;
        mbarrier_init(&s_full[i][0], 1);
        mbarrier_init(&s_full[i][1], 1);
        mbarrier_init(&p_full[i][0], 128);
        mbarrier_init(&p_full[i][1], 128);
        mbarrier_init(&o_done[i][0], 1);
        mbarrier_init(&o_done[i][1], 1);
        mbarrier_init(&o_full[i], 1);
        mbarrier_init(&drained[i], 1);
    } else if (tid >= 96 && tid < 96 + kPromptLanded) {
        mbarrier_init(&landed[tid - 96], 1);
    } else if (tid == 127) {
        mbarrier_init(&q_full, 1);
        mbarrier_init(&q_free, kSharedRows ? 1 : 2);
        mbarrier_init(&sums_full[0], 128);
        mbarrier_init(&sums_full[1], 128);
        mbarrier_init(&results_read, 128);
    } else if (tid >= 128 && tid < 131) {
        const CUtensorMap* map = tid == 128 ? &k_map : tid == 129 ? &v_map : &q_map;
        asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
    }
    if (warp == 12) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&tmem_base)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_base;
    wait_for_previous_kernel();

    // Every wait is bounded.  A thread whose wait has run out stops waiting, goes on to the end of the item, so that barriers and votes
    // are still met, and then ends; the status word says that the results are not valid.  Nothing that it goes on with leads outside
    // the tensors: items are published ones, or none.
    bool ok = true;
    auto wait = [&](uint64_t* bar, uint32_t parity) {
        if (ok) ok = mbarrier_wait_sleeping(bar, parity, a.wait_polls);
    };
    auto wait_item = [&](uint64_t* bar, uint32_t parity) {
        for (unsigned more = a.more_waits; ok && !mbarrier_wait_sleeping(bar, parity, a.wait_polls); --more) ok = more > 0;
    };
    // The next item (`n`-th of this CTA); false: there is none.
    auto next_item = [&](int n, PromptItem& item) -> bool {
        wait_item(&item_full[n % kPromptItems], (n / kPromptItems) & 1);
        if (!__all_sync(0xFFFFFFFFu, ok)) return false;
        item = items[n % kPromptItems];
        return item.valid != 0;
    };
    auto done_with_item = [&](int n) {
        __syncwarp();
        if (lane == 0) mbarrier_arrive(&item_free[n % kPromptItems]);
    };
    // Key tiles that a stream's rows see: all of the item's but the last ones, or none.
    auto stream_tiles = [&](const PromptItem& item, int s) -> int {
        const int first = kSharedRows ? 0 : (s ^ item.turned) * a.stream_tokens;
        if (first >= item.tokens) return 0;
        const int last_token = kSharedRows ? item.tokens - 1 : min(item.tokens, first + a.stream_tokens) - 1;
        const int last = min(item.last_key + item.key_step * last_token, item.end_key - 1);
        return min(item.tile1, (last + kPromptTile) / kPromptTile) - item.tile0;  // (last >= -kPromptTile where it matters: none is cut to 0 by its users)
    };

    if (warp < 8) {
        // ---- softmax streams ----
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(S::kSoftmaxRegs));
        const int s = warp >> 2, r = (warp & 3) * 32 + lane;
        const uint32_t lane_base = tmem + ((uint32_t)(warp & 3) << 21);
        const uint32_t s_col = lane_base + s * (kSharedRows ? 64 : kPromptTile), o_col = lane_base + kColO + s * S::kCols;
        const int first_key = kSharedRows ? s * 64 : 0;  // of a tile's, the first that this stream takes
        const int n_heads = a.kv_heads * a.group;
        const float c = fmaxf(a.score_scale, 1.17549435e-38f);  // (a scale of zero would make NaN of hidden scores: the smallest normal number does instead)
        const float2x c2 = pack_f2(c, c);
        const int row_token = r * a.group_inverse >> 16;
        const long long n_rows = (long long)a.q_tokens * n_heads;
        uint32_t tiles_done = 0, results_done = 0;  // of this stream
        PromptItem item;
        for (int n = 0; next_item(n, item); ++n) {
            const int first_token = kSharedRows ? 0 : (s ^ item.turned) * a.stream_tokens;
            const int my_tiles = max(stream_tiles(item, s), 0);
            // Row i of this stream's 128 counted in [token][head] rows from the item's first token and head, -1: no such row.
            const auto row_index = [&](int i) -> int {
                const int t = i * a.group_inverse >> 16, token = first_token + t;
                if (t >= a.stream_tokens || token >= item.tokens) return -1;
                return token * n_heads + (i - t * a.group);
            };
            // last key that this row sees; rows that are not there see all
            const bool there = row_token < a.stream_tokens && first_token + row_token < item.tokens;
            const int last = there ? min(item.last_key + item.key_step * (first_token + row_token), item.end_key - 1) : item.end_key - 1;
            float m = -INFINITY, l = 0.f;
            const auto hide = [](uint32_t(&v)[32], int seen) {  // the keys that a row does not see
#pragma unroll
                for (int k = 0; k < 32; ++k)
                    if (k > seen) v[k] = 0xFF800000u;
            };
            if (kSharedRows && s == 1 && my_tiles > 0) {  // its first reference is what the first stream has found
                wait(&p_full[0][tiles_done & 1], (tiles_done >> 1) & 1);
                m = *const_cast<volatile float*>(&row_reference[r]);
            } else if (my_tiles > 0) {  // the row's first scores give it its first reference
                const int buffer = kSharedRows ? tiles_done & 1 : 0;
                wait(&s_full[kSharedRows ? 0 : s][buffer], (kSharedRows ? tiles_done >> 1 : tiles_done) & 1);
                tc_fence_after();
                float top = -INFINITY;
#pragma unroll 1
                for (int q = 0; q < 2; ++q) {
                    uint32_t v[32];
                    tmem_load32(s_col + buffer * kBufferCols + q * 32, v);
                    tmem_wait_load(v);
                    if (item.tile0 >= item.masked_from) hide(v, last - item.tile0 * kPromptTile - q * 32);
#pragma unroll
                    for (int k = 0; k < 32; k += 2) top = fmaxf(fmaxf(top, __uint_as_float(v[k])), __uint_as_float(v[k + 1]));
                }
                if (top != -INFINITY) m = top * c;
                if (kSharedRows) *const_cast<volatile float*>(&row_reference[r]) = m;
            }
            for (int i = 0; i < my_tiles; ++i) {
                const int tile = item.tile0 + i;
                const bool masked = tile >= item.masked_from;
                const int lim = last - tile * kPromptTile - first_key;  // columns up to this one are seen
                const uint32_t count = tiles_done + i;
                // Half a tile at a time: its product with the values and the next tile's scores of that half run while the other half is
                // exponentiated.
#pragma unroll 1
                for (int h = 0; h < kHalves; ++h) {
                    const int buffer = kSharedRows ? count & 1 : h;
                    wait(&s_full[kSharedRows ? 0 : s][buffer], (kSharedRows ? count >> 1 : count) & 1);
                    tc_fence_after();
                    const uint32_t col = s_col + buffer * kBufferCols;
                    // One pass over the row's 64 scores gives their maximum and, with the reference as it is, the weights and their sum.
                    // Only when the maximum turns out to be more than 8 above the reference is the pass made again, with a reference
                    // that has been moved there; the scores are still in tensor memory, the weights go over them at the end.
                    uint32_t w[2][16];
                    float2x sum[2];
                    for (bool settled = false;;) {
                        // No key of the row so far: the reference is -inf, every score is -inf, and so must every weight's logarithm be.
                        const float reference = m == -INFINITY ? 0.f : m;
                        const float2x minus2 = pack_f2(kPromptWeightShift<T> - reference, kPromptWeightShift<T> - reference);
                        float t4[2] = {-INFINITY, -INFINITY};
                        sum[0] = sum[1] = pack_f2(0.f, 0.f);
                        uint32_t v2[2][32];
                        tmem_load32(col, v2[0]);
                        tmem_load32(col + 32, v2[1]);
                        tmem_wait_load(v2[0]);
                        tmem_loaded(v2[1]);
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            uint32_t(&v)[32] = v2[q];
                            if (masked) hide(v, lim - h * 64 - q * 32);
#pragma unroll
                            for (int k = 0; k < 8; ++k) {
                                float2x t0 = pack_f2(__uint_as_float(v[4 * k]), __uint_as_float(v[4 * k + 1]));
                                float2x t1 = pack_f2(__uint_as_float(v[4 * k + 2]), __uint_as_float(v[4 * k + 3]));
                                float x[4];
                                unpack_f2(t0, x[0], x[1]);
                                unpack_f2(t1, x[2], x[3]);
                                t4[0] = fmaxf(fmaxf(t4[0], x[0]), x[1]);
                                t4[1] = fmaxf(fmaxf(t4[1], x[2]), x[3]);
                                t0 = fma_f2(t0, c2, minus2);
                                t1 = fma_f2(t1, c2, minus2);
                                unpack_f2(t0, x[0], x[1]);
                                unpack_f2(t1, x[2], x[3]);
                                x[0] = ex2(x[0]);
                                x[1] = ex2(x[1]);
                                x[2] = ex2(x[2]);
                                x[3] = ex2(x[3]);
                                sum[0] = add_f2(pack_f2(x[0], x[1]), sum[0]);
                                sum[1] = add_f2(pack_f2(x[2], x[3]), sum[1]);
                                w[q][2 * k] = pack2<T>(x[0], x[1]);
                                w[q][2 * k + 1] = pack2<T>(x[2], x[3]);
                            }
                        }
                        float top = fmaxf(t4[0], t4[1]);
                        top = top == -INFINITY ? top : top * c;
                        if (settled) break;
                        float known = m;
                        if constexpr (kSharedRows) {  // the weights before these have been announced: the reference is what they left
                            if (s == 1) wait(&p_full[0][count & 1], (count >> 1) & 1);
                            else if (i > 0) wait(&p_full[1][(count - 1) & 1], ((count - 1) >> 1) & 1);
                            m = *const_cast<volatile float*>(&row_reference[r]);
                        }
                        const bool move = top > m + 8.f;
                        if (!__any_sync(0xFFFFFFFFu, move || (kSharedRows && m != known))) break;
                        settled = kSharedRows;  // (a row of a stream of its own is found settled by its maximum)
                        if (!kSharedRows || __any_sync(0xFFFFFFFFu, move)) {
                            const float alpha = move ? ex2(m - top) : 1.f;
                            if (i + h + (kSharedRows ? s : 0) > 0) {  // the products so far are complete before they are rescaled
                                // (The phase before that one is complete: the scores came behind the products whose weights they replaced.)
                                if constexpr (kSharedRows) {
                                    const uint32_t last = s == 1 ? count : count - 1;  // tile of the other stream's last weights
                                    wait(&o_done[s ^ 1][last & 1], (last >> 1) & 1);
                                } else {
                                    wait(&o_done[s][0], (2 * count + h - 1) & 1);
                                }
                                tc_fence_after();
#pragma unroll 1
                                for (int q = 0; q < (kSharedRows ? DP : S::kCols) / 16; ++q) {
                                    const uint32_t col = kSharedRows ? lane_base + kColO : o_col;
                                    uint32_t o[16];
                                    tmem_load16(col + q * 16, o);
                                    tmem_wait_load(o);
#pragma unroll
                                    for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * alpha);
                                    tmem_store16(col + q * 16, o);
                                }
                            }
                            if (move) m = top;
                            if (kSharedRows && move) *const_cast<volatile float*>(&row_reference[r]) = m;
                        }
                        if (m != known) l *= ex2(known - m);
                    }
#pragma unroll
                    for (int q = 0; q < 2; ++q) tmem_store16(col + q * 16, w[q]);
                    float part_sum[2];
                    unpack_f2(add_f2(sum[0], sum[1]), part_sum[0], part_sum[1]);
                    l += part_sum[0] + part_sum[1];
                    tmem_wait_store();
                    tc_fence_before();
                    mbarrier_arrive(&p_full[s][buffer]);
                }
            }
            tiles_done += my_tiles;

            // the item's rows
            if (my_tiles > 0) {
                wait(&o_full[kSharedRows ? 0 : s], results_done & 1);
                tc_fence_after();
                if constexpr (kSharedRows) {
                    const float known = m;
                    m = *const_cast<volatile float*>(&row_reference[r]);
                    if (m != known) l *= ex2(known - m);
                    volatile float* const sum_of_row = &row_sum[r];  // the second stream's first, then both's
                    if (s == 0) {
                        wait(&sums_full[1], results_done & 1);
                        l += *sum_of_row;
                    }
                    *sum_of_row = l;
                    mbarrier_arrive(&sums_full[s]);
                    if (s == 1) {
                        wait(&sums_full[0], results_done & 1);
                        l = *sum_of_row;
                    }
                }
                ++results_done;
                if (*reinterpret_cast<volatile int*>(&items[n % kPromptItems].bad_values) != 0) {
                    // Infinities and NaN among the keys that not all rows see were left out of the product: the rows that see them get them now.
                    const int from = max(item.last_key + 1, item.tile0 * kPromptTile);
                    const int to = there ? min(last + 1, item.tile1 * kPromptTile) : from;
                    const unsigned char* values = a.v + (long long)item.k_row * a.v_token_stride + (long long)item.kv_head * a.v_head_stride + (kSharedRows ? s * 256 : 0);
                    const int dims = min(a.dim - (kSharedRows ? s * 128 : 0), S::kCols);
#pragma unroll 1
                    for (int q = 0; q < S::kCols / 16; ++q) {
                        uint32_t o[16];
                        tmem_load16(o_col + q * 16, o);
                        tmem_wait_load(o);
                        for (int key = max(from, 0); key < to; ++key) {
                            const unsigned short* p = reinterpret_cast<const unsigned short*>(values + (long long)key * a.v_token_stride) + q * 16;
#pragma unroll
                            for (int k = 0; k < 16; ++k) {
                                if (q * 16 + k < dims) {
                                    const float x = Codec<T, 16>::to_float16(__ldg(p + k));
                                    if (!(fabsf(x) < INFINITY)) o[k] = __float_as_uint(__uint_as_float(o[k]) + x);
                                }
                            }
                        }
                        tmem_store16(o_col + q * 16, o);
                    }
                    tmem_wait_store();
                }
            }
            if (first_token >= item.tokens) {  // no rows for this stream
                done_with_item(n);
                continue;
            }
            const int my_row = row_index(r);
            const long long first_row = (long long)item.q_row * n_heads + item.kv_head * a.group;
            const bool none = l == 0.f;
            const float inv = none ? 0.f : __frcp_rn(l), total = none ? -INFINITY : m + (log2f(l) - kPromptWeightShift<T>);
            if (my_row >= 0 && (!kSharedRows || s == 0)) {
                if (a.parts > 1) a.part_lse[item.part * n_rows + first_row + my_row] = total;
                else if (a.lse) a.lse[first_row + my_row] = total * 0.69314718055994531f;
            }
            // A thread holds a row, and rows lie apart; 32 bytes at a time are whole sectors all the same.  (Results that went through shared
            // memory, so that eight lanes wrote 128 bytes of a row side by side, took twice as long to leave, 1.6 us.)
            const int dim0 = kSharedRows ? s * 128 : 0, elem = a.parts > 1 ? 4 : 2;
            unsigned char* const to = (a.parts > 1 ? reinterpret_cast<unsigned char*>(a.part_out) + item.part * n_rows * a.dim * 4 : static_cast<unsigned char*>(a.out)) +
                                      (first_row + max(my_row, 0)) * a.dim * elem;
#pragma unroll 1
            for (int q = 0; q < S::kCols; q += 32) {
                uint32_t o[32];
                if (my_tiles > 0) {
                    tmem_load32(o_col + q, o);
                    tmem_wait_load(o);
                } else {
#pragma unroll
                    for (int k = 0; k < 32; ++k) o[k] = 0;
                }
                if (my_row < 0) continue;  // (the loads are the whole warp's)
#pragma unroll
                for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * inv);
                if (a.parts > 1) {
#pragma unroll
                    for (int k = 0; k < 32; k += 8)
                        store_row<8>(to + (dim0 + q + k) * 4, o + k, dim0 + q + k, 8, a);
                } else {
                    uint32_t y[16];
#pragma unroll
                    for (int k = 0; k < 16; ++k) y[k] = pack2<T>(__uint_as_float(o[2 * k]), __uint_as_float(o[2 * k + 1]));
#pragma unroll
                    for (int k = 0; k < 16; k += 8)
                        store_row<8>(to + (dim0 + q + 2 * k) * 2, y + k, dim0 + q + 2 * k, 16, a);
                }
            }
            tc_fence_before();  // the output's columns have been read before the next item's weights are announced
            if (kSharedRows && s == 1 && my_tiles > 0) mbarrier_arrive(&results_read);  // (the first weights are the first stream's)
            done_with_item(n);
        }
    } else {
        // (one instruction for all of a warpgroup's warps, whatever their role)
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(256 - S::kSoftmaxRegs));
    }
    if (warp >= 8 && warp < 12) {
        // ---- warps that look through the values of tiles that not every row sees ----
        const int p = tid - 256;  // the tile's key
        // the first of two slots of a stream's values (shared rows)
        const auto value_slot = [](uint32_t tile, int s) -> uint32_t { return S::kKeySlots + (2 * tile + s) % S::kValuePairs * 2; };
        constexpr uint32_t kExponent = std::is_same<T, __nv_bfloat16>::value ? 0x7F807F80u : 0x7C007C00u;
        uint32_t tiles_before = 0, looked_at = 0;  // (tiles that every row sees go past these warps: a barrier of their own tells them of the others)
        PromptItem item;
        for (int n = 0; next_item(n, item); ++n) {
            for (int tile = max(item.tile0, item.masked_from); tile < item.tile1; ++tile) {
                bool found = false;
                wait_item(&landed[looked_at % kPromptLanded], (looked_at / kPromptLanded) & 1);
                ++looked_at;
                const uint32_t unit = (2 * (tiles_before + tile - item.tile0) + 1) * kUnits;
                if (tile * kPromptTile + p > item.last_key) {
#pragma unroll 1
                    for (int b = 0; b < kBlocks; ++b) {
                        unsigned char* row = ring + (unit + b / kSlotBlocks) % S::kSlots * S::kSlotBytes + b % kSlotBlocks * S::kBlockBytes + p * 128;
                        if (kSharedRows)  // two slots to a stream's values, blocks of 64 of them
                            row = ring + value_slot(tiles_before + tile - item.tile0, p / 64) * S::kSlotBytes + b * (64 * 128) + p % 64 * 128;
#pragma unroll
                        for (int u = 0; u < 8; ++u) {
                            uint4* at = reinterpret_cast<uint4*>(row + ((u ^ (p & 7)) << 4));
                            const uint4 x = *at;
                            const uint4 bad = make_uint4(__vcmpeq2(x.x & kExponent, kExponent), __vcmpeq2(x.y & kExponent, kExponent),
                                                         __vcmpeq2(x.z & kExponent, kExponent), __vcmpeq2(x.w & kExponent, kExponent));
                            if (bad.x | bad.y | bad.z | bad.w) {
                                *at = make_uint4(x.x & ~bad.x, x.y & ~bad.y, x.z & ~bad.z, x.w & ~bad.w);
                                found = true;
                            }
                        }
                    }
                }
                if (found && tile * kPromptTile + p < item.end_key) *reinterpret_cast<volatile int*>(&items[n % kPromptItems].bad_values) = 1;
                fence_async_proxy();
                asm volatile("barrier.cta.sync 1, 128;" ::: "memory");
                if (p < kUnits) mbarrier_arrive(&full[kSharedRows ? value_slot(tiles_before + tile - item.tile0, p / 2) + p % 2 : (unit + p) % S::kSlots]);
            }
            tiles_before += item.tile1 - item.tile0;
            done_with_item(n);
        }
    }
    if constexpr (kSharedRows) {
        // ---- warps that issue the products of both streams: one the scores', one the outputs' ----
        // The scores have two buffers, which the tiles take in turn, so that they are there when the softmax comes to them.  (4096 tokens, 32
        // heads on 4 of 256: one buffer, and one warp for all products, which spent more time issuing than the tensor cores computing: 307 us; two
        // warps: 279; two buffers: 259; both streams' scores in one product of 128 keys: 248.)
        constexpr uint32_t kSlot16 = S::kSlotBytes / 16;
        const int steps = (a.dim + 15) / 16;  // of 16 dims
        uint32_t tiles_before = 0, items_before = 0;
        PromptItem item;
        if (warp == 13) {
            const uint64_t q_at = tc_descriptor(tc_layout(16, 1024), smem_u32(smem) >> 4), k_base = tc_descriptor(tc_layout(16, 1024), smem_u32(ring) >> 4);
            for (int n = 0; next_item(n, item); ++n) {
                const int tiles = item.tile1 - item.tile0;
                if (tiles > 0) {
                    wait(&q_full, items_before & 1);
                    ++items_before;
                }
                for (int i = 0; i < tiles; ++i) {
                    // S = Q K^T, as soon as the weights that lie where the scores go have been used
                    const uint32_t count = tiles_before + i, buffer = count & 1;
                    if (count >= 2) {
                        wait(&o_done[0][buffer], ((count >> 1) - 1) & 1);
                        wait(&o_done[1][buffer], ((count >> 1) - 1) & 1);
                    }
#pragma unroll
                    for (int b = 0; b < kBlocks; ++b) {
                        wait(&full[b], count & 1);
                        tc_fence_after();
                        if (elect_one()) {
                            const uint64_t k_at = k_base + b * kSlot16;
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                if (b * 4 + k < steps) tc_mma_ss(tmem + buffer * kBufferCols, q_at + (b * (S::kBlockBytes / 16) + k * 2), k_at + k * 2, kScoreIdesc, b + k > 0);
                            if (b % 2 == 1) tc_commit(&empty[b - 1]);
                            if (b == kBlocks - 1) {
                                tc_commit(&s_full[0][buffer]);
                                if (i + 1 == tiles) tc_commit(&q_free);
                            }
                        }
                        __syncwarp();
                    }
                }
                tiles_before += tiles;
                done_with_item(n);
            }
        } else if (warp == 12) {
            const uint64_t v_base = tc_descriptor(tc_layout(S::kValueRows * 128, 1024), smem_u32(ring) >> 4);
            const uint32_t out_idesc = tc_instruction<T>(steps * 16, false, true);
            uint32_t pair = 0, lap = 0;
            for (int n = 0; next_item(n, item); ++n) {
                const int tiles = item.tile1 - item.tile0;
                if (tiles > 0) {
                    wait(&results_read, (items_before & 1) ^ 1);  // the second stream's of the item before
                    ++items_before;
                }
                for (int i = 0; i < tiles; ++i) {
                    const uint32_t count = tiles_before + i, buffer = count & 1;
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        // O += W V with the stream's values
                        const uint32_t slot = S::kKeySlots + 2 * pair;
                        wait(&full[slot], lap);
                        wait(&full[slot + 1], lap);
                        wait(&p_full[s][buffer], (count >> 1) & 1);
                        tc_fence_after();
                        if (elect_one()) {
#pragma unroll
                            for (int k = 0; k < kPromptTile / 32; ++k)
                                tc_mma_ts(tmem + kColO, tmem + buffer * kBufferCols + s * 64 + k * 8, v_base + (slot * kSlot16 + k * 128), out_idesc, i + s + k > 0);
                            tc_commit(&o_done[s][buffer]);
                            tc_commit(&empty[slot]);
                            if (s == 1 && i + 1 == tiles) tc_commit(&o_full[0]);
                        }
                        __syncwarp();
                        if (++pair == S::kValuePairs) {
                            pair = 0;
                            lap ^= 1;
                        }
                    }
                }
                tiles_before += tiles;
                done_with_item(n);
            }
        }
        // the tensor memory is given back only when nothing writes it any more
        if (warp == 12 || warp == 13) {
            if (elect_one()) tc_commit(&drained[warp - 12]);
            __syncwarp();
            ok = mbarrier_wait_sleeping(&drained[warp - 12], 0) && ok;
        }
    } else if (warp >= 12 && warp < 14) {
        // ---- warps that issue the products of the two streams ----
        const int s = warp - 12;
        constexpr uint64_t kRowsLayout = tc_layout(16, 1024), kColsLayout = tc_layout(S::kBlockBytes, 1024);
        constexpr uint32_t kSlot16 = S::kSlotBytes / 16, kBlock16 = S::kBlockBytes / 16;
        const uint32_t q16 = smem_u32(smem) >> 4, ring16 = smem_u32(ring) >> 4;
        const uint64_t q_at = tc_descriptor(kRowsLayout, q16 + s * (S::kQueryBytes / 16));
        const uint64_t k_base = tc_descriptor(kRowsLayout, ring16), v_base = tc_descriptor(kColsLayout, ring16);
        const uint32_t d_scores = tmem + s * kPromptTile, d_out = tmem + kColO + s * S::kCols;
        const int steps = (a.dim + 15) / 16;  // of 16 dims
        const uint32_t out_idesc = tc_instruction<T>(steps * 16, false, true);
        uint32_t tiles_before = 0, my_tiles_before = 0, items_before = 0;
        auto wait_unit = [&](uint32_t unit) {
            wait(&full[unit % S::kSlots], (unit / S::kSlots) & 1);
            tc_fence_after();
        };
        auto skip_unit = [&](uint32_t unit) {  // a tile that this stream does not need
            wait(&full[unit % S::kSlots], (unit / S::kSlots) & 1);
            if (lane == 0) mbarrier_arrive(&empty[unit % S::kSlots]);
            __syncwarp();
        };
        PromptItem item;
        for (int n = 0; next_item(n, item); ++n) {
            const int tiles = item.tile1 - item.tile0, mine = max(stream_tiles(item, s), 0);
            if (tiles > 0) {
                wait(&q_full, items_before & 1);
                tc_fence_after();
            }
            // Half h of S = Q K^T with the item's tile number i; its blocks are waited for, and freed, one after the other
            auto scores = [&](int i, int h) {
                const uint32_t unit = 2 * (tiles_before + i) * kUnits;
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) {
                    const uint32_t slot = (unit + b / kSlotBlocks) % S::kSlots;
                    if (h == 0 && b % kSlotBlocks == 0) wait_unit(unit + b / kSlotBlocks);
                    if (elect_one()) {
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            if (b * 4 + k < steps)
                                tc_mma_ss(d_scores + h * 64, q_at + (b * kBlock16 + k * 2), k_base + (slot * kSlot16 + b % kSlotBlocks * kBlock16 + k * 2 + h * (64 * 128 / 16)),
                                          kScoreIdesc, b + k > 0);
                        if (h == 1 && (b + 1) % kSlotBlocks == 0) tc_commit(&empty[slot]);
                        if (b == kBlocks - 1) {
                            tc_commit(&s_full[s][h]);
                            if (h == 1 && i + 1 == mine) tc_commit(&q_free);
                        }
                    }
                    __syncwarp();
                }
            };
            if (mine > 0) {
                scores(0, 0);
                scores(0, 1);
            } else if (tiles > 0 && lane == 0) mbarrier_arrive(&q_free);
            for (int i = 0; i < tiles; ++i) {
                const uint32_t unit = (2 * (tiles_before + i) + 1) * kUnits;  // the values'
                if (i >= mine) {
#pragma unroll 1
                    for (int b = 0; b < 2 * kUnits; ++b) skip_unit(unit - kUnits + b);
                    continue;
                }
                // O += W V
                const uint32_t slot = unit % S::kSlots;
#pragma unroll
                for (int u = 0; u < kUnits; ++u) wait_unit(unit + u);
                const uint64_t v_at = v_base + slot * kSlot16;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    wait(&p_full[s][h], (my_tiles_before + i) & 1);
                    tc_fence_after();
                    if (elect_one()) {
#pragma unroll
                        for (int k = 0; k < kPromptTile / 32; ++k)
                            tc_mma_ts(d_out, d_scores + h * 64 + k * 8, v_at + (h * 64 * 128 / 16 + k * 128), out_idesc, i + h + k > 0);
                        tc_commit(&o_done[s][0]);
                        if (h == 1) {
#pragma unroll
                            for (int u = 0; u < kUnits; ++u) tc_commit(&empty[slot + u]);
                            if (i + 1 == mine) tc_commit(&o_full[s]);
                        }
                    }
                    __syncwarp();
                    if (i + 1 < mine) scores(i + 1, h);
                }
            }
            tiles_before += tiles;
            my_tiles_before += mine;
            if (tiles > 0) ++items_before;
            done_with_item(n);
        }
        // the tensor memory is given back only when nothing writes it any more
        if (elect_one()) tc_commit(&drained[s]);
        __syncwarp();
        ok = mbarrier_wait_sleeping(&drained[s], 0) && ok;
    }
    if (warp == 14) {
        // ---- the warp that fetches ----
        uint32_t units = 0, items_before = 0, looks = 0;
        bool posted = false;
        const uint32_t query_bytes = (uint32_t)(a.stream_tokens * a.group) * 128u * kBlocks;
        // A tile of keys or values from row `row` on; `bar`, where there is one, is told of all its bytes, otherwise each slot of its own.
        auto fetch = [&](const CUtensorMap* map, int head, int row, uint64_t* bar) {
#pragma unroll
            for (int u = 0; u < kUnits; ++u) {
                const uint32_t slot = units % S::kSlots;
                wait(&empty[slot], ((units / S::kSlots) & 1) ^ 1);
                if (!a.drop_copies && elect_one()) {
                    if (!bar) mbarrier_expect_tx(&full[slot], S::kSlotBytes);
                    else if (u == 0) mbarrier_expect_tx(bar, S::kSlotBytes * kUnits);
#pragma unroll
                    for (int b = 0; b < kSlotBlocks; ++b)
                        tma_load_3d(ring + slot * S::kSlotBytes + b * S::kBlockBytes, map, (u * kSlotBlocks + b) * 64, head, row, bar ? bar : &full[slot]);
                }
                __syncwarp();
                ++units;
            }
        };
        // The same with shared rows: the tile's keys, two slots freed at a time, and a stream's values.
        uint32_t key_tiles = 0, value_pairs = 0;
        auto fetch_keys = [&](int head, int row) {
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) {
                if (b % 2 == 0) wait(&empty[b], (key_tiles & 1) ^ 1);
                if (!a.drop_copies && elect_one()) {
                    mbarrier_expect_tx(&full[b], S::kSlotBytes);
                    tma_load_3d(ring + b * S::kSlotBytes, &k_map, b * 64, head, row, &full[b]);
                }
                __syncwarp();
            }
            ++key_tiles;
        };
        auto fetch_values = [&](int s, int head, int row, uint64_t* bar) {
            const uint32_t slot = S::kKeySlots + value_pairs % S::kValuePairs * 2;
            wait(&empty[slot], ((value_pairs / S::kValuePairs) & 1) ^ 1);
            if (!a.drop_copies && elect_one()) {
                if (bar && s == 0) mbarrier_expect_tx(bar, S::kSlotBytes * 4);
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    if (!bar) mbarrier_expect_tx(&full[slot + u], S::kSlotBytes);
#pragma unroll
                    for (int b = 0; b < 2; ++b)
                        tma_load_3d(ring + (slot + u) * S::kSlotBytes + b * (64 * 128), &v_map, (u * 2 + b) * 64, head, row + s * 64, bar ? bar : &full[slot + u]);
                }
            }
            __syncwarp();
            ++value_pairs;
        };
        PromptItem item;
        for (int n = 0; next_item(n, item); ++n) {
            const int tiles = item.tile1 - item.tile0;
            if (tiles > 0) {
                wait(&q_free, (items_before & 1) ^ 1);
                if (!a.drop_copies && elect_one()) {
                    mbarrier_expect_tx(&q_full, query_bytes * S::kQueries);
#pragma unroll
                    for (int s = 0; s < S::kQueries; ++s)
#pragma unroll
                        for (int b = 0; b < kBlocks; ++b)
                            tma_load_3d(smem + s * S::kQueryBytes + b * S::kBlockBytes, &q_map, b * 64, item.kv_head * a.group, item.q_row + (S::kSharedRows ? 0 : s ^ item.turned) * a.stream_tokens, &q_full);
                }
                __syncwarp();
                posted = !a.drop_copies;
                ++items_before;
            }
            uint64_t* late = nullptr;  // barrier of the last tile's values
            for (int i = 0; i < tiles; ++i) {
                const int row = item.k_row + (item.tile0 + i) * kPromptTile;
                const bool masked = item.tile0 + i >= item.masked_from;  // then those who look through the values tell the others
                uint64_t* const bar = masked ? &landed[looks % kPromptLanded] : nullptr;
                if (masked) ++looks;
                if constexpr (kSharedRows) {  // in the order in which slots become free
                    fetch_keys(item.kv_head, row);
                    if (i > 0) fetch_values(1, item.kv_head, row - kPromptTile, late);
                    fetch_values(0, item.kv_head, row, bar);
                    late = bar;
                    if (i + 1 == tiles) fetch_values(1, item.kv_head, row, bar);
                } else {
                    fetch(&k_map, item.kv_head, row, nullptr);
                    fetch(&v_map, item.kv_head, row, bar);
                }
            }
            done_with_item(n);
        }
        // no copy is under way when the CTA ends
        if (posted) {
            for (uint32_t m = looks > kPromptLanded ? looks - kPromptLanded : 0; m < looks; ++m)
                ok = mbarrier_wait_sleeping(&landed[m % kPromptLanded], (m / kPromptLanded) & 1) && ok;
            ok = mbarrier_wait_sleeping(&q_full, (items_before - 1) & 1) && ok;
            for (uint32_t u = units > S::kSlots ? units - S::kSlots : 0; u < units; ++u) ok = mbarrier_wait_sleeping(&full[u % S::kSlots], (u / S::kSlots) & 1) && ok;
            if constexpr (kSharedRows) {
                for (int b = 0; b < kBlocks; ++b) ok = mbarrier_wait_sleeping(&full[b], (key_tiles - 1) & 1) && ok;
                for (uint32_t u = value_pairs > S::kValuePairs ? value_pairs - S::kValuePairs : 0; u < value_pairs; ++u)
                    for (int k = 0; k < 2; ++k) ok = mbarrier_wait_sleeping(&full[S::kKeySlots + u % S::kValuePairs * 2 + k], (u / S::kValuePairs) & 1) && ok;
            }
        }
    } else if (warp == 15) {
        // ---- the warp that works out the items ----
        PromptOrder order(a);
        const int per_block = a.kv_heads * a.parts;
        const long long ids = order.total * per_block;
        for (int n = 0;; ++n) {
            // there and back again, so that the CTA that had the dearest item of one round has the cheapest of the next (the same: 49.6 us without)
            const long long id = (long long)n * gridDim.x + ((n & 1) ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
            PromptItem item;
            item.valid = 0;
            if (id < ids) {
                const long long rank = ids <= 0xFFFFFFFFLL ? (long long)((unsigned)id / (unsigned)per_block) : id / per_block;
                const int rest = (int)(id - rank * per_block);
                int seq, block;
                if (a.n_seqs == 1) {
                    seq = 0;
                    block = (int)(order.total - 1 - rank);  // the last block of a causal sequence is the dearest
                } else if (a.n_seqs > PromptOrder::kKept * 32) {
                    order.find_among_many(rank, seq, block);
                } else if (ids <= gridDim.x) {
                    order.find_any(rank, seq, block);
                } else {
                    order.find(rank, seq, block);
                }
                const PromptSequence q = prompt_sequence(a, max(seq, 0));
                item.valid = 1;
                item.tokens = min(a.block_tokens, q.q_len - block * a.block_tokens);
                item.q_row = q.q_row + block * a.block_tokens;
                // Blocks that one stream can take go to the streams in turn: one's results leave while the other's next block is under way.  (300
                // sequences of 16 tokens, 32 heads on 8 of 128: 66 us, 78 with all of them to the first.)
                item.turned = item.tokens <= a.stream_tokens && (n & 1);
                item.k_row = q.k_row;
                item.end_key = q.k_len;
                item.key_step = a.causal ? 1 : 0;
                item.last_key = a.causal ? min(q.k_len - q.q_len + block * a.block_tokens, q.k_len - 1) : q.k_len - 1;
                const int last_key = min(item.last_key + item.key_step * (item.tokens - 1), q.k_len - 1);
                const int tiles = last_key < 0 ? 0 : last_key / kPromptTile + 1;
                item.masked_from = max(item.last_key + 1, 0) / kPromptTile;
                item.kv_head = rest / a.parts;
                item.part = rest - item.kv_head * a.parts;
                const int run = (tiles + a.parts - 1) / a.parts;
                item.tile0 = min(item.part * run, tiles);
                item.tile1 = min(item.tile0 + run, tiles);
                item.bad_values = 0;
            }
            wait_item(&item_free[n % kPromptItems], ((n / kPromptItems) & 1) ^ 1);
            if (!__all_sync(0xFFFFFFFFu, ok)) break;
            if (lane == 0) {
                items[n % kPromptItems] = item;
                mbarrier_arrive(&item_full[n % kPromptItems]);
            }
            __syncwarp();
            if (n == 0 && blockIdx.x == 0 && lane == 0) {
                if (!order.sound) atomicExch(a.status, kDeviceIndexCode);
                if (a.parts > 1) *a.part_ready = order.sound;
            }
            if (!item.valid) break;
        }
    }
    if (!ok) atomicExch(a.status, kDeviceTimeoutCode);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 12) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

// Joins the parts of every row: weights 2^(lse_p - max) / sum.  One warp per row; a lane looks after the weight of one part, the
// parts' outputs are fetched independently of one another.  A part that saw keys never weighs nothing, or a NaN among its values would be lost with it.
constexpr int kPromptMergeThreads = 128;
template <typename T>
__global__ void __launch_bounds__(kPromptMergeThreads) prompt_merge_kernel(const __grid_constant__ PromptArgs a)
{
    const int lane = threadIdx.x & 31, n_heads = a.kv_heads * a.group;
    const long long row = (long long)blockIdx.x * (kPromptMergeThreads / 32) + (threadIdx.x >> 5), n_rows = (long long)a.q_tokens * n_heads;
    wait_for_previous_kernel();
    const int token = (int)(row / n_heads);
    if (row >= n_rows || token < __ldg(a.q_starts) || token >= __ldg(a.q_starts + a.n_seqs) || *a.part_ready == 0) return;  // a row of no sequence
    const float lse = lane < a.parts ? a.part_lse[lane * n_rows + row] : -INFINITY;
    float top = lse;
#pragma unroll
    for (int s = 16; s >= 1; s >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, s));
    const float base = top == -INFINITY ? 0.f : top;
    float w = lse == -INFINITY ? 0.f : ex2(lse - base);
    if (w == 0.f && lse != -INFINITY) w = __uint_as_float(1u);
    float total = w;
#pragma unroll
    for (int s = 16; s >= 1; s >>= 1) total += __shfl_xor_sync(0xFFFFFFFFu, total, s);
    const float inv = total == 0.f ? 0.f : 1.0f / total;
    for (int d0 = 0; d0 < a.dim; d0 += 128) {
        const int d = d0 + lane * 4;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int p = 0; p < a.parts; ++p) {
            const float wp = __shfl_sync(0xFFFFFFFFu, w, p);
            if (wp == 0.f || d >= a.dim) continue;
            const float4 x = *reinterpret_cast<const float4*>(a.part_out + (p * n_rows + row) * a.dim + d);
            o.x = fmaf(wp, x.x, o.x); o.y = fmaf(wp, x.y, o.y);
            o.z = fmaf(wp, x.z, o.z); o.w = fmaf(wp, x.w, o.w);
        }
        if (d < a.dim)
            *reinterpret_cast<uint2*>(reinterpret_cast<unsigned char*>(a.out) + (row * a.dim + d) * 2) =
                make_uint2(pack2<T>(o.x * inv, o.y * inv), pack2<T>(o.z * inv, o.w * inv));
    }
    if (lane == 0 && a.lse) a.lse[row] = total == 0.f ? -INFINITY : (top + log2f(total)) * 0.69314718055994531f;
}

}  // namespace rt
