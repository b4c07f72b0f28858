// Attention of many rows to a shared prefix on the fifth-generation tensor cores (sm_100a, tcgen05 + tensor memory).
//
// All rows of one key/value head (every sequence's query tokens and the head's query heads) see the same keys, so the
// prefix is a plain matrix problem:  S = Q K^T,  W = 2^(score_scale S - m),  O = W V,  in one pass over the keys with a
// running reference m and sum per row.  A CTA takes one key/value head, one block of up to 256 of its rows and one run of
// key tiles of 128 (see attend_split.h), one CTA to an SM.  What it finds out is one part of its rows (two in the narrow form
// below), joined by merge_parts_kernel.
//
// Inside a CTA (16 warps):
//   warps 0-3, 4-7   two softmax streams of 128 rows, one row to a thread (tensor memory lane = row): they read S from
//                    tensor memory, keep m and the sum in registers, and write the weights back over S as the 16-bit
//                    left operand of the second product;
//   warps 8-11       fetch the paged tiles: keys and values with cp.async, 16 bytes a piece, into the 128-byte-swizzled
//                    layout that the matrix unit reads (pages may have any size, so one copy per row is the widest that
//                    always works); quantised tiles are fetched into registers, turned into fp16 and stored;
//   warps 12, 13     issue the matrix products, each for its stream (half a tile of 64 keys at a time, so that one half's
//                    products run while the other is exponentiated);
//   warps 14, 15     look up the pages and scales of the tiles to come.
// The two streams take turns on the tensor cores: while one's scores are exponentiated the other's products run.  Blocks of
// more than 128 rows (wide form): a stream is one half of the rows, both use the same tiles.  Blocks of up to 128 rows
// (narrow form): both streams use the same rows and alternate the tiles, and leave a part each.
//
// The reference m is moved only when the row's maximum exceeds it by more than 8 (a factor of 256): then the sum and the
// output row in tensor memory are rescaled by the row's own thread.  Weights are thus at most 256, which bf16 and fp16 hold
// with their full relative precision, and the quotient is the same.
//
// Quantised caches: both products run in fp16 on codes, with the scales in the exponent (see attend_keys_kernel.cuh).
//
// Bounds: 4 * 128 * 128 * dim flops and 128 * 128 exponentials per tile and stream; at dim 128 the tensor cores need 1024
// cycles for that and the SM's 16 exponentials a cycle 1024 as well.
//
// Measured: 1024 rows x 8 key/value heads of 128, prefix 32768, bf16: 177 us with the rest of the call for 137 GFLOP, 0.78 PFLOP/s
// or 0.48 of the measured matrix rate (steps: both streams' whole tiles in turn 217, CTAs that share tiles numbered
// together 201, the warp's number by shuffle 194, constant slots 188, an issuing warp per stream 177).  e4m3 codes: 241 us, the
// scales' products and sums in the softmax warps.  256 rows: 71 us, heads of 64: 162 us (half the flops for the same
// exponentials).
#pragma once

#include "attend_common.cuh"
#include "attend_split.h"
#include "tensor_core.cuh"

namespace rt {

constexpr int kTcThreads = 512;
constexpr int kTcSlots = 4;   // ring of key and value tiles
constexpr int kTcAux = 8;     // tiles whose places and constants are kept: the two under way and two ahead

template <int FMT, int DP>
struct PrefixShape {
    static constexpr bool kQuant = FMT != kKvPlain;
    // Of eight pairs of every 32 exponentials, so many go to the multiply-add pipe (see ex2_by_polynomial): the SM's special
    // function unit alone needs 2048 cycles for the two streams' tiles, as long as the tensor cores.  Measured against none: 64
    // sequences, prefix 8192, int8: 77 us, not 79.5; heads of 64: 164, not 167; 256 sequences, prefix 32768: no difference.
    static constexpr int kPolynomial = 4;
    // Registers per softmax thread; half the threads are softmax threads, and the other half gets the rest of 2 * 128.
    static constexpr int kSoftmaxRegs = 136;
    static constexpr int kTileBytes = kTcTile * DP * 2;
    static constexpr int kAuxFloats = kQuant ? 3 * kTcTile : kTcTile;
    static constexpr size_t kAuxAt = (size_t)(2 + kTcSlots) * kTileBytes;
    static constexpr size_t kOffsetsAt = kAuxAt + (size_t)kTcAux * kAuxFloats * 4;
    // Where results wait to be written row by row, 4 KB per softmax warp: heads of 64 have room for it, heads of 128 use the
    // query tiles, which are free by then.
    static constexpr size_t kStageAt = kOffsetsAt + (size_t)kTcAux * kTcTile * 8;
    static constexpr size_t kSmem = kStageAt + (DP == 64 ? 8 * 4096 : 0) + 1024;  // 1024: alignment of the tiles
};

template <typename T, int FMT, int DP>
__global__ void __launch_bounds__(kTcThreads, 1) attend_prefix_kernel(const AttendArgs a, const PrefixSplit split)
{
    using S = PrefixShape<FMT, DP>;
    constexpr bool kQuant = S::kQuant;
    using M = typename std::conditional<kQuant, __half, T>::type;
    constexpr int kBlockBytes = kTileBlockBytes;  // one 64-dim column block of a tile
    constexpr uint32_t kScoreIdesc = tc_instruction<M>(kTcTile / 2, false, false), kOutIdesc = tc_instruction<M>(DP, false, true);
    constexpr uint32_t kColO = 2 * kTcTile;

    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    unsigned char* q_tiles = smem;
    unsigned char* ring = smem + 2 * S::kTileBytes;
    float* aux = reinterpret_cast<float*>(smem + S::kAuxAt);
    long long* offsets = reinterpret_cast<long long*>(smem + S::kOffsetsAt);
    __shared__ __align__(8) uint64_t full[kTcSlots], empty[kTcSlots], aux_full[kTcAux], aux_free[kTcAux], s_full[2][2], p_full[2][2], o_done[2], o_full[2], q_full, drained[2];
    __shared__ uint32_t tmem_base;
    __shared__ float row_factor[2][kQuant ? 128 : 1];
    __shared__ uint32_t ragged[kTcAux];  // one byte for each half of the lookup: some key is not there
    __shared__ int nan_values[2];        // of a quantised cache: among a stream's tiles is a value whose scale is not finite

    // (the warp's number by shuffle: the compiler then knows that a role is taken by whole warps)
    const int tid = threadIdx.x, warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0), lane = tid & 31;
    if (tid == 0) {
        for (int i = 0; i < kTcSlots; ++i) {
            mbarrier_init(&full[i], 128);
            mbarrier_init(&empty[i], 2);
        }
        for (int i = 0; i < kTcAux; ++i) {
            mbarrier_init(&aux_full[i], 64);
            mbarrier_init(&aux_free[i], 2);
            ragged[i] = 0;
        }
        for (int i = 0; i < 2; ++i) {
            for (int h = 0; h < 2; ++h) {
                mbarrier_init(&s_full[i][h], 1);
                mbarrier_init(&p_full[i][h], 128);
            }
            mbarrier_init(&o_done[i], 1);
            mbarrier_init(&o_full[i], 1);
            mbarrier_init(&drained[i], 1);
            nan_values[i] = 0;
        }
        mbarrier_init(&q_full, 256);
    }
    for (int i = tid; i < kTcAux * kTcTile; i += kTcThreads) offsets[i] = -1;  // what is read here was published, now or for an earlier tile, or is no place
    if (warp == 12) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&tmem_base)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_base;
    wait_for_previous_kernel();
    if (a.before_suffix) let_next_kernel_start();

    // this CTA's key/value head, row block and tiles
    const int block = (int)(blockIdx.x % (unsigned)split.blocks), run_no = (int)(blockIdx.x / (unsigned)split.blocks % (unsigned)split.runs);
    const int kv_head = (int)(blockIdx.x / (unsigned)(split.blocks * split.runs));
    const int tile0 = run_no * split.run, n = min(split.tiles - tile0, split.run);
    const bool narrow = narrow_block(split, block);
    // Every wait is bounded.  A thread whose wait has run out stops waiting and goes on through the same loops, so that every
    // barrier is still met and the tensor memory is given back; the status word says that the results are not valid.  Nothing that
    // it goes on with leads outside the tensors: places are those of some tile's keys, or none, from the beginning.
    bool ok = true;
    auto wait = [&](uint64_t* bar, uint32_t parity) {
        if (ok) ok = mbarrier_wait_sleeping(bar, parity, a.wait_polls);
    };

    if (warp < 8) {
        // ---- softmax streams ----
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(S::kSoftmaxRegs));
        const int s = warp >> 2, r = (warp & 3) * 32 + lane;
        const uint32_t lane_base = tmem + ((uint32_t)(warp & 3) << 21);
        const uint32_t s_col = lane_base + s * kTcTile, o_col = lane_base + kColO + s * DP;
        const bool flip = a.score_scale < 0.f;
        const float scale = fabsf(a.score_scale);
        const int n_heads = a.kv_heads * a.group;
        const long long n_rows = (long long)a.n_seqs * a.q_len * n_heads;
        const int first_row = block * kTcBlockRows + (narrow ? 0 : s * 128);
        // [token][head] index of row i of this stream's 128, -1: no such row
        const auto row_index = [&](int i) -> long long {
            const int row = first_row + i;
            if (row >= split.rows) return -1;
            const int token = row / a.group;
            return (long long)token * n_heads + kv_head * a.group + (row - token * a.group);
        };
        // Query rows into shared memory, DP / 8 lanes to a row, so that a row is read in one piece.  Narrow form: the first
        // stream's threads do it for both.
        if (!narrow || s == 0) {
            constexpr int LANES = DP / 8, ROWS = 32 / LANES, N = 32 / ROWS;  // lanes per row, rows at once, turns
            const int u = lane % LANES;
            unsigned char* tile = q_tiles + s * S::kTileBytes + (u >> 3) * kBlockBytes;
            {
                uint4 w[N];  // all at once: behind the first tiles' copies every further round trip would take its turn
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int row = first_row + (warp & 3) * 32 + i * ROWS + lane / LANES;
                    const bool there = row < split.rows && u * 8 < a.dim;
                    const int token = there ? row / a.group : 0;
                    const long long o = (long long)token * a.q_token_stride +
                                        (long long)(kv_head * a.group + (there ? row - token * a.group : 0)) * a.q_head_stride + (there ? u * 8 : 0);
                    w[i] = __ldg(reinterpret_cast<const uint4*>(a.q + o * 2));
                    if (!there) w[i] = make_uint4(0, 0, 0, 0);
                }
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int mine = (warp & 3) * 32 + i * ROWS + lane / LANES;
                    const uint32_t sign = flip ? 0x80008000u : 0u;
                    w[i].x ^= sign; w[i].y ^= sign; w[i].z ^= sign; w[i].w ^= sign;
                    if constexpr (kQuant) {
                        uint32_t top = __vmaxu2(__vmaxu2(w[i].x & 0x7FFF7FFFu, w[i].y & 0x7FFF7FFFu), __vmaxu2(w[i].z & 0x7FFF7FFFu, w[i].w & 0x7FFF7FFFu));
#pragma unroll
                        for (int m = LANES / 2; m >= 1; m >>= 1) top = __vmaxu2(top, __shfl_xor_sync(0xFFFFFFFFu, top, m));
                        const float factor = fp16_row_factor(Codec<T, 16>::to_float16(max(top & 0xFFFFu, top >> 16)));
                        if (u == 0) row_factor[s][mine] = factor;
                        uint32_t* p = &w[i].x;
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            p[k] = pack2<__half>(Codec<T, 16>::to_float16(p[k] & 0xFFFFu) * factor, Codec<T, 16>::to_float16(p[k] >> 16) * factor);
                    }
                    *reinterpret_cast<uint4*>(tile + mine * 128 + (((u & 7) ^ (mine & 7)) << 4)) = w[i];
                }
            }
        }
        fence_async_proxy();
        mbarrier_arrive(&q_full);
        float row_c = scale;
        if constexpr (kQuant) {
            asm volatile("barrier.cta.sync 1, 256;" ::: "memory");
            row_c *= __frcp_rn(row_factor[narrow ? 0 : s][r]);
        }

        float m = -INFINITY, l = 0.f;
        const int my_tiles = narrow ? (n + 1 - s) / 2 : n;
        for (int i = 0; i < my_tiles; ++i) {
            const int t = narrow ? 2 * i + s : i, aux_i = t % kTcAux;
            wait(&aux_full[aux_i], (t / kTcAux) & 1);
            const float4* ka = reinterpret_cast<const float4*>(aux + aux_i * S::kAuxFloats);
            // Half a tile at a time: while this half is exponentiated, the products of the other one run.
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {
                wait(&s_full[s][h], i & 1);
                tc_fence_after();
                const uint32_t col = s_col + h * 64;
                // One pass over the row's 64 scores, 32 at a time, gives their maximum and, with the reference as it is, the weights
                // and their sum.  Only when the maximum turns out to be more than 8 above the reference is the pass made again, with
                // a reference that has been moved there; the scores are still in tensor memory, the weights go over them at the end.
                // (The row's first scores have no reference yet and always take two passes.)
                uint32_t w[2][16];
                float2x sum[2];
                for (;;) {
                    // No key of the row so far: the reference is -inf, every score is -inf, and so must every weight's logarithm be.
                    const float base = m == -INFINITY ? 0.f : m;
                    // A score scale of zero would make NaN of a plain cache's hidden scores: the smallest normal number does instead.
                    const float c = kQuant ? row_c : fmaxf(row_c, 1.17549435e-38f);
                    const float2x c2 = pack_f2(c, c), minus2 = pack_f2(-base, -base);
                    float t4[2] = {-INFINITY, -INFINITY};
                    sum[0] = sum[1] = pack_f2(0.f, 0.f);
                    uint32_t v2[2][32];
                    tmem_load32(col, v2[0]);
                    tmem_load32(col + 32, v2[1]);
                    tmem_wait_load(v2[0]);
                    tmem_loaded(v2[1]);
                    const bool holes = !kQuant && *reinterpret_cast<volatile uint32_t*>(&ragged[aux_i]) != 0;  // the last tile, or pages that are not there
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        uint32_t(&v)[32] = v2[q];
                        const int at4 = h * 16 + q * 8;  // constants, four keys at a time
                        if (holes) {
#pragma unroll
                            for (int k = 0; k < 8; ++k) {
                                const float4 b = ka[at4 + k];
                                if (b.x != 0.f) v[4 * k] = 0xFF800000u;
                                if (b.y != 0.f) v[4 * k + 1] = 0xFF800000u;
                                if (b.z != 0.f) v[4 * k + 2] = 0xFF800000u;
                                if (b.w != 0.f) v[4 * k + 3] = 0xFF800000u;
                            }
                        }
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            float2x t0 = pack_f2(__uint_as_float(v[4 * k]), __uint_as_float(v[4 * k + 1]));
                            float2x t1 = pack_f2(__uint_as_float(v[4 * k + 2]), __uint_as_float(v[4 * k + 3]));
                            if constexpr (kQuant) {
                                const ulonglong2* k2 = reinterpret_cast<const ulonglong2*>(ka) + at4 + k;
                                const ulonglong2 ks = k2[0], lv = k2[32];
                                t0 = fma_f2(mul_f2(t0, c2), ks.x, lv.x);
                                t1 = fma_f2(mul_f2(t1, c2), ks.y, lv.y);
                            }
                            float x[4];
                            unpack_f2(t0, x[0], x[1]);
                            unpack_f2(t1, x[2], x[3]);
                            t4[0] = fmaxf(fmaxf(t4[0], x[0]), x[1]);
                            t4[1] = fmaxf(fmaxf(t4[1], x[2]), x[3]);
                            t0 = kQuant ? add_f2(t0, minus2) : fma_f2(t0, c2, minus2);
                            t1 = kQuant ? add_f2(t1, minus2) : fma_f2(t1, c2, minus2);
                            if (k % 8 < S::kPolynomial) t1 = ex2_by_polynomial(t1);
                            unpack_f2(t0, x[0], x[1]);
                            unpack_f2(t1, x[2], x[3]);
                            x[0] = ex2(x[0]);
                            x[1] = ex2(x[1]);
                            if (k % 8 >= S::kPolynomial) {
                                x[2] = ex2(x[2]);
                                x[3] = ex2(x[3]);
                            }
                            if constexpr (kQuant) {
                                const ulonglong2 iv = reinterpret_cast<const ulonglong2*>(ka)[64 + at4 + k];
                                sum[0] = fma_f2(pack_f2(x[0], x[1]), iv.x, sum[0]);
                                sum[1] = fma_f2(pack_f2(x[2], x[3]), iv.y, sum[1]);
                            } else {
                                sum[0] = add_f2(pack_f2(x[0], x[1]), sum[0]);
                                sum[1] = add_f2(pack_f2(x[2], x[3]), sum[1]);
                            }
                            w[q][2 * k] = pack2<M>(x[0], x[1]);
                            w[q][2 * k + 1] = pack2<M>(x[2], x[3]);
                        }
                    }
                    float top = fmaxf(t4[0], t4[1]);
                    if (!kQuant) top = top == -INFINITY ? top : top * row_c;
                    const bool move = top > m + 8.f;
                    if (!__any_sync(0xFFFFFFFFu, move)) break;
                    const float alpha = move ? ex2(m - top) : 1.f;
                    if (i + h > 0) {  // the products so far are complete before they are rescaled (all but the last are: see the scores' order)
                        wait(&o_done[s], (2 * i + h - 1) & 1);
                        tc_fence_after();
#pragma unroll 1
                        for (int q = 0; q < DP / 16; ++q) {
                            uint32_t o[16];
                            tmem_load16(o_col + q * 16, o);
                            tmem_wait_load(o);
#pragma unroll
                            for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * alpha);
                            tmem_store16(o_col + q * 16, o);
                        }
                    }
                    l *= alpha;
                    if (move) m = top;
                }
#pragma unroll
                for (int q = 0; q < 2; ++q) tmem_store16(col + q * 16, w[q]);
                float part_sum[2];
                unpack_f2(add_f2(sum[0], sum[1]), part_sum[0], part_sum[1]);
                l += part_sum[0] + part_sum[1];
                tmem_wait_store();
                tc_fence_before();
                mbarrier_arrive(&p_full[s][h]);
            }
        }

        // this part of the row
        if (my_tiles > 0) {
            wait(&o_full[s], 0);
            tc_fence_after();
        }
        const long long part_at = (long long)(narrow ? 2 * run_no + s : run_no) * n_rows;
        const bool empty = l == 0.f;
        const long long my_row = row_index(r);
        if (my_row >= 0) a.part_lse[part_at + my_row] = empty ? -INFINITY : m + log2f(l);
        if (my_tiles > 0) {
            // A thread holds a row, and rows lie apart: 32 columns at a time go through shared memory, so that eight lanes
            // write 128 bytes of a row.  Rows without a key are written too; nothing reads them.
            float inv = empty ? 0.f : 1.0f / l;
            if (kQuant && *reinterpret_cast<volatile int*>(&nan_values[s]) != 0) inv = __uint_as_float(0x7FC00000u);
            unsigned char* stage = DP == 64 ? smem + S::kStageAt + warp * 4096 : q_tiles + S::kTileBytes * (narrow ? 1 : s) + (narrow ? warp : warp & 3) * 4096;
            long long to_row[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) to_row[k] = row_index((warp & 3) * 32 + k * 4 + (lane >> 3));
#pragma unroll 1
            for (int q = 0; q < DP / 32; ++q) {
                uint32_t o[32];
                tmem_load32(o_col + q * 32, o);
                tmem_wait_load(o);
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    *reinterpret_cast<float4*>(stage + lane * 128 + ((k ^ (lane & 7)) << 4)) =
                        make_float4(__uint_as_float(o[4 * k]) * inv, __uint_as_float(o[4 * k + 1]) * inv, __uint_as_float(o[4 * k + 2]) * inv,
                                    __uint_as_float(o[4 * k + 3]) * inv);
                __syncwarp();
                const int col = q * 32 + (lane & 7) * 4;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const int row = k * 4 + (lane >> 3);
                    const float4 x = *reinterpret_cast<const float4*>(stage + row * 128 + (((lane & 7) ^ (row & 7)) << 4));
                    if (to_row[k] >= 0 && col < a.dim) *reinterpret_cast<float4*>(a.part_out + (part_at + to_row[k]) * a.dim + col) = x;
                }
                __syncwarp();
            }
        }
    } else if (warp < 12) {
        // ---- fetching warps ----
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(256 - S::kSoftmaxRegs));
        const int p = tid - 256;
        // Items in the order in which the products want them.  Wide: K0, V0, K1, V1, ...; narrow: K0, K1, V0, K2, V1, ... V(n-1).
        bool values;
        auto item_places = [&](int q) -> const long long* {  // the places of item q's tile
            const int half = (q + 1) >> 1;
            int t;
            if (!narrow) {
                values = q & 1;
                t = q >> 1;
            } else {
                values = q > 0 && (!(q & 1) || half == n);
                t = q == 0 ? 0 : (q & 1) ? (values ? n - 1 : half) : half - 1;
            }
            if (!values) wait(&aux_full[t % kTcAux], (t / kTcAux) & 1);
            return offsets + (t % kTcAux) * kTcTile;
        };
        auto slot_of = [&](int q) -> unsigned char* {
            wait(&empty[q % kTcSlots], ((q / kTcSlots) & 1) ^ 1);
            return ring + (q % kTcSlots) * S::kTileBytes;
        };
        auto announce = [&](int q) {
            fence_async_proxy();
            mbarrier_arrive(&full[q % kTcSlots]);
        };
        const int items = 2 * n;
        if constexpr (kQuant) {
            using C = CodePieces<DP>;
            const int u = p % C::UNITS, r0 = p / C::UNITS;
            const int to = (u >> 2) * kTileBlockBytes + r0 * 128, lo = (((u & 3) * 2) ^ (r0 & 7)) << 4, hi = (((u & 3) * 2 + 1) ^ (r0 & 7)) << 4;
            const bool dims_there = u * 16 < a.dim;
            uint4 w[C::N];
            {
                const long long* off = item_places(0) + r0;
#pragma unroll
                for (int i = 0; i < C::N; ++i) w[i] = ld_codes(a.k + off[i * C::STEP] + u * 16, off[i * C::STEP] >= 0 && dims_there);
            }
#pragma unroll 1
            for (int q = 0; q < items; ++q) {
                const bool more = q + 1 < items;
                const long long* off = more ? item_places(q + 1) + r0 : offsets;
                const unsigned char* side = (values ? a.v : a.k) + u * 16;
                unsigned char* dst = slot_of(q) + to;
#pragma unroll
                for (int i = 0; i < C::N; ++i) {
                    store_codes<FMT>(dst + lo + i * C::STEP * 128, dst + hi + i * C::STEP * 128, w[i]);
                    const long long o = off[i * C::STEP];
                    w[i] = ld_codes(side + o, o >= 0 && dims_there && more);
                }
                announce(q);
            }
        } else {
            const bool dims_there = (p % (DP / 8)) * 8 < a.dim;
#pragma unroll 1
            for (int q = 0; q < items; ++q) {
                const long long* off = item_places(q);
                fetch_plain_tile<DP>(slot_of(q), values ? a.v : a.k, off, p, dims_there, 0);
                if (q > 0) {  // the one before has landed when only this one is outstanding
                    asm volatile("cp.async.wait_group 1;" ::: "memory");
                    announce(q - 1);
                }
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
            announce(items - 1);
        }
    } else {
        // ---- warps 12 and 13 issue the products of the two streams, warps 14 and 15 look up the places ----
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(256 - S::kSoftmaxRegs));
        if (warp < 14) {
            const int s = warp - 12;
            constexpr uint64_t kRowsLayout = tc_layout(16, 1024), kColsLayout = tc_layout(kBlockBytes, 1024);
            constexpr uint32_t kTile16 = S::kTileBytes / 16, kBlock = kBlockBytes / 16, kHalf16 = 64 * 128 / 16;
            const uint32_t q16 = smem_u32(q_tiles) >> 4, ring16 = smem_u32(ring) >> 4;
            // Descriptors of this stream's query tile and of the first ring slot; everything else is a constant away where the slot is one.
            const uint64_t q_at = tc_descriptor(kRowsLayout, q16 + (narrow ? 0 : s) * kTile16);
            const uint64_t k_base = tc_descriptor(kRowsLayout, ring16), v_base = tc_descriptor(kColsLayout, ring16);
            const uint32_t d_scores = tmem + s * kTcTile, d_out = tmem + kColO + s * DP;
            auto wait_item = [&](int i) {
                wait(&full[i % kTcSlots], (i / kTcSlots) & 1);
                tc_fence_after();
            };
            // A slot is free when both streams have released it; in the narrow form one of them does it for both.
            auto release = [&](uint64_t* bar) {
                tc_commit(bar);
                if (narrow) tc_commit(bar);
            };
            // Half h of S = Q K^T with the keys in `slot`
            auto scores = [&](int h, uint32_t slot) {
                const uint64_t k_at = k_base + (slot * kTile16 + h * kHalf16);
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < DP / 16; ++k)
                        tc_mma_ss(d_scores + h * 64, q_at + ((k >> 2) * kBlock + (k & 3) * 2), k_at + ((k >> 2) * kBlock + (k & 3) * 2), kScoreIdesc, k > 0);
                    tc_commit(&s_full[s][h]);
                    if (h == 1) release(&empty[slot]);
                }
                __syncwarp();
            };
            // O += W V with half h of the values in `slot`, of this stream's tile `t` (`first`, `last` of its tiles)
            auto output = [&](int h, uint32_t slot, int t, bool first, bool last) {
                const uint64_t v_at = v_base + (slot * kTile16 + h * kHalf16);
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < kTcTile / 32; ++k)
                        tc_mma_ts(d_out, d_scores + h * 64 + k * 8, v_at + k * 128, kOutIdesc, k + h > 0 ? 1u : (uint32_t)!first);
                    tc_commit(&o_done[s]);
                    if (h == 1) {  // the tile is done with: its values, its places and its constants
                        release(&empty[slot]);
                        release(&aux_free[t % kTcAux]);
                        if (last) tc_commit(&o_full[s]);
                    }
                }
                __syncwarp();
            };
            // Tile number i of this stream: products with its values, then the scores of the next one.
            auto tile = [&](int i, int t, uint32_t v_item, uint32_t v_slot, bool more, uint32_t k_item, uint32_t k_slot) {
                wait_item(v_item);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    wait(&p_full[s][h], i & 1);
                    tc_fence_after();
                    output(h, v_slot, t, i == 0, !more);
                    if (more) {
                        if (h == 0) wait_item(k_item);
                        scores(h, k_slot);
                    }
                }
            };
            wait(&q_full, 0);
            tc_fence_after();
            if (narrow) {
                // items: K_t is 0 or 2 t - 1, V_t is 2 t + 2, the last one 2 n - 1
                if (s < n) {
                    wait_item(s);
                    scores(0, s);
                    scores(1, s);
                }
                for (int t = s; t < n; t += 2) {
                    const uint32_t v_item = t == n - 1 ? 2 * n - 1 : 2 * t + 2, k_item = 2 * t + 3;
                    tile(t >> 1, t, v_item, v_item % kTcSlots, t + 2 < n, k_item, k_item % kTcSlots);
                }
            } else {
                // items: K_t is 2 t, V_t is 2 t + 1
                static_assert(kTcSlots == 4, "keys of even tiles in slot 0, of odd ones in slot 2");
                wait_item(0);
                scores(0, 0);
                scores(1, 0);
                for (int t = 0; t < n; t += 2) {
                    tile(t, t, 2 * t + 1, 1, t + 1 < n, 2 * t + 2, 2);
                    if (t + 1 < n) tile(t + 1, t + 1, 2 * t + 3, 3, t + 2 < n, 2 * t + 4, 0);
                }
            }
            // the tensor memory is given back only when nothing writes it any more
            if (elect_one()) tc_commit(&drained[s]);
            __syncwarp();
            ok = mbarrier_wait_sleeping(&drained[s], 0) && ok;
        } else {
            // Places of the tiles' keys and what the softmax wants to know of them, two keys to a thread, up to kTcAux tiles ahead.
            // A tile's page numbers are read while the tile before it is published.
            const int p = tid - 448;
            int page_n[2];
            auto read_pages = [&](int g) {
                const int pos = (tile0 + g) * kTcTile + p;
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    page_n[y] = -1;  // no such key
                    if (pos + 64 * y >= a.prefix_len) continue;
                    int li;
                    unsigned in_page;
                    split_position(a, pos + 64 * y, li, in_page);
                    const int page = __ldg(a.prefix_pages + li);
                    page_n[y] = page < 0 ? -2 : page;
                }
            };
            read_pages(0);
#pragma unroll 1
            for (int g = 0; g < n; ++g) {
                const int slot = g % kTcAux;
                long long o[2];
                float ks[2] = {0.f, 0.f}, vs[2] = {1.f, 1.f};
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    o[y] = -1;
                    if (page_n[y] == -1) continue;
                    if (page_n[y] < 0 || page_n[y] >= a.n_pages) {
                        atomicExch(a.status, kDeviceIndexCode);
                        continue;
                    }
                    int li;
                    unsigned in_page;
                    split_position(a, (tile0 + g) * kTcTile + p + 64 * y, li, in_page);
                    o[y] = entry_offset(a, page_n[y], in_page, kv_head, false) * (kQuant ? 1 : 2);
                    if constexpr (kQuant) {
                        const long long so = entry_offset(a, page_n[y], in_page, kv_head, true);
                        ks[y] = __ldg(a.k_scale + so);
                        vs[y] = __ldg(a.v_scale + so);
                    }
                }
                if (g + 1 < n) read_pages(g + 1);
                if (a.drop_copies) continue;
                wait(&aux_free[slot], ((g / kTcAux) & 1) ^ 1);
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const bool there = o[y] >= 0;
                    offsets[slot * kTcTile + p + 64 * y] = o[y];
                    float* to = aux + slot * S::kAuxFloats + p + 64 * y;
                    if constexpr (kQuant) {
                        const float u = usable_scale(vs[y]);
                        if (!finite_scale(vs[y])) {
                            if (!narrow || (g & 1) == 0) nan_values[0] = 1;
                            if (!narrow || (g & 1) == 1) nan_values[1] = 1;
                        }
                        to[0] = ks[y];
                        to[kTcTile] = there ? log2f(u) : -INFINITY;
                        to[2 * kTcTile] = there ? __frcp_rn(u) : 0.f;
                    } else {
                        to[0] = there ? 0.f : 1.f;
                    }
                }
                if constexpr (!kQuant) {
                    const uint32_t all = __ballot_sync(0xFFFFFFFFu, o[0] >= 0 && o[1] >= 0);
                    if (lane == 0) reinterpret_cast<unsigned char*>(&ragged[slot])[warp - 14] = all != 0xFFFFFFFFu;
                }
                mbarrier_arrive(&aux_full[slot]);
            }
        }
    }
    if (!ok) atomicExch(a.status, kDeviceTimeoutCode);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 12) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

}  // namespace rt
