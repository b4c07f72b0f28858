// Attention of many rows to a shared prefix on the fifth-generation tensor cores (sm_100a, tcgen05 + tensor memory).
//
// All rows of one key/value head (every sequence's query tokens and the head's query heads) see the same keys, so the
// prefix is a plain matrix problem:  S = Q K^T,  W = 2^(score_scale S - m),  O = W V,  in one pass over the keys with a
// running reference m and sum per row.  A "unit" is one key/value head and one block of rows (up to 256); its keys come in
// tiles of 128.  The tiles of all units are numbered through and dealt out in equal consecutive runs, one run to a CTA and
// one CTA to an SM, so the SMs finish together whatever the number of heads and rows; a run may end one unit and begin the
// next.  What a CTA finds out about a unit is one part (two in the narrow form below), joined by merge_parts_kernel.
//
// Inside a CTA (13 warps):
//   warps 0-3, 4-7   two softmax streams of 128 rows, one row to a thread (tensor memory lane = row): they read S from
//                    tensor memory, keep m and the sum in registers, and write the weights back over S as the 16-bit
//                    left operand of the second product;
//   warps 8-11       fetch the paged tiles: keys and values with cp.async, 16 bytes a piece, into the 128-byte-swizzled
//                    layout that the matrix unit reads (pages may have any size, so one copy per row is the widest that
//                    always works); quantised tiles are fetched into registers, turned into fp16 and stored;
//   warp 12          one thread issues the matrix products.
// The two streams take turns on the tensor cores: while one's scores are exponentiated the other's products run.  Blocks of
// more than 128 rows (wide form): a stream is one half of the rows, both use the same tiles.  Blocks of up to 128 rows
// (narrow form): both streams use the same rows and alternate the tiles, and leave a part each.
//
// The reference m is moved only when the row's maximum exceeds it by more than 8 (a factor of 256): then the sum and the
// output row in tensor memory are rescaled by the row's own thread.  Weights are thus at most 256, which bf16 and fp16 hold
// with their full relative precision, and the quotient is the same.
//
// Quantised caches: both products run in fp16 on codes, with the scales in the exponent, as in attend_rows_kernel.cuh.
//
// Bounds: 4 * 128 * 128 * dim flops and 128 * 128 exponentials per tile and stream; at dim 128 the tensor cores need 1024
// cycles for that and the SM's 16 exponentials a cycle 1024 as well.
#pragma once

#include "attend_common.cuh"
#include "attend_split.h"

namespace rt {

constexpr int kTcThreads = 416;
constexpr int kTcSlots = 4;   // ring of key and value tiles
constexpr int kTcAux = 4;     // tiles whose per-key constants are kept

template <int FMT, int DP>
struct PrefixShape {
    static constexpr bool kQuant = FMT != kKvPlain;
    static constexpr int kTileBytes = kTcTile * DP * 2;
    static constexpr int kAuxFloats = kQuant ? 3 * kTcTile : kTcTile;
    static constexpr size_t kAuxAt = (size_t)(2 + kTcSlots) * kTileBytes;
    static constexpr size_t kOffsetsAt = kAuxAt + (size_t)kTcAux * kAuxFloats * 4;
    static constexpr size_t kSmem = kOffsetsAt + (size_t)kTcAux * kTcTile * 8 + 1024;  // 1024: alignment of the tiles
};

// ---- tensor memory and matrix instructions -----------------------------------------------------------------

__device__ __forceinline__ void tmem_load32(uint32_t addr, uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,"
        "%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr));
}
__device__ __forceinline__ void tmem_wait_load() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_store32(uint32_t addr, const uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,"
        "%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};" ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]),
        "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]),
        "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
        "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tmem_store16(uint32_t addr, const uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::"r"(r[0]), "r"(r[1]),
        "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]),
        "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tmem_wait_store() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_async_proxy() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

__device__ __forceinline__ void tc_commit(uint64_t* bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// D (128 x N, binary32, tensor memory) (+)= A B with A and B described in shared memory.
__device__ __forceinline__ void tc_mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
                 "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate) : "memory");
}
// The same with A (128 x 16 of 16-bit elements, two to a column) in tensor memory.
__device__ __forceinline__ void tc_mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
                 "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate) : "memory");
}
// Shared memory matrix descriptor: 128-byte swizzle, strides in bytes (leading: between 64-element column blocks of an
// operand whose rows are the product's inner axis; stride: between groups of eight rows).
__device__ __forceinline__ uint64_t tc_descriptor(uint32_t smem_addr, uint32_t leading, uint32_t stride)
{
    return (uint64_t)((smem_addr >> 4) & 0x3FFFu) | ((uint64_t)((leading >> 4) & 0x3FFFu) << 16) |
           ((uint64_t)((stride >> 4) & 0x3FFFu) << 32) | (1ull << 46) | (2ull << 61);
}
// Instruction descriptor: binary32 accumulator, A and B both bf16 or both fp16, M = 128.
template <typename M>
__device__ __forceinline__ constexpr uint32_t tc_instruction(int n, bool b_inner_rows)
{
    const uint32_t type = std::is_same<M, __nv_bfloat16>::value ? 1u : 0u;
    return (1u << 4) | (type << 7) | (type << 10) | ((b_inner_rows ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | ((128u >> 4) << 24);
}

__device__ __forceinline__ void mbarrier_arrive(uint64_t* bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}

template <typename T, int FMT, int DP>
__global__ void __launch_bounds__(kTcThreads, 1) attend_prefix_kernel(const AttendArgs a, const PrefixSplit split)
{
    using S = PrefixShape<FMT, DP>;
    constexpr bool kQuant = S::kQuant;
    using M = typename std::conditional<kQuant, __half, T>::type;
    constexpr int kBlockBytes = kTcTile * 128;  // one 64-dim column block of a tile
    constexpr uint32_t kScoreIdesc = tc_instruction<M>(kTcTile, false), kOutIdesc = tc_instruction<M>(DP, true);
    constexpr uint32_t kColO = 2 * kTcTile;

    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    unsigned char* q_tiles = smem;
    unsigned char* ring = smem + 2 * S::kTileBytes;
    float* aux = reinterpret_cast<float*>(smem + S::kAuxAt);
    long long* offsets = reinterpret_cast<long long*>(smem + S::kOffsetsAt);
    __shared__ __align__(8) uint64_t full[kTcSlots], empty[kTcSlots], aux_full[kTcAux], s_full[2], p_full[2], o_full[2], q_full, drained;
    __shared__ uint32_t tmem_base;
    __shared__ uint32_t ragged[kTcAux];  // one byte per fetching warp: some key of its quarter of the tile is not there

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int i = 0; i < kTcSlots; ++i) {
            mbarrier_init(&full[i], 128);
            mbarrier_init(&empty[i], 1);
        }
        for (int i = 0; i < kTcAux; ++i) mbarrier_init(&aux_full[i], 128);
        for (int i = 0; i < 2; ++i) {
            mbarrier_init(&s_full[i], 1);
            mbarrier_init(&p_full[i], 128);
            mbarrier_init(&o_full[i], 1);
        }
        mbarrier_init(&q_full, 256);
        mbarrier_init(&drained, 1);
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

    const long long total = (long long)split.tiles * split.blocks * a.kv_heads;
    const long long begin = (long long)blockIdx.x * split.run, end = min(total, begin + split.run);
    // Every wait is bounded.  A thread whose wait has run out stops waiting and goes on through the same loops, so that every
    // barrier is still met and the tensor memory is given back; the status word says that the results are not valid.
    bool ok = true;
    auto wait = [&](uint64_t* bar, uint32_t parity) {
        if (ok) ok = mbarrier_wait_bounded(bar, parity);
    };

    if (warp < 8) {
        // ---- softmax streams ----
        const int s = warp >> 2, r = (warp & 3) * 32 + lane;
        const uint32_t lane_base = tmem + ((uint32_t)(warp & 3) << 21);
        const uint32_t s_col = lane_base + s * kTcTile, o_col = lane_base + kColO + s * DP;
        const bool flip = a.score_scale < 0.f;
        const float scale = fabsf(a.score_scale);
        uint32_t n_s = 0, n_o = 0, tile_no = 0;
        for (long long at = begin; at < end;) {
            const int unit = (int)(at / split.tiles), block = unit % split.blocks, kv_head = unit / split.blocks;
            const int tile0 = (int)(at - (long long)unit * split.tiles);
            const int n = (int)min((long long)(split.tiles - tile0), end - at);
            const bool narrow = narrow_block(split, block);
            const int first_row = block * kTcBlockRows + (narrow ? 0 : s * 128);
            // Query rows into shared memory: this thread's row (narrow form: the first stream's threads do it for both).
            // Nobody reads the tiles any more: this thread's stream has seen its last product of the previous unit, and
            // the barrier makes that so for both.
            asm volatile("bar.sync 1, 256;" ::: "memory");
            float row_c = scale;
            const int row = first_row + r;
            const bool live = row < split.rows;
            const int token = live ? row / a.group : 0, head = kv_head * a.group + (live ? row - token * a.group : 0);
            {
                const unsigned char* src = a.q + ((long long)token * a.q_token_stride + (long long)head * a.q_head_stride) * 2;
                float factor = 1.f;
                if constexpr (kQuant) {
                    uint32_t top = 0;
                    if (live) {
#pragma unroll 4
                        for (int e = 0; e < a.dim; e += 8) {
                            const uint4 w = __ldg(reinterpret_cast<const uint4*>(src + e * 2));
                            top = __vmaxu2(top, __vmaxu2(__vmaxu2(w.x & 0x7FFF7FFFu, w.y & 0x7FFF7FFFu), __vmaxu2(w.z & 0x7FFF7FFFu, w.w & 0x7FFF7FFFu)));
                        }
                    }
                    factor = fp16_row_factor(Codec<T, 16>::to_float16(max(top & 0xFFFFu, top >> 16)));
                    row_c *= __frcp_rn(factor);
                }
                if (!narrow || s == 0) {
                    unsigned char* dst = q_tiles + s * S::kTileBytes + r * 128;
#pragma unroll 4
                    for (int u = 0; u < DP / 8; ++u) {
                        uint4 w = make_uint4(0, 0, 0, 0);
                        if (live && u * 8 < a.dim) {
                            w = __ldg(reinterpret_cast<const uint4*>(src + u * 16));
                            if (flip) { w.x ^= 0x80008000u; w.y ^= 0x80008000u; w.z ^= 0x80008000u; w.w ^= 0x80008000u; }
                            if constexpr (kQuant) {
                                uint32_t* p = &w.x;
#pragma unroll
                                for (int i = 0; i < 4; ++i)
                                    p[i] = pack2<__half>(Codec<T, 16>::to_float16(p[i] & 0xFFFFu) * factor, Codec<T, 16>::to_float16(p[i] >> 16) * factor);
                            }
                        }
                        *reinterpret_cast<uint4*>(dst + (u >> 3) * kBlockBytes + (((u & 7) ^ (r & 7)) << 4)) = w;
                    }
                }
            }
            fence_async_proxy();
            mbarrier_arrive(&q_full);

            float m = -INFINITY, l = 0.f;
            const int my_tiles = narrow ? (n + 1 - s) / 2 : n;
            for (int i = 0; i < my_tiles; ++i) {
                const uint32_t t = tile_no + (narrow ? 2 * i + s : i);
                const uint32_t aux_i = t % kTcAux;
                wait(&aux_full[aux_i], (t / kTcAux) & 1);
                wait(&s_full[s], n_s & 1);
                ++n_s;
                tc_fence_after();
                const float4* ka = reinterpret_cast<const float4*>(aux + aux_i * S::kAuxFloats);
                const bool holes = !kQuant && *reinterpret_cast<volatile uint32_t*>(&ragged[aux_i]) != 0;
                // largest score of the tile
                float top = -INFINITY;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    uint32_t v[32];
                    tmem_load32(s_col + q * 32, v);
                    tmem_wait_load();
                    if constexpr (kQuant) {
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const float4 ks = ka[q * 8 + k], lv = ka[32 + q * 8 + k];
                            top = fmaxf(fmaxf(top, fmaf(__uint_as_float(v[4 * k]) * row_c, ks.x, lv.x)), fmaf(__uint_as_float(v[4 * k + 1]) * row_c, ks.y, lv.y));
                            top = fmaxf(fmaxf(top, fmaf(__uint_as_float(v[4 * k + 2]) * row_c, ks.z, lv.z)), fmaf(__uint_as_float(v[4 * k + 3]) * row_c, ks.w, lv.w));
                        }
                    } else if (holes) {
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const float4 b = ka[q * 8 + k];
                            top = fmaxf(fmaxf(top, b.x == 0.f ? __uint_as_float(v[4 * k]) : -INFINITY), b.y == 0.f ? __uint_as_float(v[4 * k + 1]) : -INFINITY);
                            top = fmaxf(fmaxf(top, b.z == 0.f ? __uint_as_float(v[4 * k + 2]) : -INFINITY), b.w == 0.f ? __uint_as_float(v[4 * k + 3]) : -INFINITY);
                        }
                    } else {
#pragma unroll
                        for (int k = 0; k < 32; k += 2) top = fmaxf(fmaxf(top, __uint_as_float(v[k])), __uint_as_float(v[k + 1]));
                    }
                }
                if (!kQuant) top = top == -INFINITY ? top : top * row_c;  // row_c may be zero
                const bool move = top > m + 8.f;
                if (__any_sync(0xFFFFFFFFu, move)) {
                    const float alpha = move ? ex2(m - top) : 1.f;
                    if (i > 0) {
#pragma unroll 1
                        for (int q = 0; q < DP / 32; ++q) {
                            uint32_t v[32];
                            tmem_load32(o_col + q * 32, v);
                            tmem_wait_load();
#pragma unroll
                            for (int k = 0; k < 32; ++k) v[k] = __float_as_uint(__uint_as_float(v[k]) * alpha);
                            tmem_store32(o_col + q * 32, v);
                        }
                    }
                    l *= alpha;
                    if (move) m = top;
                }
                const float base = m == -INFINITY ? 0.f : m;
                float sum[2] = {0.f, 0.f};
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    uint32_t v[32], w[16];
                    tmem_load32(s_col + q * 32, v);
                    tmem_wait_load();
                    if constexpr (kQuant) {
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const float4 ks = ka[q * 8 + k], lv = ka[32 + q * 8 + k], iv = ka[64 + q * 8 + k];
                            const float x0 = ex2(fmaf(__uint_as_float(v[4 * k]) * row_c, ks.x, lv.x) - base);
                            const float x1 = ex2(fmaf(__uint_as_float(v[4 * k + 1]) * row_c, ks.y, lv.y) - base);
                            const float x2 = ex2(fmaf(__uint_as_float(v[4 * k + 2]) * row_c, ks.z, lv.z) - base);
                            const float x3 = ex2(fmaf(__uint_as_float(v[4 * k + 3]) * row_c, ks.w, lv.w) - base);
                            sum[0] = fmaf(x0, iv.x, sum[0]); sum[1] = fmaf(x1, iv.y, sum[1]);
                            sum[0] = fmaf(x2, iv.z, sum[0]); sum[1] = fmaf(x3, iv.w, sum[1]);
                            w[2 * k] = pack2<M>(x0, x1);
                            w[2 * k + 1] = pack2<M>(x2, x3);
                        }
                    } else {
                        if (holes) {
#pragma unroll
                            for (int k = 0; k < 8; ++k) {
                                const float4 b = ka[q * 8 + k];
                                if (b.x != 0.f) v[4 * k] = 0xFF800000u;
                                if (b.y != 0.f) v[4 * k + 1] = 0xFF800000u;
                                if (b.z != 0.f) v[4 * k + 2] = 0xFF800000u;
                                if (b.w != 0.f) v[4 * k + 3] = 0xFF800000u;
                            }
                        }
#pragma unroll
                        for (int k = 0; k < 16; ++k) {
                            float x0 = ex2(fmaf(__uint_as_float(v[2 * k]), row_c, -base)), x1 = ex2(fmaf(__uint_as_float(v[2 * k + 1]), row_c, -base));
                            if (holes) {  // 0 * -inf when the score scale is zero
                                if (v[2 * k] == 0xFF800000u) x0 = 0.f;
                                if (v[2 * k + 1] == 0xFF800000u) x1 = 0.f;
                            }
                            sum[0] += x0;
                            sum[1] += x1;
                            w[k] = pack2<M>(x0, x1);
                        }
                    }
                    tmem_store16(s_col + q * 16, w);
                }
                l += sum[0] + sum[1];
                tmem_wait_store();
                tc_fence_before();
                mbarrier_arrive(&p_full[s]);
            }
            tile_no += n;

            // this part of the row
            if (my_tiles > 0) {
                wait(&o_full[s], n_o & 1);
                ++n_o;
                tc_fence_after();
            }
            const long long part = blockIdx.x - (long long)unit * split.tiles / split.run;
            const int part_index = (int)(narrow ? 2 * part + s : part);
            const long long n_rows = (long long)a.n_seqs * a.q_len * a.kv_heads * a.group;
            const long long out_row = (long long)part_index * n_rows + (long long)token * a.kv_heads * a.group + head;
            const bool empty = l == 0.f;
            if (my_tiles > 0) {
                const float inv = empty ? 0.f : 1.0f / l;
#pragma unroll 1
                for (int q = 0; q < DP / 32; ++q) {
                    uint32_t v[32];
                    tmem_load32(o_col + q * 32, v);
                    tmem_wait_load();
                    if (live && !empty) {
#pragma unroll
                        for (int k = 0; k < 32; k += 4)
                            if (q * 32 + k < a.dim)
                                *reinterpret_cast<float4*>(a.part_out + out_row * a.dim + q * 32 + k) =
                                    make_float4(__uint_as_float(v[k]) * inv, __uint_as_float(v[k + 1]) * inv, __uint_as_float(v[k + 2]) * inv,
                                                __uint_as_float(v[k + 3]) * inv);
                    }
                }
            }
            if (live) a.part_lse[out_row] = empty ? -INFINITY : m + log2f(l);
            tc_fence_before();
            at += n;
        }
    } else if (warp < 12) {
        // ---- fetching warps ----
        const int p = tid - 256;
        uint32_t item = 0, tile_no = 0;
        uint32_t pending = 0;          // items issued but not yet announced (plain: cp.async groups)
        auto announce = [&](uint32_t i) {
            fence_async_proxy();
            mbarrier_arrive(&full[i % kTcSlots]);
        };
        // One tile of keys or values; `t` numbers the tile, whose places are in offsets[t % kTcAux].
        auto fetch = [&](const unsigned char* side, uint32_t t) {
            wait(&empty[item % kTcSlots], ((item / kTcSlots) & 1) ^ 1);
            unsigned char* dst = ring + (item % kTcSlots) * S::kTileBytes;
            const long long* off = offsets + (t % kTcAux) * kTcTile;
            if constexpr (kQuant) {
                constexpr int UNITS = DP / 16;            // 16 codes a piece
                constexpr int STEP = 128 / UNITS, N = kTcTile / STEP;
                const int u = p % UNITS, row0 = p / UNITS;
#pragma unroll
                for (int h = 0; h < N; h += 8) {
                    uint4 w[8];
#pragma unroll
                    for (int i = 0; i < 8 && i < N; ++i) {
                        const long long o = off[row0 + (h + i) * STEP];
                        w[i] = make_uint4(0, 0, 0, 0);
                        if (o >= 0 && u * 16 < a.dim) w[i] = __ldg(reinterpret_cast<const uint4*>(side + o + u * 16));
                    }
#pragma unroll
                    for (int i = 0; i < 8 && i < N; ++i) {
                        const int r = row0 + (h + i) * STEP;
                        unsigned char* base = dst + (u >> 2) * kBlockBytes + r * 128;
                        const uint4 lo = make_uint4(pick_half2<FMT, 0, 1>(w[i].x, w[i].x), pick_half2<FMT, 2, 3>(w[i].x, w[i].x),
                                                    pick_half2<FMT, 0, 1>(w[i].y, w[i].y), pick_half2<FMT, 2, 3>(w[i].y, w[i].y));
                        const uint4 hi = make_uint4(pick_half2<FMT, 0, 1>(w[i].z, w[i].z), pick_half2<FMT, 2, 3>(w[i].z, w[i].z),
                                                    pick_half2<FMT, 0, 1>(w[i].w, w[i].w), pick_half2<FMT, 2, 3>(w[i].w, w[i].w));
                        *reinterpret_cast<uint4*>(base + ((((u & 3) * 2) ^ (r & 7)) << 4)) = lo;
                        *reinterpret_cast<uint4*>(base + ((((u & 3) * 2 + 1) ^ (r & 7)) << 4)) = hi;
                    }
                }
                announce(item);
            } else {
                constexpr int UNITS = DP / 8;             // 16 bytes a piece
                constexpr int STEP = 128 / UNITS;
                const int u = p % UNITS, row0 = p / UNITS;
#pragma unroll 8
                for (int r = row0; r < kTcTile; r += STEP) {
                    const long long o = off[r];
                    const bool there = o >= 0 && u * 8 < a.dim;
                    const unsigned char* src = there ? side + (o + u * 8) * 2 : side;
                    const uint32_t to = smem_u32(dst + (u >> 3) * kBlockBytes + r * 128 + (((u & 7) ^ (r & 7)) << 4));
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(src), "r"(there ? 16 : 0) : "memory");
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
                if (++pending == 2) {  // the one before has landed when only this one is outstanding
                    asm volatile("cp.async.wait_group 1;" ::: "memory");
                    announce(item - 1);
                    --pending;
                }
            }
            ++item;
        };
        for (long long at = begin; at < end;) {
            const int unit = (int)(at / split.tiles), block = unit % split.blocks, kv_head = unit / split.blocks;
            const int tile0 = (int)(at - (long long)unit * split.tiles);
            const int n = (int)min((long long)(split.tiles - tile0), end - at);
            const int lead = narrow_block(split, block) ? 2 : 1;
            // order of the tiles in the ring: K0 (K1), then V0 K(lead) V1 K(lead + 1) ...
            auto keys = [&](int j) {
                const uint32_t t = tile_no + j;
                const int pos = (tile0 + j) * kTcTile + p;
                long long o = -1, so = -1;
                if (pos < a.prefix_len) {
                    int li;
                    unsigned in_page;
                    split_position(a, pos, li, in_page);
                    const int page = __ldg(a.prefix_pages + li);
                    if (page >= 0 && page < a.n_pages) {
                        o = entry_offset(a, page, in_page, kv_head, false);
                        so = entry_offset(a, page, in_page, kv_head, true);
                    } else {
                        atomicExch(a.status, kDeviceIndexCode);
                    }
                }
                offsets[(t % kTcAux) * kTcTile + p] = o;
                float* to = aux + (t % kTcAux) * S::kAuxFloats + p;
                if constexpr (kQuant) {
                    const float ks = o >= 0 ? __ldg(a.k_scale + so) : 0.f, vs = o >= 0 ? usable_scale(__ldg(a.v_scale + so)) : 0.f;
                    to[0] = ks;
                    to[kTcTile] = o >= 0 ? log2f(vs) : -INFINITY;
                    to[2 * kTcTile] = o >= 0 ? __frcp_rn(vs) : 0.f;
                } else {
                    to[0] = o >= 0 ? 0.f : 1.f;
                    const uint32_t there = __ballot_sync(0xFFFFFFFFu, o >= 0);
                    if (lane == 0) reinterpret_cast<unsigned char*>(&ragged[t % kTcAux])[warp - 8] = there != 0xFFFFFFFFu;
                }
                mbarrier_arrive(&aux_full[t % kTcAux]);
                asm volatile("bar.sync 2, 128;" ::: "memory");
                fetch(a.k, t);
            };
            for (int j = 0; j < lead && j < n; ++j) keys(j);
            for (int j = 0; j < n; ++j) {
                fetch(a.v, tile_no + j);
                if (j + lead < n) keys(j + lead);
            }
            tile_no += n;
            at += n;
        }
        if constexpr (!kQuant) {
            asm volatile("cp.async.wait_all;" ::: "memory");
            if (pending) announce(item - 1);
        }
    } else {
        // ---- the thread that issues the products ----
        if (lane == 0) {
            uint32_t item = 0, n_q = 0, n_p[2] = {0, 0};
            const uint32_t q_addr = smem_u32(q_tiles), ring_addr = smem_u32(ring);
            auto wait_item = [&](uint32_t i) {
                wait(&full[i % kTcSlots], (i / kTcSlots) & 1);
                tc_fence_after();
            };
            auto scores = [&](int s, int q_tile, uint32_t i) {
                const uint32_t k_addr = ring_addr + (i % kTcSlots) * S::kTileBytes, q = q_addr + q_tile * S::kTileBytes;
    #pragma unroll
                for (int k = 0; k < DP / 16; ++k) {
                    const uint32_t step = (k >> 2) * kBlockBytes + (k & 3) * 32;
                    tc_mma_ss(tmem + s * kTcTile, tc_descriptor(q + step, 16, 1024), tc_descriptor(k_addr + step, 16, 1024), kScoreIdesc, k > 0);
                }
            };
            auto output = [&](int s, uint32_t i, bool first) {
                const uint32_t v_addr = ring_addr + (i % kTcSlots) * S::kTileBytes;
    #pragma unroll
                for (int k = 0; k < kTcTile / 16; ++k)
                    tc_mma_ts(tmem + kColO + s * DP, tmem + s * kTcTile + k * 8, tc_descriptor(v_addr + k * 2048, kBlockBytes, 1024), kOutIdesc,
                              !first || k > 0);
            };
            auto wait_weights = [&](int s) {
                wait(&p_full[s], n_p[s] & 1);
                ++n_p[s];
                tc_fence_after();
            };
            for (long long at = begin; at < end;) {
                const int unit = (int)(at / split.tiles), block = unit % split.blocks;
                const int tile0 = (int)(at - (long long)unit * split.tiles);
                const int n = (int)min((long long)(split.tiles - tile0), end - at);
                wait(&q_full, n_q & 1);
                ++n_q;
                tc_fence_after();
                if (narrow_block(split, block)) {
                    for (int j = 0; j < 2 && j < n; ++j) {
                        wait_item(item);
                        scores(j, 0, item);
                        tc_commit(&s_full[j]);
                        tc_commit(&empty[item % kTcSlots]);
                        ++item;
                    }
                    for (int j = 0; j < n; ++j) {
                        const int s = j & 1;
                        wait_item(item);
                        wait_weights(s);
                        output(s, item, j < 2);
                        tc_commit(&empty[item % kTcSlots]);
                        ++item;
                        if (j + 2 < n) {
                            wait_item(item);
                            scores(s, 0, item);
                            tc_commit(&s_full[s]);
                            tc_commit(&empty[item % kTcSlots]);
                            ++item;
                        } else {
                            tc_commit(&o_full[s]);
                        }
                    }
                } else {
                    wait_item(item);
                    for (int s = 0; s < 2; ++s) {
                        scores(s, s, item);
                        tc_commit(&s_full[s]);
                    }
                    tc_commit(&empty[item % kTcSlots]);
                    ++item;
                    for (int j = 0; j < n; ++j) {
                        const uint32_t v_item = item, k_item = item + 1;
                        const bool more = j + 1 < n;
                        wait_item(v_item);
                        for (int s = 0; s < 2; ++s) {
                            wait_weights(s);
                            output(s, v_item, j == 0);
                            if (s == 1) tc_commit(&empty[v_item % kTcSlots]);
                            if (more) {
                                if (s == 0) wait_item(k_item);
                                scores(s, s, k_item);
                                tc_commit(&s_full[s]);
                                if (s == 1) tc_commit(&empty[k_item % kTcSlots]);
                            } else {
                                tc_commit(&o_full[s]);
                            }
                        }
                        item += more ? 2 : 1;
                    }
                }
                at += n;
            }
            // the tensor memory is given back only when nothing writes it any more
            tc_commit(&drained);
            ok = mbarrier_wait_bounded(&drained, 0) && ok;
        }
        __syncwarp();
    }
    if (!ok) atomicExch(a.status, kDeviceTimeoutCode);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 12) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

}  // namespace rt
