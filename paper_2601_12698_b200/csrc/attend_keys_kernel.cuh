// Attention of a few rows to a range of keys of a paged cache on the tensor cores, keys first (sm_100a, tcgen05).
//
// A suffix belongs to one sequence: its keys serve q_len * group rows only, so the work is bound by HBM and what matters is
// that the loads never stop and that little is done per key.  The matrix unit wants 128 rows of its left operand; here these
// are the keys:
//     S^T = K Q^T            128 keys x NR rows, one key to a lane of tensor memory;
//     W^T = 2^(c S^T - m)    thread = key, NR values each, written to shared memory as 16-bit numbers;
//     O^T = V^T W^T          dim x NR, one dim to a lane, summed up in tensor memory over all tiles.
// Keys and values are used as they lie in the cache, K row by row and V column by column (the matrix unit transposes), so
// nothing touches their elements between the copy into shared memory and the product; codes are turned into fp16 on the way.
// Per key a thread handles NR scores instead of head_dim elements.
//
// The softmax needs no reduction over the keys in the usual case.  Every thread keeps the same reference m for each row and
// its own sum of weights per row (joined at the end).  Only when some score exceeds its row's reference by more than 8 (one
// vote per tile) are the tile's maxima found, the reference moved and O^T rescaled.
//
// Warps: 0-3 softmax (one key per thread; they also load the queries), 4-7 fetch the tiles (cp.async into the swizzled
// layout, or codes through registers), 8 issues the products.  Two score buffers and two weight buffers: the scores of
// tile j + 1 are under way while tile j is exponentiated.  Items of 128 keys x up to 128 dims go through a ring; heads of
// 256 take two items a side.  With NR = 16 two CTAs share an SM, so that one streams while the other begins or ends.
//
// NR = 64 (one CTA per SM) serves heads of 256 with many rows, whose two streams would not fit tensor memory in
// attend_prefix_kernel, and suffixes that many rows of their sequence read.
//
// Measured: 256 suffixes of 1 .. 2048 keys x 8 heads of 128, bf16 (1.07 GB): 206 us with the rest of the call, 5.2 TB/s; the same in
// e4m3 (0.55 GB): 247 us, bound by the chain from a tile's codes to its product, not by any unit (64 suffixes: the schedulers issue
// in 31 % of the cycles, ALU 24 %, the shared memory's pipe 35 %, HBM 1.55 TB/s).  A CTA's beginning and end take about 5 us (page numbers, queries,
// the first tile, the first reference, the result), which is why short parts cost more than they balance: 64 suffixes of 1 .. 1024
// keys take 43 us with one part each, 62 with parts of 256 keys, 98 with parts of 128.
// Tried and left: codes fetched into shared memory two items ahead (no change), or into registers two items ahead (spills: 64 us
// instead of 52 for the 64 suffixes in e4m3).
#pragma once

#include "attend_common.cuh"
#include "attend_split.h"
#include "tensor_core.cuh"

namespace rt {

constexpr int kKeysThreads = 288;

template <int FMT, int DP, int NR>
struct KeysShape {
    static constexpr bool kQuant = FMT != kKvPlain;
    static constexpr int DI = DP < 128 ? DP : 128;  // dims of an item
    static constexpr int NI = DP / DI;              // items of a tile and side
    static constexpr int kItemBytes = 128 * DI * 2;
    static constexpr int kCtas = NR == 16 && DP <= 128 ? 2 : 1;
    static constexpr int kSlots = NR == 64 ? 4 : DP == 128 ? 3 : 5;
    static constexpr int kQBytes = NR * DP * 2;
    static constexpr int kWBytes = 128 * NR * 2;
    static constexpr int kColumns = 4 * NR;         // tensor memory: two score buffers, NI <= 2 outputs
    static constexpr size_t kQAt = (size_t)kSlots * kItemBytes, kWAt = kQAt + kQBytes, kOffsetsAt = kWAt + 2 * kWBytes;
    static constexpr size_t kSmem = kOffsetsAt + 3 * 128 * 8 + 1024;  // 1024: alignment of the tiles
};

__device__ __forceinline__ float warp_max(float x)
{
    float y;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
    return y;
}
// OR of `x` over the 128 threads of named barrier 1.
__device__ __forceinline__ bool vote_any_128(bool x)
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, 1, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"((uint32_t)x) : "memory");
    return r != 0;
}
__device__ __forceinline__ void sync_128() { asm volatile("barrier.cta.sync 1, 128;" ::: "memory"); }

// Sums of 16 values over the warp: lane 2 r (and 2 r + 1) ends with the sum of v[r].
__device__ __forceinline__ float warp_sums16(const float* in, int lane)
{
    float v[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = in[i];
#pragma unroll
    for (int half = 8; half >= 1; half >>= 1) {
        const int bit = half * 2;  // lane bit that picks the half
#pragma unroll
        for (int i = 0; i < half; ++i) {
            const bool up = lane & bit;
            const float send = up ? v[i] : v[i + half], keep = up ? v[i + half] : v[i];
            v[i] = keep + __shfl_xor_sync(0xFFFFFFFFu, send, bit);
        }
    }
    return v[0] + __shfl_xor_sync(0xFFFFFFFFu, v[0], 1);
}

// The infinities and NaN among element d of the values of positions [from, to), added up: they were kept out of the product
// (see the fetching warps) and belong to the rows that see them.  0 when there are none.
template <typename T, int FMT>
__device__ __noinline__ float hidden_poison_of(const AttendArgs& a, const int32_t* pages, int list_len, int kv_head, int d, int from, int to)
{
    float sum = 0.f;
    for (int pos = from; pos < to; ++pos) {
        int li;
        unsigned in_page;
        split_position(a, pos, li, in_page);
        const int page = li < list_len ? __ldg(pages + li) : -1;
        if (page < 0 || page >= a.n_pages) continue;
        const long long at = entry_offset(a, page, in_page, kv_head, false) + d;
        float e = 0.f;
        if constexpr (FMT == kKvE4m3) {
            if ((a.v[at] & 0x7F) == 0x7F) e = __uint_as_float(0x7FC00000u);
        } else if constexpr (FMT == kKvPlain) {
            e = Codec<T, 16>::to_float16(reinterpret_cast<const unsigned short*>(a.v)[at]);
        }
        if (!(fabsf(e) < INFINITY)) sum += e;
    }
    return sum;
}

// The first prefix_ctas CTAs: NR rows of one key/value head (over all sequences) against a part of the prefix; the others: NR rows
// of one sequence and key/value head against a part of its suffix.
template <typename T, int FMT, int DP, int NR>
__global__ void __launch_bounds__(kKeysThreads, KeysShape<FMT, DP, NR>::kCtas) attend_keys_kernel(const AttendArgs a, const int prefix_ctas)
{
    using S = KeysShape<FMT, DP, NR>;
    constexpr bool kQuant = S::kQuant;
    using M = typename std::conditional<kQuant, __half, T>::type;
    constexpr int ES = kQuant ? 1 : 2, DI = S::DI, NI = S::NI, SLOTS = S::kSlots;
    constexpr int RB = NR * 2;  // bytes of a row of weights
    constexpr uint32_t kScoreIdesc = tc_instruction<M>(NR, false, false), kOutIdesc = tc_instruction<M>(NR, true, true);

    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    unsigned char* ring = smem;
    unsigned char* q_tile = smem + S::kQAt;
    unsigned char* weights = smem + S::kWAt;
    long long* offsets = reinterpret_cast<long long*>(smem + S::kOffsetsAt);  // [3][128]: places of a tile's keys
    __shared__ __align__(8) uint64_t full[SLOTS], empty[SLOTS], s_full[2], w_full[2], o_done[2], q_full, drained;
    __shared__ uint32_t tmem_base;
    // per row: factor of the scores, reference m (the same for every thread, so it need not sit in their registers), what a new
    // reference rescales by, and the four softmax warps' maxima, sums at the end, and at the beginning the places of the queries
    __shared__ __align__(16) float row_c[NR], row_ref[NR], row_alpha[NR], row_m[4][NR];
    float(&row_sum)[4][NR] = row_m;
    long long* row_q = reinterpret_cast<long long*>(&row_m[0][0]);
    __shared__ __align__(16) long long row_at[NR];  // [token][head] index of a row, -1: no such row; then where its result goes
    __shared__ int poisoned, first_nan_row;  // first_nan_row: from it on, rows see a value whose scale is not finite

    // (the warp's number by shuffle: the compiler then knows that a role is taken by whole warps)
    const int tid = threadIdx.x, warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0), lane = tid & 31;
    const bool prefix = (int)blockIdx.x < prefix_ctas;
    unsigned job = prefix ? blockIdx.x : blockIdx.x - (unsigned)prefix_ctas;
    const int kv_head = (int)(job % (unsigned)a.kv_heads);
    job /= (unsigned)a.kv_heads;
    const unsigned parts = prefix ? a.prefix_parts : a.suffix_parts;
    const int part = (int)(job % parts);
    job /= parts;
    if (tid == 0) {
        for (int i = 0; i < SLOTS; ++i) {
            mbarrier_init(&full[i], 128);
            mbarrier_init(&empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbarrier_init(&s_full[i], 1);
            mbarrier_init(&w_full[i], 128);
            mbarrier_init(&o_done[i], 1);
        }
        mbarrier_init(&q_full, 128);
        mbarrier_init(&drained, 1);
        poisoned = 0;
        first_nan_row = NR;
    }
    const bool beside_prefix = a.after_prefix != 0;  // that of another launch
    if (!beside_prefix) wait_for_previous_kernel();
    const auto leave = [&]() {
        if (beside_prefix && blockIdx.x == 0) wait_for_previous_kernel();
    };

    int len, first_token, n_rows, row0;
    const int32_t* pages;
    int list_len;
    if (prefix) {
        len = a.prefix_len;
        first_token = 0;
        n_rows = a.n_seqs * a.q_len * a.group;
        row0 = (int)job * NR;
        pages = a.prefix_pages;
        list_len = 0x7fffffff;  // the host checked that the list covers prefix_len
    } else {
        const int per_seq = (a.q_len * a.group + NR - 1) / NR;
        const int seq = (int)(job / (unsigned)per_seq);
        row0 = (int)(job % (unsigned)per_seq) * NR;
        len = suffix_length(a, seq);
        if (len < 0) {  // a padded sequence: its rows are not joined either
            leave();
            return;
        }
        first_token = seq * a.q_len;
        n_rows = a.q_len * a.group;
        pages = a.page_table + (long long)seq * a.page_table_stride;
        list_len = a.page_table_width;
    }
    const int part_keys = prefix ? a.prefix_keys : a.suffix_keys;
    const int k0 = part * part_keys, k1 = min(len, k0 + part_keys);
    const int part_index = (prefix ? 0 : a.prefix_parts) + part;
    const bool direct = a.prefix_parts + a.suffix_parts == 1;
    const int n_heads = a.kv_heads * a.group;
    const long long all_rows = (long long)a.n_seqs * a.q_len * n_heads;
    // Row r of the tile: query token first_token + (row0 + r) / group, query head kv_head * group + (row0 + r) % group.
    if (tid < NR) {
        const int r = row0 + tid, t = r / a.group, head = kv_head * a.group + (r - t * a.group);
        row_at[tid] = r < n_rows ? (long long)(first_token + t) * n_heads + head : -1;
        row_q[tid] = r < n_rows ? ((long long)(first_token + t) * a.q_token_stride + (long long)head * a.q_head_stride) * 2 : -1;
    }
    if (k0 >= k1) {  // no keys here: the part only says so
        if (tid < NR && row_at[tid] >= 0) {
            const long long at = row_at[tid];
            if (!direct) {
                a.part_lse[(long long)part_index * all_rows + at] = -INFINITY;
            } else {
                if (a.lse) a.lse[at] = -INFINITY;
                for (int d = 0; d < a.dim; d += 8)
                    *reinterpret_cast<uint4*>(reinterpret_cast<unsigned char*>(a.out) + (at * a.dim + d) * 2) = make_uint4(0, 0, 0, 0);
            }
        }
        leave();
        return;
    }
    if (warp == 8) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base)), "n"(S::kColumns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_base, tmem_o = tmem + 2 * NR;
    const int n = (k1 - k0 + 127) / 128;
    const int live_rows = min(NR, n_rows - row0);  // the rest of the tile is padding: nothing is computed for it beyond the products
    const int all_see = prefix ? len : len - a.q_len + 1;  // keys below it are seen by every row

    // Every wait is bounded.  A thread whose wait has run out stops waiting and goes on through the same loops, so that every
    // barrier is still met and the tensor memory is given back; the status word says that the results are not valid.
    bool ok = true;
    auto wait = [&](uint64_t* bar, uint32_t parity) {
        if (ok) ok = mbarrier_wait_sleeping(bar, parity, a.wait_polls);
    };
    // Page number of key `i` of tile j; -1: there is no such key.
    auto page_of = [&](int j, int i) -> int {
        const int pos = k0 + j * 128 + i;
        if (pos >= k1) return -1;
        int li;
        unsigned in_page;
        split_position(a, pos, li, in_page);
        const int page = li < list_len ? __ldg(pages + li) : -2;
        return page < 0 ? -2 : page;
    };
    auto place_of_key = [&](int j, int i, int page, bool scales) -> long long {
        if (page == -1) return -1;
        if (page < 0 || page >= a.n_pages) {
            atomicExch(a.status, kDeviceIndexCode);
            return -1;
        }
        int li;
        unsigned in_page;
        split_position(a, k0 + j * 128 + i, li, in_page);
        return entry_offset(a, page, in_page, kv_head, scales);
    };

    if (warp < 4) {
        // ---- queries, softmax, result ----
        const uint32_t lanes = (uint32_t)warp << 21;
        int page_n = page_of(0, tid), page_nn = page_of(1, tid);
        // queries: a warp takes a row at a time, all its rows fetched at once
        constexpr int QB = NR / 4;
        {
            uint4 w4[QB];
#pragma unroll
            for (int i = 0; i < QB; ++i) {
                const long long at = row_q[warp + 4 * i];
                w4[i] = make_uint4(0, 0, 0, 0);
                if (at >= 0 && lane * 8 < a.dim) w4[i] = __ldg(reinterpret_cast<const uint4*>(a.q + at + lane * 16));
            }
#pragma unroll
            for (int i = 0; i < QB; ++i) {
                const int r = warp + 4 * i;
                uint4 w = w4[i];
                float c = a.score_scale;
                if constexpr (kQuant) {
                    uint32_t top = __vmaxu2(__vmaxu2(w.x & 0x7FFF7FFFu, w.y & 0x7FFF7FFFu), __vmaxu2(w.z & 0x7FFF7FFFu, w.w & 0x7FFF7FFFu));
                    top = __reduce_max_sync(0xFFFFFFFFu, max(top & 0xFFFFu, top >> 16));
                    const float factor = fp16_row_factor(Codec<T, 16>::to_float16(top));
                    c *= __frcp_rn(factor);
                    uint32_t* p = &w.x;
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        p[k] = pack2<__half>(Codec<T, 16>::to_float16(p[k] & 0xFFFFu) * factor, Codec<T, 16>::to_float16(p[k] >> 16) * factor);
                }
                if (lane == 0) row_c[r] = c;
                if (lane < DP / 8)
                    *reinterpret_cast<uint4*>(q_tile + (lane >> 3) * (NR * 128) + r * 128 + (((lane & 7) ^ (r & 7)) << 4)) = w;
            }
        }
        if (tid < NR) row_ref[tid] = -3.402823466e38f;  // below every score
        fence_async_proxy();
        mbarrier_arrive(&q_full);
        sync_128();

        float l[NR];
#pragma unroll
        for (int r = 0; r < NR; ++r) l[r] = 0.f;
        float ks_n = 0.f, vs_n = 1.f;
        bool there_n;
        auto key_constants = [&](int j, int page) {
            const long long o = place_of_key(j, tid, page, true);
            there_n = o >= 0;
            if constexpr (kQuant) {
                ks_n = there_n ? __ldg(a.k_scale + o) : 0.f;
                vs_n = there_n ? __ldg(a.v_scale + o) : 1.f;
            }
        };
        key_constants(0, page_n);
#pragma unroll 1
        for (int j = 0; j < n; ++j) {
            const bool there = there_n;
            const float ks = ks_n, vs = usable_scale(vs_n);
            const bool value_there = finite_scale(vs_n);
            page_n = page_nn;
            if (j + 1 < n) key_constants(j + 1, page_n);
            if (j + 2 < n) page_nn = page_of(j + 2, tid);
            float lvs = 0.f, ivs = 0.f;
            if constexpr (kQuant) {
                lvs = log2f(vs);
                ivs = __frcp_rn(vs);
            }
            // rows below it do not see this thread's key
            const int hidden = prefix ? 0 : max(0, k0 + j * 128 + tid - (len - a.q_len)) * a.group - row0;
            if (kQuant && !value_there) atomicMin(&first_nan_row, hidden);
            wait(&s_full[j & 1], (j >> 1) & 1);
            tc_fence_after();
            // 16 rows' scores of this thread's key, as logarithms; more rows than that are read again where they are needed
            float t[16];
            auto scores = [&](int r0) {
                uint32_t v[16];
                tmem_load16(tmem + lanes + (j & 1) * NR + r0, v);
                tmem_wait_load(v);
#pragma unroll
                for (int k = 0; k < 16; k += 4) {
                    if (r0 + k >= live_rows) break;
                    float4 c4;
                    if constexpr (kQuant) c4 = *reinterpret_cast<const float4*>(&row_c[r0 + k]);
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        float x;
                        if constexpr (kQuant) x = fmaf(__uint_as_float(v[k + y]) * ks, (&c4.x)[y], lvs);
                        else x = __uint_as_float(v[k + y]) * a.score_scale;
                        t[k + y] = !there || r0 + k + y < hidden ? -INFINITY : x;
                    }
                }
            };
            float over = -INFINITY;
#pragma unroll
            for (int r0 = 0; r0 < NR; r0 += 16) {
                if (r0 >= live_rows) break;
                scores(r0);
#pragma unroll
                for (int k = 0; k < 16; k += 4) {
                    if (r0 + k >= live_rows) break;
                    const float4 m4 = *reinterpret_cast<const float4*>(&row_ref[r0 + k]);
                    over = fmaxf(over, fmaxf(fmaxf(t[k] - m4.x, t[k + 1] - m4.y), fmaxf(t[k + 2] - m4.z, t[k + 3] - m4.w)));
                }
            }
            if (vote_any_128(over > 8.f)) {
                // the tile's largest score of every row, over the warp and then over the four
#pragma unroll 1
                for (int r0 = 0; r0 < live_rows; r0 += 16) {
                    if (NR > 16) scores(r0);
#pragma unroll
                    for (int k = 0; k < 16; k += 4) {
                        if (r0 + k >= live_rows) break;
#pragma unroll
                        for (int r = k; r < k + 4; ++r) {
                            const float top = warp_max(t[r]);
                            if (lane == r) row_m[warp][r0 + r] = top;
                        }
                    }
                }
                sync_128();
                if (tid < NR) {
                    const float top = fmaxf(fmaxf(row_m[0][tid], row_m[1][tid]), fmaxf(row_m[2][tid], row_m[3][tid])), ref = row_ref[tid];
                    row_alpha[tid] = top > ref + 8.f ? ex2(ref - top) : 1.f;
                    if (top > ref + 8.f) row_ref[tid] = top;
                }
                sync_128();
                if (j > 0) {
                    wait(&o_done[(j - 1) & 1], ((j - 1) >> 1) & 1);  // the products so far are complete before they are rescaled
                    tc_fence_after();
#pragma unroll
                    for (int r0 = 0; r0 < NR; r0 += 16) {
                        if (r0 >= live_rows) break;
                        float alpha[16];
#pragma unroll
                        for (int r = 0; r < 16; r += 4) *reinterpret_cast<float4*>(&alpha[r]) = *reinterpret_cast<const float4*>(&row_alpha[r0 + r]);
#pragma unroll
                        for (int r = 0; r < 16; ++r) l[r0 + r] *= alpha[r];
#pragma unroll
                        for (int i = 0; i < NI; ++i) {
                            uint32_t o[16];
                            tmem_load16(tmem_o + lanes + i * NR + r0, o);
                            tmem_wait_load(o);
#pragma unroll
                            for (int r = 0; r < 16; ++r) o[r] = __float_as_uint(__uint_as_float(o[r]) * alpha[r]);
                            tmem_store16(tmem_o + lanes + i * NR + r0, o);
                        }
                        tmem_wait_store();
                    }
                }
            }
            if (j >= 2) wait(&o_done[j & 1], ((j - 2) >> 1) & 1);  // this weight buffer's last product is complete
            unsigned char* to = weights + (j & 1) * S::kWBytes + tid * RB;
#pragma unroll
            for (int r0 = 0; r0 < NR; r0 += 16) {
                if (r0 >= live_rows) break;
                if (NR > 16) scores(r0);
#pragma unroll
                for (int k = 0; k < 16; k += 4) {
                    if (r0 + k >= live_rows) break;
                    const float4 m4 = *reinterpret_cast<const float4*>(&row_ref[r0 + k]);
                    float x[4];
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        x[y] = ex2(t[k + y] - (&m4.x)[y]);
                        if constexpr (kQuant) {  // a hidden key's scale may be NaN
                            if (there && r0 + k + y >= hidden) l[r0 + k + y] = fmaf(x[y], ivs, l[r0 + k + y]);
                        } else {
                            l[r0 + k + y] += x[y];
                        }
                    }
                    const int u = (r0 + k) / 8;
                    *reinterpret_cast<uint2*>(to + ((u ^ (((tid * RB) >> 7) & (RB / 16 - 1))) << 4) + ((k & 4) << 1)) =
                        make_uint2(pack2<M>(x[0], x[1]), pack2<M>(x[2], x[3]));
                }
            }
            fence_async_proxy();
            tc_fence_before();
            mbarrier_arrive(&w_full[j & 1]);
        }

        // the sums of the weights, over the warp and then over the four
#pragma unroll
        for (int r0 = 0; r0 < NR; r0 += 16) {
            if (r0 >= live_rows) break;
            const float sum = warp_sums16(&l[r0], lane);
            if ((lane & 1) == 0) row_sum[warp][r0 + (lane >> 1)] = sum;
        }
        sync_128();
        wait(&o_done[(n - 1) & 1], ((n - 1) >> 1) & 1);
        tc_fence_after();
        // per row, by one thread each: the quotient's factor (-1: the row is not written) and the log-sum-exp
        if (tid < NR) {
            const long long at = row_at[tid];
            const float total = row_sum[0][tid] + row_sum[1][tid] + row_sum[2][tid] + row_sum[3][tid];
            const bool empty = total == 0.f;  // a row that sees a key has a sum above zero, or NaN
            bool write = at >= 0;
            if (prefix && direct && write) write = suffix_length(a, (int)((unsigned)(at / n_heads) / (unsigned)a.q_len)) >= 0;
            if (write) {
                const float lse = empty ? -INFINITY : row_ref[tid] + log2f(total);
                if (!direct) a.part_lse[(long long)part_index * all_rows + at] = lse;
                else if (a.lse) a.lse[at] = lse * 0.69314718055994531f;
            }
            // a part that saw no key is not read by the merge, the result of a call is zero
            // (a padding row is neither)
            const bool nan = kQuant && tid >= *reinterpret_cast<volatile int*>(&first_nan_row);
            row_c[tid] = empty ? 0.f : nan ? __uint_as_float(0x7FC00000u) : 1.0f / total;
            row_at[tid] = !write || (empty && !direct) ? -1 : (direct ? at : (long long)part_index * all_rows + at) * a.dim;
        }
        sync_128();
#pragma unroll 1
        for (int i = 0; i < NI; ++i) {
            const int d = i * 128 + tid;
            const bool mine = d < a.dim && (DI == 128 || tid < DI);
#pragma unroll 1
            for (int r0 = 0; r0 < live_rows; r0 += 16) {
                uint32_t o[16];
                tmem_load16(tmem_o + lanes + i * NR + r0, o);
                tmem_wait_load(o);
#pragma unroll
                for (int k = 0; k < 16; k += 4) {
                    if (r0 + k >= live_rows) break;
                    const float4 f4 = *reinterpret_cast<const float4*>(&row_c[r0 + k]);
                    const longlong2 lo = *reinterpret_cast<const longlong2*>(&row_at[r0 + k]), hi = *reinterpret_cast<const longlong2*>(&row_at[r0 + k + 2]);
                    const long long to[4] = {lo.x, lo.y, hi.x, hi.y};
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        const float f = (&f4.x)[y], x = f == 0.f ? 0.f : __uint_as_float(o[k + y]) * f;
                        if (to[y] < 0 || !mine) continue;
                        if (direct) reinterpret_cast<unsigned short*>(a.out)[to[y] + d] = (unsigned short)Codec<T, 16>::from_float16(x);
                        else a.part_out[to[y] + d] = x;
                    }
                }
            }
        }
        if (!prefix && *reinterpret_cast<volatile int*>(&poisoned) != 0) {  // the infinities kept out of the products (below)
#pragma unroll 1
            for (int r = 0; r < live_rows; ++r) {
#pragma unroll 1
                for (int i = 0; i < NI; ++i) {
                    const int d = i * 128 + tid;
                    const long long to = row_at[r];
                    if (to < 0 || d >= a.dim || (DI < 128 && tid >= DI)) continue;
                    const float poison = hidden_poison_of<T, FMT>(a, pages, list_len, kv_head, d, max(k0, all_see), min(k1, len - a.q_len + (row0 + r) / a.group + 1));
                    if (poison == 0.f) continue;
                    if (direct) reinterpret_cast<unsigned short*>(a.out)[to + d] = (unsigned short)Codec<T, 16>::from_float16(poison + Codec<T, 16>::to_float16(reinterpret_cast<unsigned short*>(a.out)[to + d]));
                    else a.part_out[to + d] += poison;
                }
            }
        }
    } else if (warp < 8) {
        // ---- fetching warps ----
        const int p = tid - 128;
        // Items in the order in which the products want them, NI of each: K0, K1, V0, K2, V1, ... K(n-1), V(n-2), V(n-1).
        const int items = 2 * n * NI;
        struct Item {
            int tile, part_of_dims;
            bool values;
        };
        auto item_at = [&](int q) -> Item {
            const int g = q / NI, half = (g + 1) >> 1;
            const bool values = g > 0 && (!(g & 1) || half == n);
            return {g == 0 ? 0 : (g & 1) ? (values ? n - 1 : half) : half - 1, q % NI, values};
        };
        // Places of a tile's keys, one thread to a key, published when the tile's first keys are fetched; its page number was
        // read two tiles earlier.  Tile j + 2 is published when every thread is past the values of tile j - 1.
        long long off_n = place_of_key(0, p, page_of(0, p), false);
        int page_n = page_of(1, p);
        auto begin_item = [&](const Item& it) -> const long long* {
            const int j = it.tile;
            if (!it.values && it.part_of_dims == 0) {
                offsets[(j % 3) * 128 + p] = off_n < 0 ? -1 : off_n * ES;
                if (j + 1 < n) off_n = place_of_key(j + 1, p, page_n, false);
                if (j + 2 < n) page_n = page_of(j + 2, p);
                asm volatile("barrier.cta.sync 2, 128;" ::: "memory");
            }
            return offsets + (j % 3) * 128;
        };
        auto slot_of = [&](int q) -> unsigned char* {
            wait(&empty[q % SLOTS], ((q / SLOTS) & 1) ^ 1);
            return ring + (q % SLOTS) * S::kItemBytes;
        };
        auto announce = [&](int q) {
            fence_async_proxy();
            if (!a.drop_copies) mbarrier_arrive(&full[q % SLOTS]);
        };
        // Some rows do not see the last keys, and 0 * infinity would reach them through the product: such values become zero in
        // the tile and are added to the rows that do see them at the end.
        auto guarded = [&](const Item& it) { return it.values && !prefix && a.q_len > 1 && k0 + it.tile * 128 + 128 > all_see; };
        if constexpr (kQuant) {
            using C = CodePieces<DI>;
            const int u = p % C::UNITS, r0 = p / C::UNITS;
            const int to = (u >> 2) * kTileBlockBytes + r0 * 128, lo = (((u & 3) * 2) ^ (r0 & 7)) << 4, hi = (((u & 3) * 2 + 1) ^ (r0 & 7)) << 4;
            uint4 w[C::N];
            Item it = item_at(0);
            {
                const long long* off = begin_item(it) + r0;
#pragma unroll
                for (int i = 0; i < C::N; ++i) w[i] = ld_codes(a.k + off[i * C::STEP] + u * 16, off[i * C::STEP] >= 0 && u * 16 < a.dim);
            }
#pragma unroll 1
            for (int q = 0; q < items; ++q) {
                const bool guard = FMT == kKvE4m3 && guarded(it);
                const int first_pos = k0 + it.tile * 128 + r0;
                const bool more = q + 1 < items;
                if (more) it = item_at(q + 1);
                const long long* off = more ? begin_item(it) + r0 : offsets;
                const unsigned char* side = (it.values ? a.v : a.k) + it.part_of_dims * DI + u * 16;
                const bool dims_there = more && it.part_of_dims * DI + u * 16 < a.dim;
                unsigned char* dst = slot_of(q) + to;
#pragma unroll
                for (int i = 0; i < C::N; ++i) {
                    if (guard && first_pos + i * C::STEP >= all_see) {
                        uint32_t* x = &w[i].x;
                        uint32_t hits = 0;
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const uint32_t hit = __vcmpeq4(x[k] & 0x7F7F7F7Fu, 0x7F7F7F7Fu);
                            hits |= hit;
                            x[k] &= ~hit;
                        }
                        if (hits) poisoned = 1;
                    }
                    store_codes<FMT>(dst + lo + i * C::STEP * 128, dst + hi + i * C::STEP * 128, w[i]);
                    const long long o = off[i * C::STEP];
                    w[i] = ld_codes(side + o, o >= 0 && dims_there);
                }
                announce(q);
            }
        } else {
#pragma unroll 1
            for (int q = 0; q < items; ++q) {
                const Item it = item_at(q);
                const long long* off = begin_item(it);
                const int dim0 = it.part_of_dims * DI;
                constexpr int UNITS = DI / 8, STEP = 128 / UNITS;
                const int u = p % UNITS, r0 = p / UNITS;
                unsigned char* dst = slot_of(q);
                fetch_plain_tile<DI>(dst, it.values ? a.v : a.k, off, p, dim0 + u * 8 < a.dim, dim0 * 2);
                if (q > 0) {  // the one before has landed when only this one is outstanding
                    asm volatile("cp.async.wait_group 1;" ::: "memory");
                    announce(q - 1);
                }
                if (guarded(it)) {
                    bool hit_any = false;
                    asm volatile("cp.async.wait_group 0;" ::: "memory");
#pragma unroll 1
                    for (int r = r0; r < 128; r += STEP) {
                        if (k0 + it.tile * 128 + r < all_see) continue;
                        uint4* at = reinterpret_cast<uint4*>(dst + (u >> 3) * kTileBlockBytes + r * 128 + (((u & 7) ^ (r & 7)) << 4));
                        uint4 w = *at;
                        uint32_t* x = &w.x;
                        constexpr uint32_t kTop = std::is_same<T, __nv_bfloat16>::value ? 0x7F807F80u : 0x7C007C00u;
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const uint32_t hit = __vcmpeq2(x[k] & kTop, kTop);
                            hit_any = hit_any || hit != 0;
                            x[k] &= ~hit;
                        }
                        *at = w;
                    }
                    if (hit_any) poisoned = 1;
                }
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
            announce(items - 1);
        }
    } else {
        // ---- the warp that issues the products ----
        uint32_t item = 0;
        constexpr uint64_t kRowsLayout = tc_layout(16, 1024);
        // heads of 64: both halves of the unit's 128 rows are the same 64 dims
        constexpr uint64_t kValuesLayout = tc_layout(DI == 64 ? 0 : kTileBlockBytes, 1024), kWeightsLayout = tc_layout<RB>(16, 8 * RB);
        const uint32_t ring16 = smem_u32(ring) >> 4, q16 = smem_u32(q_tile) >> 4, w16 = smem_u32(weights) >> 4;
        auto take = [&]() -> uint32_t {
            wait(&full[item % SLOTS], (item / SLOTS) & 1);
            tc_fence_after();
            return ring16 + (item % SLOTS) * (S::kItemBytes / 16);
        };
        auto scores = [&](int j) {
            const uint32_t d = tmem + (j & 1) * NR;
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const uint32_t k_at = take();
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < DI / 16; ++k)
                        tc_mma_ss(d, tc_descriptor(kRowsLayout, k_at + ((k >> 2) * kTileBlockBytes + (k & 3) * 32) / 16),
                                  tc_descriptor(kRowsLayout, q16 + ((i * (DI / 64) + (k >> 2)) * (NR * 128) + (k & 3) * 32) / 16), kScoreIdesc, i > 0 || k > 0);
                    tc_commit(&empty[item % SLOTS]);
                    if (i == NI - 1) tc_commit(&s_full[j & 1]);
                }
                __syncwarp();
                ++item;
            }
        };
        wait(&q_full, 0);
        tc_fence_after();
        scores(0);
        for (int j = 0; j < n; ++j) {
            if (j + 1 < n) scores(j + 1);
            wait(&w_full[j & 1], (j >> 1) & 1);
            tc_fence_after();
            const uint32_t w_at = w16 + (j & 1) * (S::kWBytes / 16);
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const uint32_t v_at = take();
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        tc_mma_ss(tmem_o + i * NR, tc_descriptor(kValuesLayout, v_at + k * 128), tc_descriptor(kWeightsLayout, w_at + k * RB), kOutIdesc,
                                  k > 0 ? 1u : (uint32_t)(j > 0));
                    tc_commit(&empty[item % SLOTS]);
                    if (i == NI - 1) tc_commit(&o_done[j & 1]);
                }
                __syncwarp();
                ++item;
            }
        }
        // The tensor memory is given back only when nothing writes it any more.  (A barrier of its own: when a wait has run out, the
        // products ran ahead of the roles that o_done keeps in step, and its parity says nothing about the last of them.)
        if (elect_one()) tc_commit(&drained);
        __syncwarp();
        ok = mbarrier_wait_sleeping(&drained, 0) && ok;
    }
    if (!ok) atomicExch(a.status, kDeviceTimeoutCode);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 8) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(S::kColumns) : "memory");
    leave();
}

}  // namespace rt
