// Attention of 16 rows to a range of keys of a paged cache, and the joining of such partial results (sm_100a).
//
// Per row, over the keys of the range that it sees, with t_j = score_scale * <q, k_j> (base-2 logarithms):
//     m = max_j t_j,  w_j = 2^(t_j - m),  out = sum_j w_j v_j / sum_j w_j,  lse = m + log2 sum_j w_j,
// in one pass: running maximum and sum, the output rescaled when the maximum moves.
//
// A suffix belongs to one sequence, so its keys serve q_len * group rows only: the work is bound by HBM, and what
// matters is that the loads never stop.  Each of the CTA's four warps walks over its own blocks of KB keys with keys and
// values coming straight from global memory into the registers in which the matrix instruction wants them, 16 bytes to
// a lane: because a dot product does not care about the order of its terms, the 16 bytes that a lane holds of a key
// are declared to be its terms of two (plain) or four (quantised) consecutive k-steps, and the query fragments are laid
// out in shared memory in that same order; and because the columns of the output may be computed in any order, the 16
// bytes of a value row that a lane holds are its column of eight (sixteen) consecutive n-tiles.  Two register
// buffers, one for keys and one for values (heads of 256: two halves of each in turn), are refilled as soon as they are
// consumed, so about 8 KB per warp are in flight all the time.  No shared memory is used for keys and values, and no
// barrier is met before the end, where the four warps' results are joined.
// mma.sync is enough here: 16 rows per tile are what there is, and tcgen05 would want 64 or 128.
//
// Quantised caches: codes are exact in fp16, so both products run in fp16, on query rows scaled by a power of two.
// With per-key scales a_j = k_scale_j, b_j = v_scale_j:
//     t_j = (score_scale / factor * <q', code_j>) a_j + log2 b_j,  w_j = 2^(t_j - m),
//     out = sum_j w_j vcode_j / sum_j (w_j / b_j):
// the value scale goes into the exponent, which keeps every weight at most 1 whatever the scales are.
#pragma once

#include "attend_common.cuh"
#include "attend_split.h"

namespace rt {

constexpr int kRowsThreads = 128;
constexpr int kRowsWarps = kRowsThreads / 32;

template <int FMT, int DP>
struct RowsShape {
    static constexpr bool kQuant = FMT != kKvPlain;
    static constexpr int PD = DP < 128 ? DP : 128;               // dims of one register buffer
    static constexpr int NP = DP / PD;                           // buffers per key block and side
    static constexpr int KB = DP == 64 ? 32 : 16;  // keys per block
    static constexpr int K_CHUNK = kQuant ? 16 : 8;              // dims in a lane's 16 bytes of a key
    static constexpr int K_CHUNKS = PD / (4 * K_CHUNK);
    static constexpr int V_CHUNK = kQuant ? (PD == 64 ? 8 : 16) : 8;  // dims in a lane's chunk of a value row
    static constexpr int V_CHUNKS = PD / (8 * V_CHUNK);
    static constexpr int V_WORDS = kQuant ? V_CHUNK / 4 : 4;
    static constexpr int K_WORDS_ALL = KB / 8 * K_CHUNKS * 4;
    static constexpr int V_WORDS_ALL = KB / 16 * 4 * V_CHUNKS * V_WORDS;
    static constexpr int WORDS = K_WORDS_ALL > V_WORDS_ALL ? K_WORDS_ALL : V_WORDS_ALL;
    static constexpr int TILES = PD / 8;                          // output n-tiles per buffer
    static constexpr int O_STRIDE = DP + 4;
    static constexpr size_t kSmem = (size_t)DP * 32 + 2 * 16 * O_STRIDE * 4;
};

// 16 or 8 bytes, or zeros.  The zeros are set ahead of a predicated load, inside one statement: written as a branch, the
// registers of both sides meet in a move that waits for the load.
__device__ __forceinline__ void ld_words4(const unsigned char* p, bool there, uint32_t* w)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %5, 0;\n\tmov.u32 %0, 0;\n\tmov.u32 %1, 0;\n\tmov.u32 %2, 0;\n\tmov.u32 %3, 0;\n\t"
                 "@p ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];\n\t}"
                 : "=&r"(w[0]), "=&r"(w[1]), "=&r"(w[2]), "=&r"(w[3]) : "l"(p), "r"((uint32_t)there));
}
__device__ __forceinline__ void ld_words2(const unsigned char* p, bool there, uint32_t* w)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %3, 0;\n\tmov.u32 %0, 0;\n\tmov.u32 %1, 0;\n\t"
                 "@p ld.global.L1::no_allocate.v2.u32 {%0,%1}, [%2];\n\t}"
                 : "=&r"(w[0]), "=&r"(w[1]) : "l"(p), "r"((uint32_t)there));
}

// PREFIX: the rows of one key/value head (16 of them) against a part of the prefix; else the rows of one sequence and
// key/value head against a part of its suffix.
template <typename T, int FMT, int DP, bool PREFIX>
__global__ void __launch_bounds__(kRowsThreads, DP == 256 ? 2 : 3) attend_rows_kernel(const AttendArgs a)
{
    using S = RowsShape<FMT, DP>;
    constexpr bool kQuant = S::kQuant;
    using M = typename std::conditional<kQuant, __half, T>::type;  // type of both matrix products
    constexpr int ES = kQuant ? 1 : 2;                             // bytes per element of the cache
    extern __shared__ __align__(16) unsigned char smem[];
    uint4* qfrag = reinterpret_cast<uint4*>(smem);                 // [DP / 16 k-steps][32 lanes]
    float* obuf = reinterpret_cast<float*>(smem + (size_t)DP * 32);  // [2][16][O_STRIDE]
    __shared__ float row_scale[16];
    __shared__ float warp_m[kRowsWarps][16], warp_l[kRowsWarps][16];
    __shared__ int poisoned;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3;
    if (tid == 0) poisoned = 0;
    // job: key/value head fastest (neighbouring CTAs read neighbouring heads of the same tokens), then part, then tile
    unsigned job = blockIdx.x;
    const int kv_head = (int)(job % (unsigned)a.kv_heads);
    job /= (unsigned)a.kv_heads;
    const unsigned parts = PREFIX ? a.prefix_parts : a.suffix_parts;
    const int part = (int)(job % parts);
    job /= parts;
    wait_for_previous_kernel();
    int len, first_token, n_rows, row0;
    const int32_t* pages;
    int list_len;
    if constexpr (PREFIX) {
        len = a.prefix_len;
        first_token = 0;
        n_rows = a.n_seqs * a.q_len * a.group;
        row0 = (int)job * 16;
        pages = a.prefix_pages;
        list_len = 0x7fffffff;  // the host checked that the list covers prefix_len
    } else {
        const int per_seq = (a.q_len * a.group + 15) / 16;
        const int seq = (int)(job / (unsigned)per_seq);
        row0 = (int)(job % (unsigned)per_seq) * 16;
        len = suffix_length(a, seq);
        if (len < 0) return;  // a padded sequence: its rows are not joined either
        first_token = seq * a.q_len;
        n_rows = a.q_len * a.group;
        pages = a.page_table + (long long)seq * a.page_table_stride;
        list_len = a.page_table_width;
    }
    const int part_keys = PREFIX ? a.prefix_keys : a.suffix_keys;
    const int k0 = part * part_keys;
    const int k1 = min(len, k0 + part_keys);
    const int part_index = (PREFIX ? 0 : a.prefix_parts) + part;
    const bool direct = a.prefix_parts + a.suffix_parts == 1;
    const long long n_tokens = (long long)a.n_seqs * a.q_len;
    const int n_heads = a.kv_heads * a.group;
    // Row r of the tile: query token first_token + (row0 + r) / group, query head kv_head * group + (row0 + r) % group.
    if (k0 >= k1 && !direct) {  // nothing here: the part only says so
        if (tid < 16 && row0 + tid < n_rows) {
            const int r = row0 + tid, t = r / a.group;
            a.part_lse[((long long)part_index * n_tokens + first_token + t) * n_heads + kv_head * a.group + (r - t * a.group)] = -INFINITY;
        }
        return;
    }

    // query rows into fragment order
    if constexpr (kQuant) {
#pragma unroll 1
        for (int r = warp; r < 16; r += kRowsWarps) {
            float top = 0.f;
            if (row0 + r < n_rows) {
                const int t = (row0 + r) / a.group, h = kv_head * a.group + (row0 + r - t * a.group);
                const unsigned char* src = a.q + ((long long)(first_token + t) * a.q_token_stride + (long long)h * a.q_head_stride) * 2;
                uint32_t joined = 0;
                for (int e = lane * 8; e < a.dim; e += 256) {
                    const uint4 w = __ldg(reinterpret_cast<const uint4*>(src + e * 2));
                    joined = __vmaxu2(joined, __vmaxu2(__vmaxu2(w.x & 0x7FFF7FFFu, w.y & 0x7FFF7FFFu), __vmaxu2(w.z & 0x7FFF7FFFu, w.w & 0x7FFF7FFFu)));
                }
                joined = __reduce_max_sync(0xFFFFFFFFu, max(joined & 0xFFFFu, joined >> 16));
                top = Codec<T, 16>::to_float16(joined);
            }
            if (lane == 0) row_scale[r] = fp16_row_factor(top);
        }
        __syncthreads();
    }
#pragma unroll 1
    for (int i = tid; i < DP / 16 * 32; i += kRowsThreads) {
        const int step = i >> 5, l = i & 31, lc = l & 3;
        const int in_piece = step % (S::PD / 16), piece = step / (S::PD / 16);
        const int dim0 = piece * S::PD + (kQuant ? 64 * (in_piece >> 2) + 16 * lc + 4 * (in_piece & 3) : 32 * (in_piece >> 1) + 8 * lc + 4 * (in_piece & 1));
        uint2 w[2];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int r = row0 + (l >> 2) + 8 * half;
            w[half] = make_uint2(0, 0);
            if (r < n_rows && dim0 < a.dim) {
                const int t = r / a.group, h = kv_head * a.group + (r - t * a.group);
                w[half] = __ldg(reinterpret_cast<const uint2*>(a.q + ((long long)(first_token + t) * a.q_token_stride + (long long)h * a.q_head_stride + dim0) * 2));
                if constexpr (kQuant) {
                    const float f = row_scale[(l >> 2) + 8 * half];
                    float x[4];
                    x[0] = Codec<T, 16>::to_float16(w[half].x & 0xFFFFu); x[1] = Codec<T, 16>::to_float16(w[half].x >> 16);
                    x[2] = Codec<T, 16>::to_float16(w[half].y & 0xFFFFu); x[3] = Codec<T, 16>::to_float16(w[half].y >> 16);
                    w[half] = make_uint2(pack2<__half>(x[0] * f, x[1] * f), pack2<__half>(x[2] * f, x[3] * f));
                }
            }
        }
        qfrag[i] = make_uint4(w[0].x, w[1].x, w[0].y, w[1].y);
    }
    __syncthreads();

    // this lane's rows: g and g + 8 of the tile
    int limit[2];  // keys that the row sees
    float row_c[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const int r = row0 + g + 8 * x;
        limit[x] = PREFIX ? len : len - a.q_len + (r < n_rows ? r / a.group : a.q_len - 1) + 1;
        row_c[x] = a.score_scale;
        if constexpr (kQuant) row_c[x] *= __frcp_rn(row_scale[g + 8 * x]);
    }
    const int all_see = PREFIX ? len : len - a.q_len + 1;  // keys below it are seen by every row

    float acc[S::NP][S::TILES][4];
#pragma unroll
    for (int p = 0; p < S::NP; ++p)
#pragma unroll
        for (int t = 0; t < S::TILES; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[p][t][e] = 0.f;
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
    bool saw_poison = false;

    // Places of the keys of a block: lane j (j < KB) keeps key j's.  Three blocks are in the pipe: the one being
    // computed, the one whose keys and values are being fetched, and the one whose page numbers are.
    const int n_blocks = (k1 - k0 + S::KB - 1) / S::KB;
    auto page_of = [&](int b) -> int {  // page number of this lane's key of block b, -1: no such key
        const int pos = k0 + b * S::KB + lane;
        if (lane >= S::KB || pos >= k1 || b >= n_blocks) return -1;
        int li;
        unsigned in_page;
        split_position(a, pos, li, in_page);
        if (li >= list_len) {
            atomicExch(a.status, kDeviceIndexCode);
            return -1;
        }
        const int page = __ldg(pages + li);
        return page < 0 ? -2 : page;
    };
    auto place = [&](int b, int page, bool scales) -> long long {
        if (page == -1) return -1;
        if (page < 0 || page >= a.n_pages) {
            atomicExch(a.status, kDeviceIndexCode);
            return -1;
        }
        int li;
        unsigned in_page;
        split_position(a, k0 + b * S::KB + lane, li, in_page);
        return entry_offset(a, page, in_page, kv_head, scales);
    };

    uint32_t buf[2][S::WORDS];
    auto load_keys = [&](uint32_t (&w)[S::WORDS], long long off, int piece) {
#pragma unroll
        for (int nt = 0; nt < S::KB / 8; ++nt) {
            const long long o = __shfl_sync(0xFFFFFFFFu, off, nt * 8 + g);
#pragma unroll
            for (int i = 0; i < S::K_CHUNKS; ++i) {
                const int d = piece * S::PD + i * 4 * S::K_CHUNK + c * S::K_CHUNK;
                uint32_t* to = &w[(nt * S::K_CHUNKS + i) * 4];
                ld_words4(a.k + (o + d) * ES, o >= 0 && d < a.dim, to);
            }
        }
    };
    auto load_values = [&](uint32_t (&w)[S::WORDS], long long off, int piece) {
#pragma unroll
        for (int u = 0; u < S::KB / 16; ++u)
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const long long o = __shfl_sync(0xFFFFFFFFu, off, u * 16 + 2 * c + (y & 1) + 8 * (y >> 1));
#pragma unroll
                for (int i = 0; i < S::V_CHUNKS; ++i) {
                    const int d = piece * S::PD + i * 8 * S::V_CHUNK + g * S::V_CHUNK;
                    uint32_t* to = &w[((u * 4 + y) * S::V_CHUNKS + i) * S::V_WORDS];
                    if constexpr (S::V_WORDS == 4) ld_words4(a.v + (o + d) * ES, o >= 0 && d < a.dim, to);
                    else ld_words2(a.v + (o + d) * ES, o >= 0 && d < a.dim, to);
                }
            }
    };
    // piece p of a block: 0 .. NP-1 keys, NP .. 2*NP-1 values; it lives in buffer p % 2
    auto load_piece = [&](int p, long long off) {
        if (p < S::NP) load_keys(buf[p & 1], off, p);
        else load_values(buf[p & 1], off, p - S::NP);
    };

    int page_b = page_of(warp), page_n = page_of(warp + kRowsWarps), page_nn;
    long long off = place(warp, page_b, false), off_n;
    float ks = 0.f, vs = 1.f, ks_n = 0.f, vs_n = 1.f;
    auto load_scales = [&](int b, int page, float& k_out, float& v_out) {
        if constexpr (kQuant) {
            const long long o = place(b, page, true);
            k_out = o >= 0 ? __ldg(a.k_scale + o) : 0.f;
            v_out = o >= 0 ? __ldg(a.v_scale + o) : 1.f;
        }
    };
    if (warp < n_blocks) {
        load_piece(0, off);
        load_piece(1, off);
        load_scales(warp, page_b, ks, vs);
    }
#pragma unroll 1
    for (int b = warp; b < n_blocks; b += kRowsWarps) {
        page_nn = page_of(b + 2 * kRowsWarps);
        off_n = place(b + kRowsWarps, page_n, false);
        load_scales(b + kRowsWarps, page_n, ks_n, vs_n);
        const unsigned valid = __ballot_sync(0xFFFFFFFFu, off >= 0);
        const int pos0 = k0 + b * S::KB;

        float s[S::KB / 8][4];
#pragma unroll
        for (int nt = 0; nt < S::KB / 8; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[nt][e] = 0.f;
#pragma unroll
        for (int p = 0; p < S::NP; ++p) {
#pragma unroll
            for (int ks16 = 0; ks16 < S::PD / 16; ++ks16) {
                const uint4 qf = qfrag[(p * (S::PD / 16) + ks16) * 32 + lane];
                const uint32_t af[4] = {qf.x, qf.y, qf.z, qf.w};
#pragma unroll
                for (int nt = 0; nt < S::KB / 8; ++nt) {
                    if constexpr (kQuant) {
                        const uint32_t w = buf[p & 1][(nt * S::K_CHUNKS + ks16 / 4) * 4 + ks16 % 4];
                        mma_16x8x16<M>(s[nt], af, pick_half2<FMT, 0, 1>(w, w), pick_half2<FMT, 2, 3>(w, w));
                    } else {
                        const uint32_t* w = &buf[p & 1][(nt * S::K_CHUNKS + ks16 / 2) * 4 + 2 * (ks16 % 2)];
                        mma_16x8x16<M>(s[nt], af, w[0], w[1]);
                    }
                }
            }
            load_piece((p + 2) % (2 * S::NP), p + 2 < 2 * S::NP ? off : off_n);
        }

        // scores in base-2 logarithms, hidden ones -inf
        float lvs = 0.f, ivs = 0.f;
        if constexpr (kQuant) {
            const float u = usable_scale(vs);
            lvs = log2f(u);
            ivs = __frcp_rn(u);
        }
        const bool ragged = valid != (S::KB == 32 ? 0xFFFFFFFFu : (1u << (S::KB & 31)) - 1u) || pos0 + S::KB > all_see;
        float inv_scale[S::KB / 8][2];
#pragma unroll
        for (int nt = 0; nt < S::KB / 8; ++nt) {
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const int j = nt * 8 + 2 * c + y;
                if constexpr (kQuant) {
                    const float kj = __shfl_sync(0xFFFFFFFFu, ks, j), lj = __shfl_sync(0xFFFFFFFFu, lvs, j);
                    inv_scale[nt][y] = __shfl_sync(0xFFFFFFFFu, ivs, j);
                    s[nt][y] = fmaf(s[nt][y] * row_c[0], kj, lj);
                    s[nt][2 + y] = fmaf(s[nt][2 + y] * row_c[1], kj, lj);
                } else {
                    s[nt][y] *= row_c[0];
                    s[nt][2 + y] *= row_c[1];
                }
                if (ragged) {
                    const bool there = (valid >> j) & 1u;
                    if (!there || pos0 + j >= limit[0]) s[nt][y] = -INFINITY;
                    if (!there || pos0 + j >= limit[1]) s[nt][2 + y] = -INFINITY;
                }
            }
        }
        float alpha[2];
        bool moved = false;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            float top = m[x];
#pragma unroll
            for (int nt = 0; nt < S::KB / 8; ++nt) top = fmaxf(top, fmaxf(s[nt][2 * x], s[nt][2 * x + 1]));
            top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
            const float base = top == -INFINITY ? 0.f : top;
            alpha[x] = ex2(m[x] - base);
            moved = moved || top != m[x];
            m[x] = top;
            float sum = 0.f;
#pragma unroll
            for (int nt = 0; nt < S::KB / 8; ++nt)
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const float w = ex2(s[nt][2 * x + y] - base);
                    s[nt][2 * x + y] = w;
                    if constexpr (kQuant) sum += ragged && w == 0.f ? 0.f : w * inv_scale[nt][y];  // a hidden key's scale may be NaN
                    else sum += w;
                }
            l[x] = l[x] * alpha[x] + sum;
        }
        if (__any_sync(0xFFFFFFFFu, moved)) {
#pragma unroll
            for (int p = 0; p < S::NP; ++p)
#pragma unroll
                for (int t = 0; t < S::TILES; ++t) {
                    acc[p][t][0] *= alpha[0]; acc[p][t][1] *= alpha[0];
                    acc[p][t][2] *= alpha[1]; acc[p][t][3] *= alpha[1];
                }
        }
        uint32_t pf[S::KB / 16][4];
#pragma unroll
        for (int u = 0; u < S::KB / 16; ++u) {
            pf[u][0] = pack2<M>(s[2 * u][0], s[2 * u][1]);
            pf[u][1] = pack2<M>(s[2 * u][2], s[2 * u][3]);
            pf[u][2] = pack2<M>(s[2 * u + 1][0], s[2 * u + 1][1]);
            pf[u][3] = pack2<M>(s[2 * u + 1][2], s[2 * u + 1][3]);
        }
#pragma unroll
        for (int p = 0; p < S::NP; ++p) {
            uint32_t(&w)[S::WORDS] = buf[(S::NP + p) & 1];
            if (!PREFIX && pos0 + S::KB > all_see) {
                // Some rows do not see the last keys, and 0 * infinity would reach them through the product: such
                // values leave the product here and are added to the rows that do see them at the end.
#pragma unroll
                for (int u = 0; u < S::KB / 16; ++u)
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        if (pos0 + u * 16 + 2 * c + (y & 1) + 8 * (y >> 1) < all_see) continue;
#pragma unroll
                        for (int i = 0; i < S::V_CHUNKS * S::V_WORDS; ++i) {
                            uint32_t& x = w[(u * 4 + y) * S::V_CHUNKS * S::V_WORDS + i];
                            constexpr uint32_t kTop = kQuant ? 0x7F7F7F7Fu : (std::is_same<T, __nv_bfloat16>::value ? 0x7F807F80u : 0x7C007C00u);
                            if constexpr (FMT == kKvInt8) continue;
                            const uint32_t hit = kQuant ? __vcmpeq4(x & kTop, kTop) : __vcmpeq2(x & kTop, kTop);
                            saw_poison = saw_poison || hit != 0;
                            x &= ~hit;
                        }
                    }
            }
#pragma unroll
            for (int u = 0; u < S::KB / 16; ++u)
#pragma unroll
                for (int i = 0; i < S::V_CHUNKS; ++i) {
                    const uint32_t* w0 = &w[((u * 4 + 0) * S::V_CHUNKS + i) * S::V_WORDS];
                    const uint32_t* w1 = &w[((u * 4 + 1) * S::V_CHUNKS + i) * S::V_WORDS];
                    const uint32_t* w2 = &w[((u * 4 + 2) * S::V_CHUNKS + i) * S::V_WORDS];
                    const uint32_t* w3 = &w[((u * 4 + 3) * S::V_CHUNKS + i) * S::V_WORDS];
#pragma unroll
                    for (int k = 0; k < S::V_WORDS; ++k) {
                        if constexpr (kQuant) {
                            float(*to)[4] = &acc[p][i * S::V_CHUNK + 4 * k];
                            mma_16x8x16<M>(to[0], pf[u], pick_half2<FMT, 0, 4>(w0[k], w1[k]), pick_half2<FMT, 0, 4>(w2[k], w3[k]));
                            mma_16x8x16<M>(to[1], pf[u], pick_half2<FMT, 1, 5>(w0[k], w1[k]), pick_half2<FMT, 1, 5>(w2[k], w3[k]));
                            mma_16x8x16<M>(to[2], pf[u], pick_half2<FMT, 2, 6>(w0[k], w1[k]), pick_half2<FMT, 2, 6>(w2[k], w3[k]));
                            mma_16x8x16<M>(to[3], pf[u], pick_half2<FMT, 3, 7>(w0[k], w1[k]), pick_half2<FMT, 3, 7>(w2[k], w3[k]));
                        } else {
                            float(*to)[4] = &acc[p][i * S::V_CHUNK + 2 * k];
                            mma_16x8x16<M>(to[0], pf[u], __byte_perm(w0[k], w1[k], 0x5410), __byte_perm(w2[k], w3[k], 0x5410));
                            mma_16x8x16<M>(to[1], pf[u], __byte_perm(w0[k], w1[k], 0x7632), __byte_perm(w2[k], w3[k], 0x7632));
                        }
                    }
                }
            const int next = S::NP + p + 2;
            load_piece(next % (2 * S::NP), next < 2 * S::NP ? off : off_n);
        }
        off = off_n;
        ks = ks_n;
        vs = vs_n;
        page_n = page_nn;
    }

    // the four warps' results, joined in a fixed order
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        l[x] += __shfl_xor_sync(0xFFFFFFFFu, l[x], 1);
        l[x] += __shfl_xor_sync(0xFFFFFFFFu, l[x], 2);
        if (c == 0) {
            warp_m[warp][g + 8 * x] = m[x];
            warp_l[warp][g + 8 * x] = l[x];
        }
    }
    if (saw_poison) poisoned = 1;
    __syncthreads();
    float mult[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < kRowsWarps; ++w) top = fmaxf(top, warp_m[w][g + 8 * x]);
        mult[x] = top == -INFINITY ? 0.f : ex2(m[x] - top);
    }
#pragma unroll
    for (int phase = 0; phase < 2; ++phase) {
        if ((warp >> 1) == phase) {
            float* to = obuf + (warp & 1) * 16 * S::O_STRIDE;
#pragma unroll
            for (int p = 0; p < S::NP; ++p)
#pragma unroll
                for (int i = 0; i < S::V_CHUNKS; ++i)
#pragma unroll
                    for (int x = 0; x < 4; ++x)  // rows g (x < 2) and g + 8, columns 2c (even x) and 2c + 1
#pragma unroll
                        for (int j = 0; j < S::V_CHUNK; j += 4) {
                            const int d = p * S::PD + i * 8 * S::V_CHUNK + (2 * c + (x & 1)) * S::V_CHUNK + j;
                            float4* at = reinterpret_cast<float4*>(to + (g + 8 * (x >> 1)) * S::O_STRIDE + d);
                            const float f = mult[x >> 1];
                            float4 o = make_float4(acc[p][i * S::V_CHUNK + j][x] * f, acc[p][i * S::V_CHUNK + j + 1][x] * f,
                                                   acc[p][i * S::V_CHUNK + j + 2][x] * f, acc[p][i * S::V_CHUNK + j + 3][x] * f);
                            if (phase == 1) {
                                const float4 old = *at;
                                o.x += old.x; o.y += old.y; o.z += old.z; o.w += old.w;
                            }
                            *at = o;
                        }
        }
        __syncthreads();
    }
    for (int i = tid; i < 16 * (DP / 8); i += kRowsThreads) {
        const int r = i / (DP / 8), d = (i % (DP / 8)) * 8;
        if (row0 + r >= n_rows || d >= a.dim) continue;
        float top = -INFINITY, total = 0.f;
#pragma unroll
        for (int w = 0; w < kRowsWarps; ++w) top = fmaxf(top, warp_m[w][r]);
#pragma unroll
        for (int w = 0; w < kRowsWarps; ++w)
            if (warp_l[w][r] != 0.f) total += warp_l[w][r] * ex2(warp_m[w][r] - top);  // NaN scores stay NaN
        const bool empty = total == 0.f;  // a warp that saw a key has a sum above zero, or NaN
        const float inv = empty ? 0.f : 1.0f / total;
        const int t = (row0 + r) / a.group, h = kv_head * a.group + (row0 + r - t * a.group);
        float o[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float sum = obuf[r * S::O_STRIDE + d + j] + obuf[(16 + r) * S::O_STRIDE + d + j];
            o[j] = empty ? 0.f : sum * inv;
        }
        if (!PREFIX && poisoned) {
            const int sees = min(k1, len - a.q_len + t + 1);
            for (int pos = max(k0, all_see); pos < sees; ++pos) {
                int li;
                unsigned in_page;
                split_position(a, pos, li, in_page);
                const int page = li < list_len ? __ldg(pages + li) : -1;
                if (page < 0 || page >= a.n_pages) continue;
                const unsigned char* src = a.v + (entry_offset(a, page, in_page, kv_head, false) + d) * ES;
                for (int j = 0; j < 8; ++j) {
                    float v;
                    if constexpr (kQuant) {
                        v = (src[j] & 0x7F) == 0x7F && FMT == kKvE4m3 ? __uint_as_float(0x7FC00000u) : 0.f;
                    } else {
                        v = Codec<T, 16>::to_float16(reinterpret_cast<const unsigned short*>(src)[j]);
                    }
                    if (!(fabsf(v) < INFINITY)) o[j] += v;
                }
            }
        }
        const long long row = (long long)(first_token + t) * n_heads + h;
        if (direct) {
            if (PREFIX && __ldg(a.suffix_lens + t / a.q_len) < 0) continue;  // a padded sequence
            *reinterpret_cast<uint4*>(reinterpret_cast<unsigned char*>(a.out) + (row * a.dim + d) * 2) =
                make_uint4(pack2<T>(o[0], o[1]), pack2<T>(o[2], o[3]), pack2<T>(o[4], o[5]), pack2<T>(o[6], o[7]));
            if (d == 0 && a.lse) a.lse[row] = empty ? -INFINITY : (top + log2f(total)) * 0.69314718055994531f;
        } else {
            const long long at = (long long)part_index * n_tokens * n_heads + row;
            float4* to = reinterpret_cast<float4*>(a.part_out + at * a.dim + d);
            to[0] = make_float4(o[0], o[1], o[2], o[3]);
            to[1] = make_float4(o[4], o[5], o[6], o[7]);
            if (d == 0) a.part_lse[at] = empty ? -INFINITY : top + log2f(total);
        }
    }
}

// Joins the parts of every row: weights 2^(lse_p - max) / sum.  One warp per row.  A lane first looks after the weight of
// one part in 32; the outputs of the parts are then fetched U at a time, independently of one another (the parts come out of
// L2, so what counts is how many of its round trips follow one another).  A row of DP = 64 takes half a warp's lanes, so that
// two parts are fetched at once; heads of 256 take two vectors a lane.  Parts that saw no key are not read.
constexpr int kMergePartsThreads = 128;
template <typename T, int DP>
__global__ void __launch_bounds__(kMergePartsThreads) merge_parts_kernel(const AttendArgs a, const PrefixSplit split)
{
    constexpr int LANES = DP == 64 ? 16 : 32, VECS = DP == 256 ? 2 : 1, SIDE = 32 / LANES, U = 8 / VECS;
    const int lane = threadIdx.x & 31;
    const long long row = (long long)blockIdx.x * (kMergePartsThreads / 32) + (threadIdx.x >> 5);
    const int n_heads = a.kv_heads * a.group;
    const long long n_rows = (long long)a.n_seqs * a.q_len * n_heads;
    const int token = (int)((unsigned)row / (unsigned)n_heads), head = (int)(row - (long long)token * n_heads);
    int prefix_parts = a.prefix_parts;
    if (split.run > 0) {  // the prefix was dealt out by tiles: the row's unit has so many parts
        const int kv_head = head / a.group, block = (token * a.group + (head - kv_head * a.group)) / kTcBlockRows;
        prefix_parts = parts_of_unit(split, kv_head * split.blocks + block, block);
    }
    const int skip = a.prefix_parts - prefix_parts;  // parts of the workspace that this row does not use
    const int parts = prefix_parts + a.suffix_parts;
    wait_for_previous_kernel();
    if (row >= n_rows || __ldg(a.suffix_lens + (unsigned)token / (unsigned)a.q_len) < 0) return;
    const int side = lane / LANES, d = (lane % LANES) * 4;
    float m = -INFINITY, total = 0.f;
    float4 o[VECS];
#pragma unroll
    for (int v = 0; v < VECS; ++v) o[v] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int p0 = 0; p0 < parts; p0 += 32) {
        const int mine = p0 + lane;
        const int mine_at = mine < prefix_parts ? mine : mine + skip;
        const float lse = mine < parts ? a.part_lse[(long long)mine_at * n_rows + row] : -INFINITY;
        float top = fmaxf(m, lse);
#pragma unroll
        for (int s = 16; s >= 1; s >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, s));
        const float base = top == -INFINITY ? 0.f : top;
        // A NaN among the parts (a NaN score) is skipped by the maximum and kept by the weights.
        const float w = lse == -INFINITY ? 0.f : ex2(lse - base), keep = m == -INFINITY ? 0.f : ex2(m - base);
        float sum = w;
#pragma unroll
        for (int s = 16; s >= 1; s >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, s);
        total = total * keep + sum;
        m = top;
#pragma unroll
        for (int v = 0; v < VECS; ++v) { o[v].x *= keep; o[v].y *= keep; o[v].z *= keep; o[v].w *= keep; }
        const int here = min(32, parts - p0);
        for (int i0 = 0; i0 < here; i0 += U * SIDE) {
            float4 x[U][VECS];
            float wi[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = i0 + u * SIDE + side;
                wi[u] = __shfl_sync(0xFFFFFFFFu, w, i & 31);
                const bool there = i < here && wi[u] != 0.f;
                const int p = p0 + i;
                const float* from = a.part_out + ((long long)(p < prefix_parts ? p : p + skip) * n_rows + row) * a.dim + d;
#pragma unroll
                for (int v = 0; v < VECS; ++v) {
                    x[u][v] = make_float4(0.f, 0.f, 0.f, 0.f);
                    if (there && d + v * 128 < a.dim) x[u][v] = *reinterpret_cast<const float4*>(from + v * 128);
                }
                if (!there) wi[u] = 0.f;
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int v = 0; v < VECS; ++v) {
                    o[v].x = fmaf(wi[u], x[u][v].x, o[v].x); o[v].y = fmaf(wi[u], x[u][v].y, o[v].y);
                    o[v].z = fmaf(wi[u], x[u][v].z, o[v].z); o[v].w = fmaf(wi[u], x[u][v].w, o[v].w);
                }
        }
    }
    const bool empty = total == 0.f;  // a part that saw a key has a weight of 1, or NaN
    const float inv = empty ? 0.f : 1.0f / total;
#pragma unroll
    for (int v = 0; v < VECS; ++v) {
        if constexpr (SIDE == 2) {
            o[v].x += __shfl_xor_sync(0xFFFFFFFFu, o[v].x, 16); o[v].y += __shfl_xor_sync(0xFFFFFFFFu, o[v].y, 16);
            o[v].z += __shfl_xor_sync(0xFFFFFFFFu, o[v].z, 16); o[v].w += __shfl_xor_sync(0xFFFFFFFFu, o[v].w, 16);
        }
        if (side == 0 && d + v * 128 < a.dim)
            *reinterpret_cast<uint2*>(reinterpret_cast<unsigned char*>(a.out) + (row * a.dim + d + v * 128) * 2) =
                make_uint2(pack2<T>(o[v].x * inv, o[v].y * inv), pack2<T>(o[v].z * inv, o[v].w * inv));
    }
    if (lane == 0 && a.lse) a.lse[row] = empty ? -INFINITY : (m + log2f(total)) * 0.69314718055994531f;
}

}  // namespace rt
