// The paged key/value cache: entries quantised as they are written, and read back (sm_100a).
//
//   write:  amax = max(max_j |x_j|, 1e-12);  scale = amax / M;  code_j = rne(x_j * (M / amax))     per (token, head)
//   read:   x_j = round(code_j * scale)
//
// An entry is a vector of head_dim elements.  A group of LANES lanes (a power of two, at most a warp) holds one vector in
// registers, E elements to a lane and chunk, so that the largest magnitude is found with shuffles inside the group and
// the vector is touched once.  A CTA takes the 2 * kv_heads vectors (keys, then values) of a few consecutive tokens:
// neighbouring groups then read neighbouring heads of one token.
//
// Both kernels are bound by HBM at the large sizes and by one round of latency (slot, then vector, then store) at the
// small ones.  U vectors per group are loaded before the first is used.
#pragma once

#include <cuda_fp8.h>

#include "add_rmsnorm_kernel.cuh"

namespace rt {

constexpr int kDeviceIndexCode = 12;  // RT_ERR_INDEX, written to the status word
constexpr int kCacheThreads = 256;

enum { kKvPlain = 0, kKvE4m3 = 1, kKvInt8 = 2 };

struct CacheArgs {
    unsigned char* side[2];        // cache: k, v
    float* scale[2];               // k_scale, v_scale
    unsigned char* tokens[2];      // key and value of the tokens (read by the write kernel, written by the read kernel)
    long long token_stride[2];     // of key and value, in elements
    long long token_head_stride[2];
    const long long* slots;
    long long n_tokens;
    long long n_slots;
    long long page_stride, entry_stride, head_stride;  // of the cache, in elements
    long long scale_page_stride, scale_entry_stride, scale_head_stride;
    unsigned page_size;
    int page_shift;   // log2(page_size), or -1
    int heads;
    int dim;
    int tokens_per_cta;
    int* status;
};

struct SlotPlace {
    long long page;
    unsigned offset;
};
__device__ __forceinline__ SlotPlace place_of(long long slot, unsigned page_size, int page_shift)
{
    SlotPlace p;
    if (page_shift >= 0) {
        p.page = slot >> page_shift;
        p.offset = (unsigned)slot & (page_size - 1u);
    } else if (slot < (1LL << 32)) {
        const unsigned q = (unsigned)slot / page_size;
        p.page = q;
        p.offset = (unsigned)slot - q * page_size;
    } else {
        p.page = slot / page_size;
        p.offset = (unsigned)(slot - p.page * page_size);
    }
    return p;
}

// E consecutive elements of type T as 32-bit words (E * sizeof(T) is 1, 2, 4, 8, 16 or 32 bytes).
template <int BYTES>
struct Chunk {
    uint32_t w[(BYTES + 3) / 4];
};
template <int BYTES>
__device__ __forceinline__ Chunk<BYTES> ld_chunk(const unsigned char* p)
{
    Chunk<BYTES> c;
    if constexpr (BYTES == 1) {
        unsigned short h;
        asm volatile("ld.global.L1::no_allocate.u8 %0, [%1];" : "=h"(h) : "l"(p));
        c.w[0] = h;
    } else if constexpr (BYTES == 32) {  // two 16-byte accesses: rows of a cache are 16-byte aligned at best
        const Vec<16> a = ld_stream<16>(p), b = ld_stream<16>(p + 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) { c.w[i] = a.w[i]; c.w[4 + i] = b.w[i]; }
    } else {
        const Vec<BYTES> a = ld_stream<BYTES>(p);
#pragma unroll
        for (int i = 0; i < (BYTES + 3) / 4; ++i) c.w[i] = a.w[i];
    }
    return c;
}
template <int BYTES>
__device__ __forceinline__ void st_chunk(unsigned char* p, const Chunk<BYTES>& c)
{
    if constexpr (BYTES == 1) {
        asm volatile("st.global.u8 [%0], %1;" ::"l"(p), "h"((unsigned short)c.w[0]) : "memory");
    } else if constexpr (BYTES == 32) {
        Vec<16> a, b;
#pragma unroll
        for (int i = 0; i < 4; ++i) { a.w[i] = c.w[i]; b.w[i] = c.w[4 + i]; }
        st_stream<16>(p, a);
        st_stream<16>(p + 16, b);
    } else {
        Vec<BYTES> a;
#pragma unroll
        for (int i = 0; i < (BYTES + 3) / 4; ++i) a.w[i] = c.w[i];
        st_stream<BYTES>(p, a);
    }
}

template <typename T, int E>
__device__ __forceinline__ void chunk_to_float(const Chunk<E * (int)sizeof(T)>& c, float (&f)[E])
{
    using C = Codec<T, (E * (int)sizeof(T) > 32 ? 32 : E * (int)sizeof(T))>;
    Vec<E * (int)sizeof(T)> v;
#pragma unroll
    for (int i = 0; i < (E * (int)sizeof(T) + 3) / 4; ++i) v.w[i] = c.w[i];
    C::unpack(v, f);
}
template <typename T, int E>
__device__ __forceinline__ Chunk<E * (int)sizeof(T)> chunk_from_float(const float (&f)[E])
{
    using C = Codec<T, E * (int)sizeof(T)>;
    const Vec<E * (int)sizeof(T)> v = C::pack(f);
    Chunk<E * (int)sizeof(T)> c;
#pragma unroll
    for (int i = 0; i < (E * (int)sizeof(T) + 3) / 4; ++i) c.w[i] = v.w[i];
    return c;
}

// Magnitudes of E elements joined into `top` as bit patterns: patterns of non-negative floats order like the values, with
// infinity and then NaN on top, so an integer maximum propagates both.  16-bit types keep two running maxima in one
// word (joined by magnitude_of at the end).
template <typename T, int BYTES>
__device__ __forceinline__ uint32_t join_magnitude(uint32_t top, const Chunk<BYTES>& c)
{
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < BYTES / 4; ++i) top = max(top, c.w[i] & 0x7FFFFFFFu);
    } else {
#pragma unroll
        for (int i = 0; i < (BYTES + 3) / 4; ++i) top = __vmaxu2(top, c.w[i] & 0x7FFF7FFFu);
    }
    return top;
}
template <typename T>
__device__ __forceinline__ float magnitude_of(uint32_t top)
{
    if constexpr (sizeof(T) == 4) return __uint_as_float(top);
    else return Codec<T, 16>::to_float16(max(top & 0xFFFFu, top >> 16));
}

// E binary32 values to E codes.
template <int FMT, int E>
__device__ __forceinline__ Chunk<E> encode(const float (&f)[E], float inv)
{
    Chunk<E> c;
    if constexpr (FMT == kKvE4m3) {
        if constexpr (E == 1) {
            c.w[0] = __nv_cvt_float_to_fp8(f[0] * inv, __NV_SATFINITE, __NV_E4M3);
        } else {
#pragma unroll
            for (int i = 0; i < E; i += 4) {
                const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(f[i] * inv, f[i + 1] * inv), __NV_SATFINITE, __NV_E4M3);
                const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(f[i + 2] * inv, f[i + 3] * inv), __NV_SATFINITE, __NV_E4M3);
                c.w[i / 4] = lo | (hi << 16);
            }
        }
    } else {
        // |x * inv| <= 127 after rounding, so adding 1.5 * 2^23 leaves the nearest even integer in the low byte
        uint32_t b[E];
#pragma unroll
        for (int i = 0; i < E; ++i) b[i] = __float_as_uint(__fadd_rn(__fmul_rn(f[i], inv), 12582912.0f));
        if constexpr (E == 1) {
            c.w[0] = b[0] & 0xFFu;
        } else {
#pragma unroll
            for (int i = 0; i < E; i += 4)
                c.w[i / 4] = __byte_perm(__byte_perm(b[i], b[i + 1], 0x0040), __byte_perm(b[i + 2], b[i + 3], 0x0040), 0x5410);
        }
    }
    return c;
}
template <int FMT, int E>
__device__ __forceinline__ void decode(const Chunk<E>& c, float (&f)[E])
{
    if constexpr (FMT == kKvE4m3 && E % 2 == 0) {
#pragma unroll
        for (int i = 0; i < E; i += 2) {
            const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(c.w[i / 4] >> (8 * (i % 4))), __NV_E4M3);
            f[i] = __half2float(__half(__half_raw{h.x}));
            f[i + 1] = __half2float(__half(__half_raw{h.y}));
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const uint32_t b = (c.w[i / 4] >> (8 * (i % 4))) & 0xFFu;
        if constexpr (FMT == kKvE4m3) {
            const __half_raw h = __nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)b, __NV_E4M3);
            f[i] = __half2float(__half(h));
        } else {
            f[i] = (float)(signed char)b;
        }
    }
}

template <int FMT>
__device__ __forceinline__ constexpr float code_max()
{
    return FMT == kKvE4m3 ? 448.0f : 127.0f;
}

// Vector v of a CTA: v counts token, side, head.
struct CacheVector {
    bool live;
    int side, head, token;  // token: within the CTA
};
__device__ __forceinline__ CacheVector cache_vector(const CacheArgs& a, int v, int per_token, int n_vec)
{
    CacheVector c;
    c.live = v < n_vec;
    c.token = (int)((unsigned)(c.live ? v : 0) / (unsigned)per_token);
    const int in_token = (c.live ? v : 0) - c.token * per_token;
    c.side = in_token >= a.heads;
    c.head = in_token - (c.side ? a.heads : 0);
    return c;
}
// Where the entry and its scale lie; false: no such entry (padding, or a slot beyond the cache).
__device__ __forceinline__ bool cache_place(const CacheArgs& a, long long slot, int head, size_t& entry, size_t& scale_entry)
{
    if (slot >= a.n_slots) atomicExch(a.status, kDeviceIndexCode);
    if (slot < 0 || slot >= a.n_slots) return false;
    const SlotPlace p = place_of(slot, a.page_size, a.page_shift);
    entry = (size_t)p.page * a.page_stride + (size_t)p.offset * a.entry_stride + (size_t)head * a.head_stride;
    scale_entry = (size_t)p.page * a.scale_page_stride + (size_t)p.offset * a.scale_entry_stride + (size_t)head * a.scale_head_stride;
    return true;
}

// T: type of key and value.  E elements per lane and chunk, NCH chunks per lane, U vectors in flight per group.
// The key and value vectors do not depend on the slots, so both are fetched at once.  The two divisions of a vector are
// made by one lane for each of the U vectors at a time, not by all lanes for all of them: they are correctly rounded ones
// (the codes are the definition's bit for bit) and cost as much as the rest of a vector.
template <typename T, int FMT, int E, int LANES, int NCH, int U>
__global__ void __launch_bounds__(kCacheThreads) kv_cache_write_kernel(const CacheArgs a)
{
    constexpr int IN = E * (int)sizeof(T);
    static_assert(U <= LANES, "a lane for every vector in flight");
    const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
    constexpr int GROUPS = kCacheThreads / LANES;
    const int per_token = 2 * a.heads;
    const long long first = (long long)blockIdx.x * a.tokens_per_cta;
    const int n_vec = (int)min((long long)a.tokens_per_cta, a.n_tokens - first) * per_token;
    wait_for_previous_kernel();
    for (int v0 = 0; v0 < n_vec; v0 += GROUPS * U) {  // uniform over the CTA: whole warps take part in the shuffles
        Chunk<IN> x[U][NCH];
        long long slot[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const CacheVector c = cache_vector(a, v0 + u * GROUPS + group, per_token, n_vec);
            slot[u] = c.live ? __ldg(a.slots + first + c.token) : -1;
            const unsigned char* src = a.tokens[c.side] +
                ((size_t)(first + c.token) * a.token_stride[c.side] + (size_t)c.head * a.token_head_stride[c.side]) * sizeof(T);
#pragma unroll
            for (int i = 0; i < NCH; ++i) {
                const int e = (i * LANES + lane) * E;
                if (c.live && e < a.dim) {
                    x[u][i] = ld_chunk<IN>(src + (size_t)e * sizeof(T));
                } else {
#pragma unroll
                    for (int k = 0; k < (IN + 3) / 4; ++k) x[u][i].w[k] = 0;
                }
            }
        }
        float my_inv = 0.f, my_scale = 0.f;  // of the vector that this lane divides for: lane % U
        if constexpr (FMT != kKvPlain) {
            uint32_t my_top = 0;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                uint32_t top = 0;
#pragma unroll
                for (int i = 0; i < NCH; ++i) top = join_magnitude<T, IN>(top, x[u][i]);
#pragma unroll
                for (int m = LANES / 2; m >= 1; m >>= 1) {
                    const uint32_t other = __shfl_xor_sync(0xFFFFFFFFu, top, m);
                    if constexpr (sizeof(T) == 4) top = max(top, other);
                    else top = __vmaxu2(top, other);
                }
                if (u == 0 || lane % U == u) my_top = top;
            }
            float amax = magnitude_of<T>(my_top);
            amax = amax < 1e-12f ? 1e-12f : amax;  // keeps a NaN
            my_inv = __fdiv_rn(code_max<FMT>(), amax);
            my_scale = __fdiv_rn(amax, code_max<FMT>());
            if (!(amax < INFINITY)) my_scale = __uint_as_float(0x7FC00000u);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const CacheVector c = cache_vector(a, v0 + u * GROUPS + group, per_token, n_vec);
            const int from = (threadIdx.x & 31) - lane + u;  // lane u of this group
            const float inv = __shfl_sync(0xFFFFFFFFu, my_inv, from), scale = __shfl_sync(0xFFFFFFFFu, my_scale, from);
            size_t entry, scale_entry;
            if (!cache_place(a, slot[u], c.head, entry, scale_entry)) continue;
            if constexpr (FMT == kKvPlain) {
                unsigned char* dst = a.side[c.side] + entry * sizeof(T);
#pragma unroll
                for (int i = 0; i < NCH; ++i) {
                    const int e = (i * LANES + lane) * E;
                    if (e < a.dim) st_chunk<IN>(dst + (size_t)e * sizeof(T), x[u][i]);
                }
            } else {
                unsigned char* dst = a.side[c.side] + entry;
#pragma unroll
                for (int i = 0; i < NCH; ++i) {
                    const int e = (i * LANES + lane) * E;
                    if (e < a.dim) {
                        float f[E];
                        chunk_to_float<T, E>(x[u][i], f);
                        st_chunk<E>(dst + e, encode<FMT, E>(f, inv));
                    }
                }
                if (lane == 0) a.scale[c.side][scale_entry] = scale;
            }
        }
    }
}

template <typename T, int FMT, int E, int LANES, int NCH, int U>
__global__ void __launch_bounds__(kCacheThreads) kv_cache_read_kernel(const CacheArgs a)
{
    constexpr int OUT = E * (int)sizeof(T);
    constexpr int HELD = FMT == kKvPlain ? OUT : E;
    constexpr int HELD_SIZE = FMT == kKvPlain ? (int)sizeof(T) : 1;
    const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
    constexpr int GROUPS = kCacheThreads / LANES;
    const int per_token = 2 * a.heads;
    const long long first = (long long)blockIdx.x * a.tokens_per_cta;
    const int n_vec = (int)min((long long)a.tokens_per_cta, a.n_tokens - first) * per_token;
    wait_for_previous_kernel();
    for (int v0 = 0; v0 < n_vec; v0 += GROUPS * U) {
        Chunk<HELD> x[U][NCH];
        float scale[U];
        long long slot[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const CacheVector c = cache_vector(a, v0 + u * GROUPS + group, per_token, n_vec);
            slot[u] = c.live ? __ldg(a.slots + first + c.token) : -1;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const CacheVector c = cache_vector(a, v0 + u * GROUPS + group, per_token, n_vec);
            size_t entry, scale_entry;
            scale[u] = 0.f;
            if (!cache_place(a, slot[u], c.head, entry, scale_entry)) {
                slot[u] = -1;
                continue;
            }
            const unsigned char* src = a.side[c.side] + entry * HELD_SIZE;
            if (FMT != kKvPlain) scale[u] = __ldg(a.scale[c.side] + scale_entry);
#pragma unroll
            for (int i = 0; i < NCH; ++i) {
                const int e = (i * LANES + lane) * E;
                if (e < a.dim) x[u][i] = ld_chunk<HELD>(src + (size_t)e * HELD_SIZE);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (slot[u] < 0) continue;
            const CacheVector c = cache_vector(a, v0 + u * GROUPS + group, per_token, n_vec);
            unsigned char* dst = a.tokens[c.side] +
                ((size_t)(first + c.token) * a.token_stride[c.side] + (size_t)c.head * a.token_head_stride[c.side]) * sizeof(T);
#pragma unroll
            for (int i = 0; i < NCH; ++i) {
                const int e = (i * LANES + lane) * E;
                if (e >= a.dim) continue;
                if constexpr (FMT == kKvPlain) {
                    st_chunk<OUT>(dst + (size_t)e * sizeof(T), x[u][i]);
                } else {
                    float f[E];
                    decode<FMT, E>(x[u][i], f);
#pragma unroll
                    for (int k = 0; k < E; ++k) f[k] = __fmul_rn(f[k], scale[u]);
                    st_chunk<OUT>(dst + (size_t)e * sizeof(T), chunk_from_float<T, E>(f));
                }
            }
        }
    }
}

}  // namespace rt
