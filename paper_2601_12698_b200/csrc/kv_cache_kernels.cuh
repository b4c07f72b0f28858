// The paged key/value cache: entries quantised as they are written, and read back (sm_100a).
//
//   write:  amax = max(max_j |x_j|, 1e-12);  scale = amax / M;  code_j = rne(x_j * (M / amax))     per (token, head)
//   read:   x_j = round(code_j * scale)
//
// An entry is a vector of head_dim elements.  A group of LANES lanes (a power of two, at most a warp) holds one vector in
// registers, E elements to a lane, so that the largest magnitude is found with shuffles inside the group and
// the vector is touched once.  A CTA takes the 2 * kv_heads vectors (keys, then values) of a few consecutive tokens:
// neighbouring groups then read neighbouring heads of one token.
//
// The large sizes want HBM's time and come near it once little is done per element: with 8 elements to a lane, 64-bit products for
// every place and conversions one at a time, the write kernel issued 26.6 M warp instructions for 16384 tokens x 8 heads of
// 128 (0.79 a cycle and scheduler) and took 30 us; with 16 elements to a lane, places in 32-bit factors and packed products and
// conversions it takes 19.6 us (write) and 19.8 us (read) when repeated on the same tensors, 22.3 and 22.1 us on tensors that
// have left L2: 102 MB at 4.6 TB/s, 0.70 of the measured copy bandwidth.  The small ones take one round of latency (slot, then
// vector, then store): 1.8 us a launch in a graph for 64 tokens.  U vectors per group are loaded before the first is used.
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
    int vec_shift;    // log2(2 * heads), or -1
    int heads;
    int dim;
    int tokens_per_cta;
    int* status;
};

struct SlotPlace {
    unsigned page, offset;  // the host checked that there are fewer than 2^31 pages
};
__device__ __forceinline__ SlotPlace place_of(long long slot, unsigned page_size, int page_shift)
{
    SlotPlace p;
    if (page_shift >= 0) {
        p.page = (unsigned)(slot >> page_shift);
        p.offset = (unsigned)slot & (page_size - 1u);
    } else if (slot < (1LL << 32)) {
        p.page = (unsigned)slot / page_size;
        p.offset = (unsigned)slot - p.page * page_size;
    } else {
        p.page = (unsigned)(slot / page_size);
        p.offset = (unsigned)(slot - (long long)p.page * page_size);
    }
    return p;
}
// index * stride: two multiplications, not the three or four of a 64-bit product.
__device__ __forceinline__ size_t times(unsigned index, long long stride) { return (size_t)index * (size_t)stride; }

// Consecutive elements as 32-bit words.
template <int BYTES>
struct Chunk {
    uint32_t w[BYTES / 4];
};
// Bytes of one access to a chunk of E elements whose places are multiples of AL elements of `size` bytes, and from one access to
// the next: where AL elements are less than a chunk, neighbouring accesses are those of neighbouring lanes.
__host__ __device__ constexpr int access_bytes(int al, int size) { return al * size < 16 ? al * size : 16; }
__host__ __device__ constexpr int access_stride(int al, int e, int size, int lanes) { return al < e ? lanes * al * size : access_bytes(al, size); }
// A chunk in accesses of ACCESS bytes, STRIDE bytes apart.  RAGGED: accesses from byte `there` on do not exist, they read as zero.
template <int BYTES, int ACCESS, int STRIDE, bool RAGGED>
__device__ __forceinline__ Chunk<BYTES> ld_chunk(const unsigned char* p, int there)
{
    Chunk<BYTES> c;
    if constexpr (ACCESS < 4) {  // lanes and accesses share sectors: these loads go through L1
#pragma unroll
        for (int k = 0; k < BYTES / ACCESS; ++k) {
            uint32_t x = 0;
            if (k * STRIDE < there) {
                if constexpr (ACCESS == 1) x = *(p + STRIDE * k);
                else x = *reinterpret_cast<const unsigned short*>(p + STRIDE * k);
            }
            constexpr int PER = 4 / ACCESS;
            c.w[k / PER] = k % PER == 0 ? x : c.w[k / PER] | x << (k % PER * 8 * ACCESS);
        }
    } else {
        constexpr int WORDS = ACCESS / 4;
#pragma unroll
        for (int k = 0; k < BYTES / ACCESS; ++k) {
            Vec<ACCESS> a;
#pragma unroll
            for (int i = 0; i < WORDS; ++i) a.w[i] = 0;
            if (!RAGGED || k * STRIDE < there) a = ld_stream<ACCESS>(p + STRIDE * k);
#pragma unroll
            for (int i = 0; i < WORDS; ++i) c.w[WORDS * k + i] = a.w[i];
        }
    }
    return c;
}
template <int BYTES, int ACCESS, int STRIDE, bool RAGGED>
__device__ __forceinline__ void st_chunk(unsigned char* p, const Chunk<BYTES>& c, int there)
{
    if constexpr (ACCESS < 4) {
#pragma unroll
        for (int k = 0; k < BYTES / ACCESS; ++k) {
            constexpr int PER = 4 / ACCESS;
            const uint32_t x = c.w[k / PER] >> (k % PER * 8 * ACCESS);
            if (k * STRIDE < there) {
                if constexpr (ACCESS == 1) *(p + STRIDE * k) = (unsigned char)x;
                else *reinterpret_cast<unsigned short*>(p + STRIDE * k) = (unsigned short)x;
            }
        }
    } else {
        constexpr int WORDS = ACCESS / 4;
#pragma unroll
        for (int k = 0; k < BYTES / ACCESS; ++k) {
            Vec<ACCESS> a;
#pragma unroll
            for (int i = 0; i < WORDS; ++i) a.w[i] = c.w[WORDS * k + i];
            if (!RAGGED || k * STRIDE < there) st_stream<ACCESS>(p + STRIDE * k, a);
        }
    }
}

template <typename T, int E>
__device__ __forceinline__ void chunk_to_float(const Chunk<E * (int)sizeof(T)>& c, float (&f)[E])
{
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < E; ++i) f[i] = __uint_as_float(c.w[i]);
    } else if constexpr (std::is_same<T, __nv_bfloat16>::value) {
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
            f[2 * i] = __uint_as_float(c.w[i] << 16);
            f[2 * i + 1] = __uint_as_float(c.w[i] & 0xFFFF0000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
            const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&c.w[i]));
            f[2 * i] = x.x;
            f[2 * i + 1] = x.y;
        }
    }
}
template <typename T, int E>
__device__ __forceinline__ Chunk<E * (int)sizeof(T)> chunk_from_float(const float (&f)[E])
{
    Chunk<E * (int)sizeof(T)> c;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < E; ++i) c.w[i] = __float_as_uint(f[i]);
    } else {
#pragma unroll
        for (int i = 0; i < E / 2; ++i) c.w[i] = Codec<T, 16>::from_float16x2(f[2 * i], f[2 * i + 1]);
    }
    return c;
}

__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// Magnitudes of E elements joined into `top` as bit patterns: patterns of non-negative floats order like the values, with
// infinity and then NaN on top, so an integer maximum propagates both.  16-bit types keep two running maxima in one
// word (joined by magnitude_of at the end).
template <typename T, int BYTES>
__device__ __forceinline__ uint32_t join_magnitude(const Chunk<BYTES>& c)
{
    uint32_t top = 0;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < BYTES / 4; ++i) top = max(top, c.w[i] & 0x7FFFFFFFu);
    } else {
#pragma unroll
        for (int i = 0; i < BYTES / 4; ++i) top = max_u16x2(top, c.w[i] & 0x7FFF7FFFu);
    }
    return top;
}
template <typename T>
__device__ __forceinline__ float magnitude_of(uint32_t top)
{
    if constexpr (sizeof(T) == 4) return __uint_as_float(top);
    else return Codec<T, 16>::to_float16(max(top & 0xFFFFu, top >> 16));
}

// Two binary32 numbers in one register pair: the packed operations of sm_100 do both at once, each correctly rounded.
typedef unsigned long long float2x;
__device__ __forceinline__ float2x pack_f2(float lo, float hi)
{
    float2x r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void unpack_f2(float2x x, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(x)); }
__device__ __forceinline__ float2x fma_f2(float2x a, float2x b, float2x c)
{
    float2x r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ float2x mul_f2(float2x a, float2x b)
{
    float2x r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ float2x add_f2(float2x a, float2x b)
{
    float2x r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// E binary32 values to E codes.
template <int FMT, int E>
__device__ __forceinline__ Chunk<E> encode(const float (&f)[E], float inv)
{
    Chunk<E> c;
    const float2x inv2 = pack_f2(inv, inv);
#pragma unroll
    for (int i = 0; i < E; i += 4) {
        float x[4];
        float2x a = mul_f2(pack_f2(f[i], f[i + 1]), inv2), b = mul_f2(pack_f2(f[i + 2], f[i + 3]), inv2);
        if constexpr (FMT == kKvE4m3) {
            unpack_f2(a, x[0], x[1]);
            unpack_f2(b, x[2], x[3]);
            asm("{\n\t.reg .b16 lo, hi;\n\tcvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n\tmov.b32 %0, {lo, hi};\n\t}"
                : "=r"(c.w[i / 4]) : "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]));
        } else {
            // |x * inv| <= 127 after rounding, so adding 1.5 * 2^23 leaves the nearest even integer in the low byte
            // (added one by one: a packed addition behind a packed product came out as one rounding, not two)
            unpack_f2(a, x[0], x[1]);
            unpack_f2(b, x[2], x[3]);
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = __fadd_rn(x[k], 12582912.0f);
            c.w[i / 4] = __byte_perm(__byte_perm(__float_as_uint(x[0]), __float_as_uint(x[1]), 0x0040),
                                     __byte_perm(__float_as_uint(x[2]), __float_as_uint(x[3]), 0x0040), 0x5410);
        }
    }
    return c;
}
// E codes times the scale.
template <int FMT, int E>
__device__ __forceinline__ void decode(const Chunk<E>& c, float scale, float (&f)[E])
{
    const float2x scale2 = pack_f2(scale, scale);
#pragma unroll
    for (int i = 0; i < E; i += 4) {
        float x[4];
        if constexpr (FMT == kKvE4m3) {
            uint32_t lo, hi;
            asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
                : "=r"(lo), "=r"(hi) : "r"(c.w[i / 4]));
            const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&lo)), q = __half22float2(*reinterpret_cast<const __half2*>(&hi));
            x[0] = p.x; x[1] = p.y; x[2] = q.x; x[3] = q.y;
        } else {
            // 2^23 + (code + 128) as binary32 bits, minus 2^23 + 128: exact
            const uint32_t w = c.w[i / 4] ^ 0x80808080u;
            x[0] = __uint_as_float(__byte_perm(w, 0x4B000000u, 0x7650)) - 8388736.0f;
            x[1] = __uint_as_float(__byte_perm(w, 0x4B000000u, 0x7651)) - 8388736.0f;
            x[2] = __uint_as_float(__byte_perm(w, 0x4B000000u, 0x7652)) - 8388736.0f;
            x[3] = __uint_as_float(__byte_perm(w, 0x4B000000u, 0x7653)) - 8388736.0f;
        }
        unpack_f2(mul_f2(pack_f2(x[0], x[1]), scale2), f[i], f[i + 1]);
        unpack_f2(mul_f2(pack_f2(x[2], x[3]), scale2), f[i + 2], f[i + 3]);
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
    unsigned side, head, token;  // token: within the CTA
};
__device__ __forceinline__ CacheVector cache_vector(const CacheArgs& a, unsigned v, unsigned n_vec)
{
    CacheVector c;
    c.live = v < n_vec;
    v = c.live ? v : 0;
    const unsigned heads = (unsigned)a.heads;
    c.token = a.vec_shift >= 0 ? v >> a.vec_shift : v / (2 * heads);
    const unsigned in_token = v - c.token * 2 * heads;
    c.side = in_token >= heads;
    c.head = in_token - (c.side ? heads : 0);
    return c;
}
__device__ __forceinline__ unsigned char* token_vector(const CacheArgs& a, const CacheVector& c, long long first, int size)
{
    const long long ts = c.side ? a.token_stride[1] : a.token_stride[0], hs = c.side ? a.token_head_stride[1] : a.token_head_stride[0];
    return (c.side ? a.tokens[1] : a.tokens[0]) + ((size_t)(first * ts) + times(c.token, ts) + times(c.head, hs)) * size;
}
// Where the entry and its scale lie; false: no such entry (padding, or a slot beyond the cache).
__device__ __forceinline__ bool cache_place(const CacheArgs& a, long long slot, unsigned head, size_t& entry, size_t& scale_entry)
{
    if (slot >= a.n_slots) atomicExch(a.status, kDeviceIndexCode);
    if (slot < 0 || slot >= a.n_slots) return false;
    const SlotPlace p = place_of(slot, a.page_size, a.page_shift);
    entry = times(p.page, a.page_stride) + times(p.offset, a.entry_stride) + times(head, a.head_stride);
    scale_entry = times(p.page, a.scale_page_stride) + times(p.offset, a.scale_entry_stride) + times(head, a.scale_head_stride);
    return true;
}

// T: type of key and value.  E elements to a lane, AL of them to an access, U vectors in flight per group.
// The key and value vectors do not depend on the slots, so both are fetched at once.  The two divisions of a vector are
// made by one lane for each of the U vectors at a time, not by all lanes for all of them: they are correctly rounded ones
// (the codes are the definition's bit for bit) and cost as much as the rest of a vector.
template <typename T, int FMT, int E, int AL, int LANES, int U>
__global__ void __launch_bounds__(kCacheThreads) kv_cache_write_kernel(const CacheArgs a)
{
    constexpr int IN = E * (int)sizeof(T), SIZE = (int)sizeof(T), CODE = FMT == kKvPlain ? SIZE : 1;
    constexpr bool RAGGED = AL < E;
    static_assert(AL == E || AL * SIZE <= 16, "AL elements are one access");
    static_assert(U <= LANES, "a lane for every vector in flight");
    const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES, e = lane * (AL < E ? AL : E);
    constexpr int GROUPS = kCacheThreads / LANES;
    const long long first = (long long)blockIdx.x * a.tokens_per_cta;
    const unsigned n_vec = (unsigned)min((long long)a.tokens_per_cta, a.n_tokens - first) * 2u * (unsigned)a.heads;
    wait_for_previous_kernel();
    for (unsigned v0 = 0; v0 < n_vec; v0 += GROUPS * U) {  // uniform over the CTA: whole warps take part in the shuffles
        Chunk<IN> x[U];
        long long slot[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const CacheVector c = cache_vector(a, v0 + u * GROUPS + group, n_vec);
            slot[u] = c.live ? __ldg(a.slots + first + c.token) : -1;
            const unsigned char* src = token_vector(a, c, first, sizeof(T));
            if (c.live && e < a.dim) {
                x[u] = ld_chunk<IN, access_bytes(AL, SIZE), access_stride(AL, E, SIZE, LANES), RAGGED>(src + (size_t)e * SIZE, (a.dim - e) * SIZE);
            } else {
#pragma unroll
                for (int k = 0; k < IN / 4; ++k) x[u].w[k] = 0;
            }
        }
        float my_inv = 0.f, my_scale = 0.f;  // of the vector that this lane divides for: lane % U
        if constexpr (FMT != kKvPlain) {
            uint32_t my_top = 0;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                uint32_t top = join_magnitude<T, IN>(x[u]);
#pragma unroll
                for (int m = LANES / 2; m >= 1; m >>= 1) {
                    const uint32_t other = __shfl_xor_sync(0xFFFFFFFFu, top, m);
                    if constexpr (sizeof(T) == 4) top = max(top, other);
                    else top = max_u16x2(top, other);
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
            const CacheVector c = cache_vector(a, v0 + u * GROUPS + group, n_vec);
            const int from = (threadIdx.x & 31) - lane + u;  // lane u of this group
            const float inv = __shfl_sync(0xFFFFFFFFu, my_inv, from), scale = __shfl_sync(0xFFFFFFFFu, my_scale, from);
            size_t entry, scale_entry;
            if (!cache_place(a, slot[u], c.head, entry, scale_entry)) continue;
            if constexpr (FMT == kKvPlain) {
                unsigned char* dst = (c.side ? a.side[1] : a.side[0]) + entry * sizeof(T);
                if (e < a.dim) st_chunk<IN, access_bytes(AL, SIZE), access_stride(AL, E, SIZE, LANES), RAGGED>(dst + (size_t)e * SIZE, x[u], (a.dim - e) * SIZE);
            } else {
                unsigned char* dst = (c.side ? a.side[1] : a.side[0]) + entry;
                if (e < a.dim) {
                    float f[E];
                    chunk_to_float<T, E>(x[u], f);
                    st_chunk<E, access_bytes(AL, CODE), access_stride(AL, E, CODE, LANES), RAGGED>(dst + e, encode<FMT, E>(f, inv), a.dim - e);
                }
                if (lane == 0) (c.side ? a.scale[1] : a.scale[0])[scale_entry] = scale;
            }
        }
    }
}

template <typename T, int FMT, int E, int AL, int LANES, int U>
__global__ void __launch_bounds__(kCacheThreads) kv_cache_read_kernel(const CacheArgs a)
{
    constexpr int OUT = E * (int)sizeof(T), SIZE = (int)sizeof(T);
    constexpr bool RAGGED = AL < E;
    static_assert(AL == E || AL * SIZE <= 16, "AL elements are one access");
    constexpr int HELD = FMT == kKvPlain ? OUT : E;
    constexpr int HELD_SIZE = FMT == kKvPlain ? (int)sizeof(T) : 1;
    const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES, e = lane * (AL < E ? AL : E);
    constexpr int GROUPS = kCacheThreads / LANES;
    const long long first = (long long)blockIdx.x * a.tokens_per_cta;
    const unsigned n_vec = (unsigned)min((long long)a.tokens_per_cta, a.n_tokens - first) * 2u * (unsigned)a.heads;
    wait_for_previous_kernel();
    for (unsigned v0 = 0; v0 < n_vec; v0 += GROUPS * U) {
        Chunk<HELD> x[U];
        float scale[U];
        long long slot[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const CacheVector c = cache_vector(a, v0 + u * GROUPS + group, n_vec);
            slot[u] = c.live ? __ldg(a.slots + first + c.token) : -1;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const CacheVector c = cache_vector(a, v0 + u * GROUPS + group, n_vec);
            size_t entry, scale_entry;
            scale[u] = 0.f;
            if (!cache_place(a, slot[u], c.head, entry, scale_entry)) {
                slot[u] = -1;
                continue;
            }
            const unsigned char* src = (c.side ? a.side[1] : a.side[0]) + entry * HELD_SIZE;
            if (FMT != kKvPlain) scale[u] = __ldg((c.side ? a.scale[1] : a.scale[0]) + scale_entry);
            if (e < a.dim) x[u] = ld_chunk<HELD, access_bytes(AL, HELD_SIZE), access_stride(AL, E, HELD_SIZE, LANES), RAGGED>(src + (size_t)e * HELD_SIZE, (a.dim - e) * HELD_SIZE);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (slot[u] < 0) continue;
            const CacheVector c = cache_vector(a, v0 + u * GROUPS + group, n_vec);
            unsigned char* dst = token_vector(a, c, first, sizeof(T));
            if (e >= a.dim) continue;
            if constexpr (FMT == kKvPlain) {
                st_chunk<OUT, access_bytes(AL, SIZE), access_stride(AL, E, SIZE, LANES), RAGGED>(dst + (size_t)e * SIZE, x[u], (a.dim - e) * SIZE);
            } else {
                float f[E];
                decode<FMT, E>(x[u], scale[u], f);
                st_chunk<OUT, access_bytes(AL, SIZE), access_stride(AL, E, SIZE, LANES), RAGGED>(dst + (size_t)e * SIZE, chunk_from_float<T, E>(f), (a.dim - e) * SIZE);
            }
        }
    }
}

}  // namespace rt
