// What the attention kernels over a paged key/value cache share: arguments, places in the cache, codes, exponentials.
#pragma once

#include <cuda_fp8.h>

#include "add_rmsnorm_kernel.cuh"
#include "kv_cache_kernels.cuh"

namespace rt {

// One call of shared_prefix_attention_launch.  A "row" is one query head of one query token; the rows of one key/value
// head (all its query heads of all query tokens) attend to the same keys of the prefix.  Every key range that one CTA works
// through is a "part": it leaves a normalised output and the base-2 logarithm of its softmax denominator, and
// merge_parts_kernel joins the parts of a row.  Parts 0 .. prefix_parts-1 belong to the prefix, the rest to the suffix.
struct AttendArgs {
    const unsigned char* k;
    const unsigned char* v;
    const float* k_scale;
    const float* v_scale;
    long long page_stride, token_stride, head_stride;  // of the cache, in elements (bytes when quantised)
    long long scale_page_stride, scale_token_stride, scale_head_stride;
    long long n_pages;
    unsigned page_size;
    int page_shift;  // log2(page_size), or -1
    const int32_t* prefix_pages;
    const int32_t* page_table;
    const int32_t* suffix_lens;
    long long page_table_stride;
    int page_table_width;
    int prefix_len;
    int max_suffix_len;
    int n_seqs;
    int q_len;
    int kv_heads;
    int group;  // query heads per key/value head
    int dim;
    const unsigned char* q;
    long long q_token_stride, q_head_stride;  // elements
    float score_scale;                        // softmax_scale * log2(e)
    int prefix_parts, prefix_keys;            // parts of the prefix and keys in each (the last may have fewer)
    int suffix_parts, suffix_keys;
    int before_suffix;  // for the prefix kernel: the suffix kernel is launched behind it
    int after_prefix;   // for the suffix kernel: it runs beside that prefix kernel
    float* part_out;  // [part][token][head][dim]
    float* part_lse;  // [part][token][head]
    void* out;        // [token][head][dim]
    float* lse;       // [token][head] or NULL
    int* status;
    unsigned wait_polls;  // polls a bounded wait may take (kMbarrierPollLimit unless the caller lowered it)
    int drop_copies;      // diagnostic: 1 = no tile is announced, so that waits run out and report it
};

// The prefix kernel lets the suffix kernel start once all its own CTAs have started and the kernel before both has completed: they
// read the same inputs and write different parts.  (With more CTAs than SMs that is its last wave.)  The suffix kernel therefore does not wait for its predecessor before it starts; its first CTA does
// before it ends, so that the kernel that joins the parts, which waits for the suffix kernel, finds the prefix's parts too.  (One
// CTA is enough, and CTAs that waited would keep others from the SMs that they hold.)
__device__ __forceinline__ void let_next_kernel_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// Offset of token `pos` of a page list in k and v (`scales`: in the scale tensors), -1 when its page is not in the cache.
__device__ __forceinline__ long long entry_offset(const AttendArgs& a, int page, unsigned in_page, int head, bool scales)
{
    if (scales) return (long long)page * a.scale_page_stride + (long long)in_page * a.scale_token_stride + (long long)head * a.scale_head_stride;
    return (long long)page * a.page_stride + (long long)in_page * a.token_stride + (long long)head * a.head_stride;
}
__device__ __forceinline__ void split_position(const AttendArgs& a, int pos, int& list_index, unsigned& in_page)
{
    if (a.page_shift >= 0) {
        list_index = pos >> a.page_shift;
        in_page = (unsigned)pos & (a.page_size - 1u);
    } else {
        list_index = (int)((unsigned)pos / a.page_size);
        in_page = (unsigned)pos - (unsigned)list_index * a.page_size;
    }
}

// Number of keys in the suffix of `seq` that the page table can name; below 0 for a padded sequence.  A longer one is reported by every
// kernel that asks: there may be no suffix kernel.
__device__ __forceinline__ int suffix_length(const AttendArgs& a, int seq)
{
    int len = __ldg(a.suffix_lens + seq);
    if (len > a.max_suffix_len) {
        atomicExch(a.status, kDeviceIndexCode);
        len = a.max_suffix_len;
    }
    return len;
}

template <typename T>
__device__ __forceinline__ uint32_t pack2(float lo, float hi)
{
    return Codec<T, 16>::from_float16x2(lo, hi);
}

// 2^x, 2 ulp; results below 2^-126 are zero.
__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Two e4m3 codes as two fp16 values.  Both formats fit fp16 exactly.
__device__ __forceinline__ uint32_t e4m3_to_half2(uint32_t low_bytes)
{
    uint32_t h;
    asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;\n\t}" : "=r"(h) : "r"(low_bytes));
    return h;
}
__device__ __forceinline__ uint32_t e4m3_high_to_half2(uint32_t word)
{
    uint32_t h;
    asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, hi;\n\t}" : "=r"(h) : "r"(word));
    return h;
}
// Four codes as four fp16 values.
template <int FMT>
__device__ __forceinline__ void codes_to_half4(uint32_t w, uint32_t& lo, uint32_t& hi)
{
    if constexpr (FMT == kKvE4m3) {
        lo = e4m3_to_half2(w);
        hi = e4m3_high_to_half2(w);
    } else {
        // 1024 + (code + 128) as fp16 bits, minus 1152: exact for -128 .. 127
        const __half2 bias = __half2half2(__ushort_as_half((unsigned short)0x6480));
        const uint32_t x = w ^ 0x80808080u, a = __byte_perm(x, 0x64646464u, 0x4140), b = __byte_perm(x, 0x64646464u, 0x4342);
        const __half2 p = __hsub2(*reinterpret_cast<const __half2*>(&a), bias), q = __hsub2(*reinterpret_cast<const __half2*>(&b), bias);
        lo = *reinterpret_cast<const uint32_t*>(&p);
        hi = *reinterpret_cast<const uint32_t*>(&q);
    }
}
// 16 codes of a tile that is read once, or zeros.  The zeros are set ahead of a predicated load, inside one statement: written
// as a branch, the registers of both sides meet in a move that waits for the load.
__device__ __forceinline__ uint4 ld_codes(const unsigned char* p, bool there)
{
    uint4 w;
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %5, 0;\n\tmov.u32 %0, 0;\n\tmov.u32 %1, 0;\n\tmov.u32 %2, 0;\n\tmov.u32 %3, 0;\n\t"
                 "@p ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];\n\t}"
                 : "=&r"(w.x), "=&r"(w.y), "=&r"(w.z), "=&r"(w.w) : "l"(p), "r"((uint32_t)there));
    return w;
}

// 2^x for two numbers on the multiply-add pipe, beside the special function unit (16 exponentials a cycle per SM): x = n + f with
// n the nearest integer, 2^f by the polynomial of degree 4 of least relative error on [-1/2, 1/2] (found by exchange of the extrema; 2.7e-6 in binary32, 4e-8 on average), times 2^n.  Below -126: 2^-126.
__device__ __forceinline__ float2x ex2_by_polynomial(float2x x)
{
    float lo, hi;
    unpack_f2(x, lo, hi);
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(lo) : "f"(lo), "f"(-126.f));
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(hi) : "f"(hi), "f"(-126.f));
    x = pack_f2(lo, hi);
    const float2x magic = pack_f2(12582912.f, 12582912.f), minus_magic = pack_f2(-12582912.f, -12582912.f), minus_one = pack_f2(-1.f, -1.f);
    const float2x y = add_f2(x, magic);  // n in the low bits
    const float2x f = fma_f2(add_f2(y, minus_magic), minus_one, x);
    float2x p = pack_f2(0.009570102207362652f, 0.009570102207362652f);
    p = fma_f2(p, f, pack_f2(0.05591785907745361f, 0.05591785907745361f));
    p = fma_f2(p, f, pack_f2(0.240247443318367f, 0.240247443318367f));
    p = fma_f2(p, f, pack_f2(0.6931217908859253f, 0.6931217908859253f));
    p = fma_f2(p, f, pack_f2(0.9999992847442627f, 0.9999992847442627f));
    unpack_f2(y, lo, hi);
    return mul_f2(p, pack_f2(__uint_as_float(__float_as_uint(lo) * (1u << 23) + 0x3F800000u), __uint_as_float(__float_as_uint(hi) * (1u << 23) + 0x3F800000u)));
}

// The power of two that brings a row's largest magnitude into [2^14, 2^15), so that a bf16 row fits fp16 without loss
// (elements 2^-28 below the largest lose bits, which no binary32 sum would keep either).  Its inverse is exact too.
__device__ __forceinline__ float fp16_row_factor(float amax)
{
    if (!(amax < INFINITY) || amax == 0.f) return 1.0f;
    int e = (int)((__float_as_uint(amax) >> 23) & 0xFFu) - 127;
    e = max(e, -112);
    return __uint_as_float((uint32_t)(127 + 14 - e) << 23);
}

// A value scale as the weights use it: log2 and reciprocal are taken of it, so a zero (an entry never written) becomes tiny, and one
// that is not finite 1: the log-sum-exp, which values have no part in, stays that of the scores, and the rows that see such a key
// are made NaN when they are written.
__device__ __forceinline__ bool finite_scale(float s) { return s < INFINITY; }  // false for a NaN
__device__ __forceinline__ float usable_scale(float s) { return !finite_scale(s) ? 1.f : s < 1e-30f ? 1e-30f : s; }

}  // namespace rt
