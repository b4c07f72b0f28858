// The parts that the attention kernels leave of every row, joined (sm_100a).
#pragma once

#include "attend_common.cuh"
#include "attend_split.h"

namespace rt {

// Joins the parts of every row: weights 2^(lse_p - max) / sum.  One warp per row.  A lane first looks after the weight of
// one part in 32; the outputs of the parts are then fetched U at a time, independently of one another (the parts come out of
// L2, so what counts is how many of its round trips follow one another).  A row of DP = 64 takes half a warp's lanes, so that
// two parts are fetched at once; a row of DP = 256 takes two warps, one for each half.  Parts that saw no key are not read.
// Bound by latency: 8 parts of 1024 rows of 256 (8.4 MB) take about 8 us under the profiler, which empties the caches.
constexpr int kMergePartsThreads = 128;
template <typename T, int DP>
__global__ void __launch_bounds__(kMergePartsThreads) merge_parts_kernel(const AttendArgs a, const PrefixSplit split)
{
    constexpr int LANES = DP == 64 ? 16 : 32, SIDE = 32 / LANES, U = 8, WARPS = DP == 256 ? 2 : 1;
    const int lane = threadIdx.x & 31;
    const long long warp = (long long)blockIdx.x * (kMergePartsThreads / 32) + (threadIdx.x >> 5), row = warp / WARPS;
    const int n_heads = a.kv_heads * a.group;
    const long long n_rows = (long long)a.n_seqs * a.q_len * n_heads;
    const int token = (int)((unsigned)row / (unsigned)n_heads), head = (int)(row - (long long)token * n_heads);
    int prefix_parts = a.prefix_parts;
    if (split.run > 0)  // the prefix was dealt out by tiles
        prefix_parts = parts_of_block(split, (token * a.group + head % a.group) / kTcBlockRows);
    const int skip = a.prefix_parts - prefix_parts;  // parts of the workspace that this row does not use
    const int parts = prefix_parts + a.suffix_parts;
    wait_for_previous_kernel();
    if (row >= n_rows || suffix_length(a, (int)((unsigned)token / (unsigned)a.q_len)) < 0) return;
    const int side = lane / LANES, d = (int)(warp % WARPS) * 128 + (lane % LANES) * 4;
    float m = -INFINITY, total = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int p0 = 0; p0 < parts; p0 += 32) {
        const int mine = p0 + lane;
        const int mine_at = mine < prefix_parts ? mine : mine + skip;
        const float lse = mine < parts ? a.part_lse[(long long)mine_at * n_rows + row] : -INFINITY;
        float top = fmaxf(m, lse);
#pragma unroll
        for (int s = 16; s >= 1; s >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, s));
        const float base = top == -INFINITY ? 0.f : top;
        // A NaN among the parts (a NaN score) is skipped by the maximum and kept by the weights.
        // A part that saw keys never weighs nothing, or a NaN among its values would be lost with it: 2^-149 where the exponential is zero.
        float w = lse == -INFINITY ? 0.f : ex2(lse - base);
        if (w == 0.f && lse != -INFINITY) w = __uint_as_float(1u);
        const float keep = m == -INFINITY ? 0.f : ex2(m - base);
        float sum = w;
#pragma unroll
        for (int s = 16; s >= 1; s >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, s);
        total = total * keep + sum;
        m = top;
        o.x *= keep; o.y *= keep; o.z *= keep; o.w *= keep;
        const int here = min(32, parts - p0);
        for (int i0 = 0; i0 < here; i0 += U * SIDE) {
            float4 x[U];
            float wi[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = i0 + u * SIDE + side;
                wi[u] = __shfl_sync(0xFFFFFFFFu, w, i & 31);
                const bool there = i < here && wi[u] != 0.f;
                const int p = p0 + i;
                x[u] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (there && d < a.dim)
                    x[u] = *reinterpret_cast<const float4*>(a.part_out + ((long long)(p < prefix_parts ? p : p + skip) * n_rows + row) * a.dim + d);
                if (!there) wi[u] = 0.f;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                o.x = fmaf(wi[u], x[u].x, o.x); o.y = fmaf(wi[u], x[u].y, o.y);
                o.z = fmaf(wi[u], x[u].z, o.z); o.w = fmaf(wi[u], x[u].w, o.w);
            }
        }
    }
    const bool empty = total == 0.f;  // a part that saw a key has a weight of 1, or NaN
    const float inv = empty ? 0.f : 1.0f / total;
    if constexpr (SIDE == 2) {
        o.x += __shfl_xor_sync(0xFFFFFFFFu, o.x, 16); o.y += __shfl_xor_sync(0xFFFFFFFFu, o.y, 16);
        o.z += __shfl_xor_sync(0xFFFFFFFFu, o.z, 16); o.w += __shfl_xor_sync(0xFFFFFFFFu, o.w, 16);
    }
    if (side == 0 && d < a.dim)
        *reinterpret_cast<uint2*>(reinterpret_cast<unsigned char*>(a.out) + (row * a.dim + d) * 2) =
            make_uint2(pack2<T>(o.x * inv, o.y * inv), pack2<T>(o.z * inv, o.w * inv));
    if (lane == 0 && d < 128 && a.lse) a.lse[row] = empty ? -INFINITY : (m + log2f(total)) * 0.69314718055994531f;
}

}  // namespace rt
