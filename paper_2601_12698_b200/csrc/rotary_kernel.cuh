// Rotary positions of queries and keys (sm_100a).
//
//   y1 = m (x1 cos a - x2 sin a),  y2 = m (x2 cos a + x1 sin a),  a = 2 pi frac(position * turns_j)
//
// turns_j is a 64-bit binary fraction of a turn, so the product modulo 2^64 is the place on the circle with no more error than the fraction's
// own, below 2^-63 of a turn, times the position; its top 32 bits, in binary32, are the angle to 2^-26 of a turn: no range reduction, no binary64.
//
// Bound by HBM: every element is read and written once.  A thread owns P pairs of one token (two vectors of P elements: j and
// j + rot / 2, or two neighbouring ones) and walks over the heads with them, so that sines and cosines are computed once per
// token and pair and stay in registers; U heads are fetched before the first is turned.  Elements behind the turned ones go through
// threads of their own, two vectors each.
//
// Measured: 16384 tokens x 40 heads of 128, bf16, 336 MB: 55.8 us, 6.0 TB/s, 0.93 of the copy bandwidth.  64 tokens: 2.6 us in a graph,
// the round trip for the position and the angles' arithmetic.
#pragma once

#include "add_rmsnorm_kernel.cuh"

namespace rt {

struct RotarySide {
    const unsigned char* in;
    unsigned char* out;
    long long in_token, in_head, out_token, out_head;  // strides in bytes
    int heads;
    int copy_tail;  // the elements from rot on are copied (not in place)
};
struct RotaryArgs {
    RotarySide side[2];  // q, k
    const unsigned long long* turns;
    const long long* positions;
    long long n_tokens;
    int items;           // threads of one token and head group that turn: rot / 2 / P
    int lanes;           // those and the ones that copy what is behind
    int second;          // bytes from a thread's first vector to its second
    int first_step;      // bytes from one item's first vector to the next one's
    int rot_bytes;
    int interleaved;
    int tail;            // vectors of P elements behind the turned ones
    int split;           // threads of one token and item, each with every split-th head
    int tokens_per_cta;
    float magnitude;
    float sign;          // -1: the gradient
};

constexpr int kRotaryThreads = 256;

template <typename T, int P, int U>
__global__ void __launch_bounds__(kRotaryThreads, U == 2 ? 3 : 2) rotary_kernel(const RotaryArgs a)
{
    constexpr int VB = P * (int)sizeof(T);
    const int item = threadIdx.x % a.lanes, group = threadIdx.x / a.lanes;
    const int part = group % a.split, in_cta = group / a.split;
    const long long token = (long long)blockIdx.x * a.tokens_per_cta + in_cta;
    wait_for_previous_kernel();
    if (in_cta >= a.tokens_per_cta || token >= a.n_tokens) return;
    const long long position = __ldg(a.positions + token);

    const int n_q = a.side[0].heads, heads = n_q + a.side[1].heads;
    const auto in_at = [&](int h) {
        const RotarySide& s = a.side[h >= n_q];
        return s.in + token * s.in_token + (long long)(h >= n_q ? h - n_q : h) * s.in_head;
    };
    const auto out_at = [&](int h) {
        const RotarySide& s = a.side[h >= n_q];
        return s.out + token * s.out_token + (long long)(h >= n_q ? h - n_q : h) * s.out_head;
    };
    Vec<VB> x[U][2];
    if (item >= a.items) {  // what is behind the turned elements
        const int vector = (item - a.items) * 2, first = a.rot_bytes + vector * VB;
        const bool pair = vector + 1 < a.tail;
        if (position < 0) return;
        for (int h0 = part; h0 < heads; h0 += U * a.split) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int h = h0 + u * a.split;
                if (h < heads && a.side[h >= n_q].copy_tail) {
                    x[u][0] = ld_stream<VB>(in_at(h) + first);
                    if (pair) x[u][1] = ld_stream<VB>(in_at(h) + first + VB);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int h = h0 + u * a.split;
                if (h < heads && a.side[h >= n_q].copy_tail) {
                    st_stream<VB>(out_at(h) + first, x[u][0]);
                    if (pair) st_stream<VB>(out_at(h) + first + VB, x[u][1]);
                }
            }
        }
        return;
    }
    const int first = item * a.first_step;
    const auto fetch = [&](int h0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int h = h0 + u * a.split;
            if (h < heads) {
                const unsigned char* p = in_at(h) + first;
                x[u][0] = ld_stream<VB>(p);
                x[u][1] = ld_stream<VB>(p + a.second);
            }
        }
    };
    fetch(part);  // under way while the position comes and the angles are worked out
    if (position < 0) return;
    float c[P], s[P];
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const unsigned long long place = (unsigned long long)position * __ldg(a.turns + item * P + i) + 0x80000000ull;
        float sine, cosine;
        sincospif((float)(int)(place >> 32) * 0x1p-31f, &sine, &cosine);
        c[i] = cosine * a.magnitude;
        s[i] = sine * a.magnitude * a.sign;
    }
    for (int h0 = part; h0 < heads; h0 += U * a.split) {
        if (h0 != part) fetch(h0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int h = h0 + u * a.split;
            if (h >= heads) break;
            float lo[P], hi[P], y[P], z[P];
            Codec<T, VB>::unpack(x[u][0], lo);
            Codec<T, VB>::unpack(x[u][1], hi);
            if (a.interleaved) {  // pairs side by side: the two vectors hold x1 x2 x1 x2 ...
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    const float x1 = 2 * i < P ? lo[(2 * i) % P] : hi[(2 * i) % P], x2 = 2 * i + 1 < P ? lo[(2 * i + 1) % P] : hi[(2 * i + 1) % P];
                    const float y1 = x1 * c[i] - x2 * s[i], y2 = x2 * c[i] + x1 * s[i];
                    if (2 * i < P) y[(2 * i) % P] = y1;
                    else z[(2 * i) % P] = y1;
                    if (2 * i + 1 < P) y[(2 * i + 1) % P] = y2;
                    else z[(2 * i + 1) % P] = y2;
                }
            } else {
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    y[i] = lo[i] * c[i] - hi[i] * s[i];
                    z[i] = hi[i] * c[i] + lo[i] * s[i];
                }
            }
            unsigned char* p = out_at(h) + first;
            st_stream<VB>(p, Codec<T, VB>::pack(y));
            st_stream<VB>(p + a.second, Codec<T, VB>::pack(z));
        }
    }
}

}  // namespace rt
