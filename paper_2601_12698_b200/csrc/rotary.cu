// Entry points of the rotary positions: frequencies, argument checks, the launch rule and the kernel's instances.
#include <float.h>
#include <math.h>
#include <string.h>

#include "rotary_kernel.cuh"
#include "tuner_internal.h"

namespace rt {
namespace {

typedef long double Real;  // x87: 64 bits of mantissa
static_assert(LDBL_MANT_DIG >= 64, "fractions of a turn are whole numbers of 64 bits");

constexpr Real kTwoPi = 6.283185307179586476925286766559005768L;

bool positive(double x) { return x > 0 && x < INFINITY; }

int check_spec(const rt_rotary_spec* s)
{
    if (s->rot_dim < 2 || s->rot_dim > RT_KV_MAX_HEAD_DIM || s->rot_dim % 2 || s->scaling < RT_ROTARY_NONE || s->scaling > RT_ROTARY_YARN) {
        set_error("rot_dim=%d or scaling=%d out of range", (int)s->rot_dim, (int)s->scaling);
        return RT_ERR_SHAPE;
    }
    const bool stretched = s->scaling != RT_ROTARY_NONE, by_length = s->scaling == RT_ROTARY_BANDS || s->scaling == RT_ROTARY_YARN;
    if (!(s->base > 1 && s->base < INFINITY) || (stretched && !positive(s->factor)) || (by_length && !positive(s->original_len)) ||
        (s->scaling == RT_ROTARY_NTK && s->rot_dim < 4) ||
        (s->scaling == RT_ROTARY_BANDS && !(positive(s->low_turns) && positive(s->high_turns) && s->low_turns < s->high_turns)) ||
        (s->scaling == RT_ROTARY_YARN && !(positive(s->slow_turns) && positive(s->fast_turns) && s->slow_turns < s->fast_turns))) {
        set_error("base, factor, original_len or turns out of range for scaling %d", (int)s->scaling);
        return RT_ERR_SHAPE;
    }
    return RT_OK;
}

Real between_0_and_1(Real x) { return x < 0 ? 0 : x > 1 ? 1 : x; }

typedef void (*RotaryKernel)(RotaryArgs);

template <typename T, int P, int U>
int launch_rotary(RotaryArgs a, cudaStream_t stream)
{
    const int heads = a.side[0].heads + a.side[1].heads, groups = kRotaryThreads / a.lanes;
    a.split = std::min(groups, (heads + U - 1) / U);
    a.tokens_per_cta = groups / a.split;
    const long long ctas = (a.n_tokens + a.tokens_per_cta - 1) / a.tokens_per_cta;
    if (ctas > 0x7fffffffLL) {
        set_error("n_tokens=%lld needs too many CTAs", (long long)a.n_tokens);
        return RT_ERR_SHAPE;
    }
    const int threads = (a.tokens_per_cta * a.split * a.lanes + 31) / 32 * 32;
    void* params[] = {&a};
    return launch_kernel((const void*)(RotaryKernel)rotary_kernel<T, P, U>, dim3((unsigned)ctas), dim3((unsigned)threads), 0, stream, params);
}

// A thread takes up to U heads of its token and fetches them all at once; its P sines and cosines are worked out meanwhile.  Eight heads to a
// thread where that fills the device twice over, two otherwise: 16384 tokens x 40 heads of 128 bf16: 55.8 us, 63.8 with two (81.8 with four
// heads at a time, ten times over); 64 tokens: 4.2 us in a graph with eight, 2.6 with two.
template <typename T, int P>
int launch_width(RotaryArgs a, int rot, int tail_elems, bool interleaved, cudaStream_t stream)
{
    constexpr int VB = P * (int)sizeof(T);
    a.items = rot / 2 / P;
    a.second = interleaved ? VB : rot / 2 * (int)sizeof(T);
    a.interleaved = interleaved;
    a.first_step = interleaved ? 2 * VB : VB;
    a.tail = tail_elems / P;
    a.lanes = a.items + (a.tail + 1) / 2;
    rt_limits L;
    const int st = current_limits(&L);
    if (st != RT_OK) return st;
    const int heads = a.side[0].heads + a.side[1].heads;
    if (a.n_tokens * ((heads + 7) / 8) * a.items >= (long long)L.sm_count * 1024) return launch_rotary<T, P, 8>(a, stream);
    return launch_rotary<T, P, 2>(a, stream);
}

template <typename T>
int launch_typed(const RotaryArgs& a, int width, int rot, int tail, bool interleaved, cudaStream_t stream)
{
    if constexpr (sizeof(T) == 2) {
        if (width == 8) return launch_width<T, 8>(a, rot, tail, interleaved, stream);
    }
    if (width >= 4) return launch_width<T, 4>(a, rot, tail, interleaved, stream);
    if (width >= 2) return launch_width<T, 2>(a, rot, tail, interleaved, stream);
    return launch_width<T, 1>(a, rot, tail, interleaved, stream);
}

}  // namespace
}  // namespace rt

extern "C" {

int rotary_frequencies(const rt_rotary_spec* s, uint64_t* turns, float* magnitude)
{
    using namespace rt;
    if (!s || !turns || !magnitude) {
        set_error("spec, turns or magnitude is NULL");
        return RT_ERR_NULL;
    }
    const int st = check_spec(s);
    if (st != RT_OK) return st;
    // In 64 bits of mantissa: what is wrong with a fraction counts once for every position.
    const int rot = s->rot_dim;
    const Real factor = s->factor, original_len = s->original_len;
    const Real base = s->scaling == RT_ROTARY_NTK ? s->base * powl(factor, (Real)rot / (rot - 2)) : (Real)s->base;
    Real first = 0, last = 0;
    if (s->scaling == RT_ROTARY_YARN) {
        const auto pair = [&](Real n) { return rot * logl(original_len / (kTwoPi * n)) / (2 * logl(base)); };
        first = fmaxl(0, floorl(pair(s->fast_turns)));
        last = fminl(rot - 1, ceill(pair(s->slow_turns)));
    }
    for (int j = 0; j < rot / 2; ++j) {
        Real theta = powl(base, (Real)(-2 * j) / rot);
        if (s->scaling == RT_ROTARY_LINEAR) theta /= factor;
        if (s->scaling == RT_ROTARY_BANDS) {
            const Real keep = between_0_and_1((original_len * theta / kTwoPi - s->low_turns) / ((Real)s->high_turns - s->low_turns));
            theta = theta * keep + theta / factor * (1 - keep);
        }
        if (s->scaling == RT_ROTARY_YARN) {
            const Real divided = between_0_and_1((j - first) / fmaxl(last - first, 0.001L));
            theta = theta / factor * divided + theta * (1 - divided);
        }
        const Real part = theta / kTwoPi, scaled = roundl(ldexpl(part - floorl(part), 64));
        turns[j] = scaled >= 18446744073709551616.0L ? 0 : (uint64_t)scaled;
    }
    *magnitude = s->scaling == RT_ROTARY_YARN ? (float)(0.1 * log(s->factor) + 1) : 1.0f;
    return RT_OK;
}

int rotary_launch(const rt_rotary* r, const int64_t* positions, int64_t n_tokens, int32_t head_dim, const rt_rotary_side* sides, int dtype,
                  void* stream)
{
    using namespace rt;
    if (!r || !sides) {
        set_error("rotary or sides is NULL");
        return RT_ERR_NULL;
    }
    if (dtype < RT_BF16 || dtype > RT_FP32) {
        set_error("dtype %d is not an rt_dtype", dtype);
        return RT_ERR_DTYPE;
    }
    if (n_tokens < 0 || head_dim < 2 || head_dim > RT_KV_MAX_HEAD_DIM || r->rot_dim < 2 || r->rot_dim > head_dim || r->rot_dim % 2) {
        set_error("n_tokens=%lld head_dim=%d rot_dim=%d out of range", (long long)n_tokens, (int)head_dim, (int)r->rot_dim);
        return RT_ERR_SHAPE;
    }
    const int64_t size = elem_bytes_of(dtype);
    RotaryArgs a;
    memset(&a, 0, sizeof(a));
    // The widest vectors of P elements that rot / 2, the tail, the pointers and the strides allow.
    int width = size == 2 ? 8 : 4;
    while (width > 1 && (r->rot_dim / 2 % width || (head_dim - r->rot_dim) % width)) width /= 2;
    uintptr_t places = 0;
    bool copies = false;
    for (int i = 0; i < 2; ++i) {
        const rt_rotary_side* s = &sides[i];
        if (s->heads == 0) continue;
        if (s->heads < 0 || s->heads > 65535 || s->in_token_stride < 0 || s->in_head_stride < 0 || s->out_token_stride < 0 || s->out_head_stride < 0 ||
            (n_tokens > 1 && s->out_token_stride == 0) || (s->heads > 1 && s->out_head_stride == 0)) {
            set_error("heads=%lld or a stride out of range", (long long)s->heads);
            return RT_ERR_SHAPE;
        }
        if (n_tokens == 0) continue;
        if (!s->in || !s->out) {
            set_error("a tensor pointer is NULL");
            return RT_ERR_NULL;
        }
        if (((uintptr_t)s->in | (uintptr_t)s->out) & (uintptr_t)(size - 1)) {
            set_error("a tensor is not aligned to its element size");
            return RT_ERR_ALIGN;
        }
        RotarySide& d = a.side[i];
        d.in = (const unsigned char*)s->in;
        d.out = (unsigned char*)s->out;
        d.in_token = s->in_token_stride * size;
        d.in_head = s->in_head_stride * size;
        d.out_token = s->out_token_stride * size;
        d.out_head = s->out_head_stride * size;
        d.heads = (int)s->heads;
        const bool same = s->in == s->out && (n_tokens == 1 || d.in_token == d.out_token) && (d.heads == 1 || d.in_head == d.out_head);
        if (s->in == s->out && !same) {
            set_error("in and out overlap with different strides");
            return RT_ERR_SHAPE;
        }
        d.copy_tail = !same;
        copies = copies || !same;
        places |= (uintptr_t)s->in | (uintptr_t)s->out;
        if (n_tokens > 1) places |= (uintptr_t)d.in_token | (uintptr_t)d.out_token;
        if (d.heads > 1) places |= (uintptr_t)d.in_head | (uintptr_t)d.out_head;
    }
    if (n_tokens == 0 || a.side[0].heads + a.side[1].heads == 0) return RT_OK;
    if (!positions || !r->turns) {
        set_error("positions or turns is NULL");
        return RT_ERR_NULL;
    }
    if (((uintptr_t)positions | (uintptr_t)r->turns) & 7u) {
        set_error("positions or turns is not aligned to 8 bytes");
        return RT_ERR_ALIGN;
    }
    if (a.side[0].heads > 0 && a.side[1].heads > 0 &&
        (a.side[0].out == a.side[1].out || a.side[0].out == a.side[1].in || a.side[1].out == a.side[0].in)) {
        set_error("the two sides overlap");
        return RT_ERR_SHAPE;
    }
    while (width > 1 && (places & (uintptr_t)(width * size - 1))) width /= 2;
    a.turns = (const unsigned long long*)r->turns;
    a.positions = (const long long*)positions;
    a.n_tokens = n_tokens;
    a.rot_bytes = r->rot_dim * (int)size;
    a.magnitude = r->magnitude;
    a.sign = r->backward ? -1.f : 1.f;
    const int tail = copies ? head_dim - r->rot_dim : 0;
    const bool inter = r->interleaved != 0;
    switch (dtype) {
        case RT_BF16: return launch_typed<__nv_bfloat16>(a, width, r->rot_dim, tail, inter, (cudaStream_t)stream);
        case RT_FP16: return launch_typed<__half>(a, width, r->rot_dim, tail, inter, (cudaStream_t)stream);
        default: return launch_typed<float>(a, width, r->rot_dim, tail, inter, (cudaStream_t)stream);
    }
}

}  // extern "C"
