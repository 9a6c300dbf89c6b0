// What the kernels of linear attention share.
#pragma once

#include <algorithm>

#include "rps_rows.cuh"

namespace rps_ops {
namespace {

// The decay's powers, as double: a log_decay of minus infinity is a decay of zero, whose power 0 is one; a positive one or NaN gives NaN.
__device__ __forceinline__ double power(float log_decay, int64_t exponent)
{
    if (!(log_decay <= 0.0f)) return nan("");
    return exp((double)fmaxf(log_decay, -1e4f) * (double)exponent);
}

// The upper halves of two fp32 values as a word of bf16, and these less zero.
__device__ __forceinline__ Pair upper_halves(const Pair& v, uint32_t& word)
{
    float lo, hi;
    v.get(lo, hi);
    word = __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x7632);
    return Pair(__uint_as_float((__float_as_uint(lo) & 0xFFFF0000u) ^ 0x80000000u), __uint_as_float((__float_as_uint(hi) & 0xFFFF0000u) ^ 0x80000000u));
}

// The largest fp32 value below a positive one (0 of 0), as a factor makes it.
constexpr float kBelow = 0x1.fffffep-1f;

// Two products v * factor as three bf16 parts each, as words: 8 bits at a time, which add up to the product but for 2^-24 of it.  `below`: factor * kBelow.
// All parts have the product's sign, and none is zero unless it is: the first is cut off from a little less than the product, so that something is left,
// and of what the second leaves 2^-24 of it are left in any case (2^-31 of the product).  So an infinity of the other operand meets no zero: infinity times a
// number is infinity.  What is itself infinite or NaN has NaN as its second and third part (keep_infinities).
__device__ __forceinline__ void cut_in_parts(const Pair& v, const Pair& factor, const Pair& below, uint32_t& first, uint32_t& second, uint32_t& third)
{
    const Pair rest = fma(v, factor, upper_halves(v * below, first));
    float lo, hi;
    fma(upper_halves(rest, second), Pair(kBelow), rest).get(lo, hi);
    third = two_bf16(lo, hi);
}

// Of the exponents of two bf16 values those that are all ones, as the sign bit of each half.
__device__ __forceinline__ uint32_t has_infinite_exponent(uint32_t word) { return ((word & 0x7F807F80u) + 0x00800080u) & 0x80008000u; }

// A further part of infinity or NaN: the value itself, as the first one is.
__device__ __forceinline__ uint32_t keep_infinities(uint32_t first, uint32_t further)
{
    const uint32_t mask = (has_infinite_exponent(first) >> 15) * 0xFFFFu;
    return (further & ~mask) | (first & mask);
}

__device__ __forceinline__ uint4 keep_infinities(const uint4& first, const uint4& further)
{
    return make_uint4(keep_infinities(first.x, further.x), keep_infinities(first.y, further.y), keep_infinities(first.z, further.z), keep_infinities(first.w, further.w));
}

struct Place {
    int w, sequence, head;
    int64_t length;  // tokens of the sequence that take part
};

__device__ __forceinline__ Place place_of(const MixParams& prm, int64_t unit)
{
    Place p;
    p.head = (int)(unit % prm.heads);
    const int64_t s = unit / prm.heads;
    p.w = (int)(s / prm.sequences), p.sequence = (int)(s % prm.sequences);
    p.length = prm.tokens;
    if (prm.lengths != nullptr) p.length = max((int64_t)0, min(prm.tokens, __ldg(prm.lengths + s)));
    return p;
}

template <typename T>
__device__ __forceinline__ const T* first_token(const MixOperand& o, const Place& p)
{
    return static_cast<const T*>(o.base) + p.w * o.worker + p.sequence * o.sequence + p.head * o.head;
}

// What all operands' rows of a call can be moved in.
template <typename T>
int mix_alignment(const MixParams& prm)
{
    const auto of = [](const MixOperand& o, int64_t cols) {
        return std::min({alignment<T>(o.base, cols, o.token), alignment<T>(o.base, cols, o.head), alignment<T>(o.base, cols, o.sequence), alignment<T>(o.base, cols, o.worker)});
    };
    int align = 16;
    for (int i = 0; i < prm.terms; ++i) {
        const MixTerm& t = prm.term[i];
        align = std::min({align, of(t.x, t.a), of(t.y, t.a), of(t.z, t.b), alignment<T>(t.out, t.b, t.b)});
    }
    return align;
}

}  // namespace
}  // namespace rps_ops
