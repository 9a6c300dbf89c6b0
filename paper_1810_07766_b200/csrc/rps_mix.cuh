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

// The upper halves of two fp32 values as a word of bf16, and what they leave (taken from infinity or NaN: NaN).
__device__ __forceinline__ Pair cut(const Pair& v, uint32_t& word)
{
    float lo, hi;
    v.get(lo, hi);
    word = __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x7632);
    return v + Pair(__uint_as_float((__float_as_uint(lo) & 0xFFFF0000u) ^ 0x80000000u), __uint_as_float((__float_as_uint(hi) & 0xFFFF0000u) ^ 0x80000000u));
}

// Two fp32 values as bf16 parts, as words: 8 of the 24 bits at a time, cut off, so three parts add up to the value exactly and have its sign.
// Parts that would be zero are 2^-50 of the value, which changes no sum (it is below half of a last place of any part that is not zero, and 2^-26 of one
// of the value's), so that an infinity of the other operand meets none that is zero where the value is not: infinity times a number is infinity.
// What is itself infinite or NaN leaves NaN behind the first part (keep_infinities).
__device__ __forceinline__ Pair next_part(const Pair& value, const Pair& rest, uint32_t& word) { return cut(fma(value, Pair(0x1p-50f), rest), word); }

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
