// What both kernels of linear attention share.
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
