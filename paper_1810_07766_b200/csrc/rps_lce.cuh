// Device code of the loss that the tensor cores' path and the one for a few tokens share.
#pragma once

#include <algorithm>

#include "rps_rows.cuh"

namespace rps_ops {

// The worker's tokens in a new order: those that take part in theirs, then the ignored ones.  A thread takes four tokens at a time; a
// scan over the lanes and one over the warps give each its place.  Returns how many take part; `write`: also what later kernels
// need of it goes out; row_of (or NULL): the order, for this CTA.
template <int THREADS>
__device__ __forceinline__ int select_tokens(const LceParams& prm, int w, bool write, int* row_of)
{
    constexpr int kEach = 4, kWarps = THREADS / 32;
    static_assert(kWarps <= 32, "a lane for each warp's count");
    __shared__ int warp_count[kWarps];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int64_t* targets = prm.targets + w * prm.tokens;
    int* rows = prm.rows + w * prm.tokens;
    const int64_t padded = w * prm.tokens_padded;
    int kept = 0;
    for (int64_t t0 = 0; t0 < prm.tokens; t0 += THREADS * kEach) {
        const int64_t t = t0 + threadIdx.x * kEach;
        int64_t y[kEach];
        int mine = 0;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            y[j] = t + j < prm.tokens ? targets[t + j] : prm.ignore_index;
            mine += y[j] != prm.ignore_index;
        }
        int upto = mine;  // of this lane and those before it
#pragma unroll
        for (int s = 1; s < 32; s *= 2) {
            const int n = __shfl_up_sync(0xFFFFFFFFu, upto, s);
            if (lane >= s) upto += n;
        }
        if (lane == 31) warp_count[warp] = upto;
        __syncthreads();
        int warps_upto = lane < kWarps ? warp_count[lane] : 0;
#pragma unroll
        for (int s = 1; s < 32; s *= 2) {
            const int n = __shfl_up_sync(0xFFFFFFFFu, warps_upto, s);
            if (lane >= s) warps_upto += n;
        }
        const int before = __shfl_sync(0xFFFFFFFFu, warps_upto, warp > 0 ? warp - 1 : 0);
        int at = kept + upto - mine + (warp > 0 ? before : 0);
        kept += __shfl_sync(0xFFFFFFFFu, warps_upto, 31);
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            if (t + j >= prm.tokens) break;
            const bool in = y[j] != prm.ignore_index;
            // ignored tokens are filled in from the end, so that the places do not depend on the count: number i lies i from the end
            const int place = in ? at : (int)prm.tokens - 1 - ((int)t + j - at);
            if (row_of != nullptr) row_of[place] = (int)t + j;
            if (write) {
                rows[place] = (int)t + j;
                if (in) {
                    const bool names_a_row = y[j] >= 0 && y[j] < prm.vocab;
                    prm.target[padded + at] = names_a_row ? (int)y[j] : -1;
                    if (prm.backward) {
                        const float g = prm.reduction == RPS_REDUCE_NONE ? prm.dloss[w * prm.tokens + t + j] : 1.0f;
                        prm.info[padded + at] = make_float2(prm.lse_in[w * prm.tokens + t + j], names_a_row ? g : nanf(""));
                    } else if (!names_a_row) {
                        const_cast<float*>(prm.hit)[padded + at] = nanf("");  // the others' are found among the logits
                    }
                } else if (!prm.backward) {
                    prm.lse[w * prm.tokens + t + j] = 0.0f;
                    if (prm.reduction == RPS_REDUCE_NONE) prm.loss[w * prm.tokens + t + j] = 0.0f;
                }
            }
            if (in) ++at;
        }
        __syncthreads();
    }
    if (threadIdx.x == 0 && write) {
        prm.count[w] = kept;
        if (prm.backward) {
            // A factor that all rows share stays out of dl: near a token's target dl is p - 1, which bf16 holds all but exactly, and
            // (p - 1) times a factor it does not (relative error of the gradients: 2.7e-3 -> 1.7e-3, 1.65e-3 of it the rounding of the
            // result).
            prm.scale[w] = prm.factor * (prm.reduction == RPS_REDUCE_NONE || kept == 0 ? 1.0f : prm.reduction == RPS_REDUCE_MEAN ? prm.dloss[w] / (float)kept : prm.dloss[w]);
        } else {
            prm.done[w] = 0;
            if (kept == 0 && prm.reduction != RPS_REDUCE_NONE) prm.loss[w] = 0.0f;
        }
    }
    return kept;
}

template <typename T>
int aligned_source(const void* p, int64_t cols, int64_t row, int64_t worker)
{
    return std::min(alignment<T>(p, cols, row), alignment<T>(p, cols, worker));
}

}  // namespace rps_ops
