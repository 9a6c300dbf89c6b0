// The loss around its matrix products: which tokens take part, their rows laid out for the tensor cores, and the end of
// the softmax statistics.
#include "rps_ops_kernels.h"

namespace rps_ops {
namespace {

constexpr int kSelectThreads = 1024;
constexpr int kMergeThreads = 128;

// One CTA per worker.  rows[] becomes a permutation of the worker's tokens: those that take part in their order, then
// the ignored ones; a ballot and a scan over the warps' counts give each token its place.
__global__ void __launch_bounds__(kSelectThreads) rps_lce_select_kernel(const LceParams prm)
{
    __shared__ int warp_count[kSelectThreads / 32];
    const int w = blockIdx.x, lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int64_t* targets = prm.targets + w * prm.tokens;
    int* rows = prm.rows + w * prm.tokens;
    int* target = prm.target + w * prm.tokens_padded;
    int kept = 0;
    for (int64_t t0 = 0; t0 < prm.tokens; t0 += kSelectThreads) {
        const int64_t t = t0 + threadIdx.x;
        const int64_t y = t < prm.tokens ? targets[t] : prm.ignore_index;
        const bool in = t < prm.tokens && y != prm.ignore_index;
        const unsigned mask = __ballot_sync(0xFFFFFFFFu, in);
        if (lane == 0) warp_count[warp] = __popc(mask);
        __syncthreads();
        int before = __popc(mask & ((1u << lane) - 1)), total = 0;
        for (int i = 0; i < kSelectThreads / 32; ++i) {
            if (i < warp) before += warp_count[i];
            total += warp_count[i];
        }
        if (in) {
            const int at = kept + before;
            const bool names_a_row = y >= 0 && y < prm.vocab;
            rows[at] = (int)t;
            target[at] = names_a_row ? (int)y : -1;
            if (!prm.backward) const_cast<float*>(prm.hit)[w * prm.tokens_padded + at] = names_a_row ? 0.0f : nanf("");
        } else if (t < prm.tokens) {
            // filled from the end, so that the places do not depend on the count: ignored token number i lies i from the end
            const int ignored = (int)t - (kept + before);
            rows[prm.tokens - 1 - ignored] = (int)t;
            if (!prm.backward) {
                prm.lse[w * prm.tokens + t] = 0.0f;
                if (prm.reduction == RPS_REDUCE_NONE) prm.loss[w * prm.tokens + t] = 0.0f;
            }
        }
        kept += total;
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        prm.count[w] = kept;
        if (!prm.backward) prm.done[w] = 0;
    }
    if (!prm.backward) {
        if (kept == 0 && prm.reduction != RPS_REDUCE_NONE && threadIdx.x == 0) prm.loss[w] = 0.0f;
        return;
    }
    // A factor that all rows share stays out of dl: near a token's target dl is p - 1, which bf16 holds all but exactly, and
    // (p - 1) times a factor it does not (relative error of the gradients: 2.7e-3 -> 1.7e-3, 1.65e-3 of it the rounding of the result).
    if (threadIdx.x == 0)
        prm.scale[w] = prm.reduction == RPS_REDUCE_NONE || kept == 0 ? 1.0f : prm.reduction == RPS_REDUCE_MEAN ? prm.dloss[w] / (float)kept : prm.dloss[w];
    __syncthreads();  // rows[] and target[] of this CTA's own threads
    for (int i = threadIdx.x; i < kept; i += kSelectThreads) {
        const int t = rows[i];
        float g = prm.reduction == RPS_REDUCE_NONE ? prm.dloss[w * prm.tokens + t] : 1.0f;
        if (target[i] < 0) g = nanf("");
        prm.info[w * prm.tokens_padded + i] = make_float2(prm.lse_in[w * prm.tokens + t], g);
    }
}

template <typename T>
__global__ void __launch_bounds__(256) rps_lce_gather_kernel(const LceParams prm)
{
    const int w = blockIdx.y;
    const int64_t i = blockIdx.x;
    const int count = prm.count[w];
    const bool in = i < count;
    if (!in && i < prm.tokens && prm.backward) {  // an ignored token's gradient
        T* out = static_cast<T*>(prm.dhidden) + (w * prm.tokens + prm.rows[w * prm.tokens + i]) * prm.cols;
        for (int64_t c = threadIdx.x; c < prm.cols; c += blockDim.x) out[c] = from_float<T>(0.0f);
    }
    // products read whole token tiles: the rows behind the last one are cleared
    if (i >= (count + kTokenTile - 1) / kTokenTile * kTokenTile) return;
    const T* src = static_cast<const T*>(prm.hidden) + w * prm.hidden_worker + (in ? prm.rows[w * prm.tokens + i] : 0) * prm.hidden_row;
    bf16* dst = prm.packed + (w * prm.planes * prm.tokens_padded + i) * prm.cols_padded;
    const int64_t plane = prm.tokens_padded * prm.cols_padded;
    for (int64_t c = threadIdx.x; c < prm.cols_padded; c += blockDim.x) {
        const float v = in && c < prm.cols ? to_float<T>(src[c]) : 0.0f;
        if (prm.planes == 1) {
            dst[c] = __float2bfloat16_rn(v);
        } else {
            bf16 p[3];
            split_planes(v, p);
            for (int q = 0; q < 3; ++q) dst[q * plane + c] = p[q];
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(256) rps_planes_kernel(const PlanesParams prm)
{
    const int w = blockIdx.y;
    const int64_t i = blockIdx.x;
    const T* src = static_cast<const T*>(prm.src) + w * prm.src_worker + i * prm.src_row;
    bf16* dst = prm.dst + w * prm.dst_worker + i * prm.dst_row;
    for (int64_t c = threadIdx.x; c < prm.dst_row; c += blockDim.x) {
        const float v = i < prm.valid && c < prm.cols ? to_float<T>(src[c]) : 0.0f;
        if (prm.planes == 1) {
            dst[c] = __float2bfloat16_rn(v);
        } else {
            bf16 p[3];
            split_planes(v, p);
            for (int q = 0; q < 3; ++q) dst[q * prm.dst_plane + c] = p[q];
        }
    }
}

// Joins the (maximum, sum) pairs of a row's vocabulary tiles, a thread for each row.  The sum over a worker's rows is made
// of the blocks' sums by the block that finishes last, always in the same order.
__global__ void __launch_bounds__(kMergeThreads) rps_lce_merge_kernel(const LceParams prm)
{
    __shared__ float warp_sum[kMergeThreads / 32];
    __shared__ bool last;
    const int w = blockIdx.y, count = prm.count[w];
    const int blocks = (count + kMergeThreads - 1) / kMergeThreads;
    if ((int)blockIdx.x >= blocks) return;
    const int i = blockIdx.x * kMergeThreads + threadIdx.x;
    float loss = 0.0f;
    if (i < count) {
        const float2* part = prm.part + w * prm.stat_tiles * prm.tokens_padded + i;
        float top = -INFINITY, sum = 0.0f;
        for (int64_t v = 0; v < prm.stat_tiles; ++v) {
            const float2 p = part[v * prm.tokens_padded];
            const float m = fmaxf(top, p.x), at = m == -INFINITY ? 0.0f : m;
            sum = sum * __expf(top - at) + p.y * __expf(p.x - at);
            top = m;
        }
        const float lse = top + logf(sum);
        loss = lse - prm.hit[w * prm.tokens_padded + i];
        const int64_t t = prm.rows[w * prm.tokens + i];
        prm.lse[w * prm.tokens + t] = lse;
        if (prm.reduction == RPS_REDUCE_NONE) prm.loss[w * prm.tokens + t] = loss;
    }
    if (prm.reduction == RPS_REDUCE_NONE) return;
    for (int s = 16; s > 0; s /= 2) loss += __shfl_xor_sync(0xFFFFFFFFu, loss, s);
    if (threadIdx.x % 32 == 0) warp_sum[threadIdx.x / 32] = loss;
    __syncthreads();
    if (threadIdx.x != 0) return;
    float sum = 0.0f;
    for (int k = 0; k < kMergeThreads / 32; ++k) sum += warp_sum[k];
    float* sums = prm.sums + w * gridDim.x;
    sums[blockIdx.x] = sum;
    __threadfence();
    last = atomicAdd(&prm.done[w], 1) == blocks - 1;
    if (!last) return;
    __threadfence();
    double all = 0.0;
    for (int b = 0; b < blocks; ++b) all += (double)__ldcg(&sums[b]);
    if (prm.reduction == RPS_REDUCE_MEAN) all /= (double)count;
    prm.loss[w] = (float)all;
}

}  // namespace

cudaError_t launch_lce_select(const LceParams& prm, cudaStream_t stream)
{
    rps_lce_select_kernel<<<prm.n, kSelectThreads, 0, stream>>>(prm);
    return cudaGetLastError();
}

cudaError_t launch_lce_gather(const LceParams& prm, cudaStream_t stream)
{
    const dim3 grid((unsigned)prm.tokens_padded, (unsigned)prm.n);
    if (prm.f32)
        rps_lce_gather_kernel<float><<<grid, 256, 0, stream>>>(prm);
    else
        rps_lce_gather_kernel<bf16><<<grid, 256, 0, stream>>>(prm);
    return cudaGetLastError();
}

int64_t lce_merge_blocks(int64_t tokens) { return ceil_div(tokens, kMergeThreads); }

cudaError_t launch_lce_merge(const LceParams& prm, cudaStream_t stream)
{
    const dim3 grid((unsigned)lce_merge_blocks(prm.tokens), (unsigned)prm.n);
    rps_lce_merge_kernel<<<grid, kMergeThreads, 0, stream>>>(prm);
    return cudaGetLastError();
}

cudaError_t launch_planes(const PlanesParams& prm, cudaStream_t stream)
{
    const dim3 grid((unsigned)prm.rows, (unsigned)prm.n);
    if (prm.f32)
        rps_planes_kernel<float><<<grid, 256, 0, stream>>>(prm);
    else
        rps_planes_kernel<bf16><<<grid, 256, 0, stream>>>(prm);
    return cudaGetLastError();
}

}  // namespace rps_ops
