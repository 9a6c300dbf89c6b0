// The loss around its matrix products: which tokens take part, their rows laid out for the tensor cores, and the end of
// the softmax statistics.
#include "rps_lce.cuh"

namespace rps_ops {
namespace {

constexpr int kSelectThreads = 1024;
constexpr int kMergeThreads = 512, kMergeRows = 8, kManyMergeRows = 32;
constexpr int kRowThreads = 256;
constexpr int kFewTokens = 4 * kRowThreads;

// One CTA per worker.
__global__ void __launch_bounds__(kSelectThreads) rps_lce_select_kernel(const LceParams prm)
{
    after_the_kernel_before();
    select_tokens<kSelectThreads>(prm, blockIdx.x, true, nullptr);
}

// Eight columns from c on, as fp32; zero from `cols` on.
template <typename T, int ALIGN>
__device__ __forceinline__ void load_eight(const T* row, int c, int cols, float (&v)[8])
{
    if constexpr (sizeof(T) == 2) {
        widen(load_slice<T, ALIGN, true>(row, c, cols), v);
    } else {
        float a[4], b[4];
        widen(load_slice<T, ALIGN, true>(row, c, cols), a);
        widen(load_slice<T, ALIGN, true>(row, c + 4, cols), b);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = a[j], v[4 + j] = b[j];
    }
}

template <typename T>
__device__ __forceinline__ void store_parts(bf16* dst, int64_t plane, const float (&v)[8])
{
    if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<uint4*>(dst) = narrow(v);
    } else {
        uint4 parts[3];
        split_slice(v, parts);
#pragma unroll
        for (int q = 0; q < 3; ++q) *reinterpret_cast<uint4*>(dst + q * plane) = parts[q];
    }
}

// Rows of hidden laid out in the new order, a warp to a row.  SELECT (at most kFewTokens): every CTA finds the order out for itself, the
// first one of a worker also for the kernels to come, which saves a launch (one / two, us: 1 token 2.5 / 5.1; 1000 tokens x 256 bf16
// 3.3 / 5.7; of 8 workers x 512 bf16 8.2 / 8.5, x 1024 fp32 18.7 / 20.0: with more rows the order is found too often to gain by it).
template <typename T, int ALIGN, bool SELECT>
__global__ void __launch_bounds__(kRowThreads) rps_lce_gather_kernel(const LceParams prm)
{
    after_the_kernel_before();
    __shared__ int row_of[SELECT ? kFewTokens : 1];
    const int w = blockIdx.y, lane = threadIdx.x % 32;
    const int64_t i = (int64_t)blockIdx.x * (kRowThreads / 32) + threadIdx.x / 32;
    const int count = SELECT ? select_tokens<kRowThreads>(prm, w, blockIdx.x == 0 && blockIdx.z == 0, row_of) : prm.count[w], D = (int)prm.cols;
    const bool in = i < count;
    const int c0 = (blockIdx.z * 32 + lane) * 8, step = gridDim.z * 256;
    const int64_t token = i < prm.tokens ? (SELECT ? row_of[i] : prm.rows[w * prm.tokens + i]) : 0;
    if (!in && i < prm.tokens && prm.backward) {  // an ignored token's gradient
        T* out = static_cast<T*>(prm.dhidden) + (w * prm.tokens + token) * prm.cols;
        for (int c = blockIdx.z * 32 + lane; c < D; c += gridDim.z * 32) out[c] = from_float<T>(0.0f);
    }
    // the product with dl over the tokens reads whole blocks of rows: those behind the last one are cleared
    if (i >= (count + kTokenBlock - 1) / kTokenBlock * kTokenBlock) return;
    const T* src = static_cast<const T*>(prm.hidden) + w * prm.hidden_worker + (in ? token : 0) * prm.hidden_row;
    bf16* dst = prm.packed + (w * prm.planes * prm.tokens_padded + i) * prm.cols_padded;
    const int64_t plane = prm.tokens_padded * prm.cols_padded;
#pragma unroll 4
    for (int c = c0; c < prm.cols_padded; c += step) {
        float v[8];
        load_eight<T, ALIGN>(src, c, in ? D : 0, v);
        store_parts<T>(dst + c, plane, v);
    }
}

// Rows of a matrix of each worker as operands, eight columns to a thread.
template <typename T, int ALIGN>
__global__ void __launch_bounds__(kRowThreads) rps_planes_kernel(const PlanesParams prm)
{
    after_the_kernel_before();
    const int w = blockIdx.y, per_row = (int)(prm.dst_row / 8);
    const uint32_t total = (uint32_t)(prm.rows * per_row);  // below 2^32 (launch_planes)
    const uint32_t step = gridDim.x * kRowThreads;
    const T* src = static_cast<const T*>(prm.src) + w * prm.src_worker;
    bf16* dst = prm.dst + w * prm.dst_worker;
    constexpr int kAtATime = 4;
    for (uint64_t u0 = blockIdx.x * kRowThreads + threadIdx.x; u0 < total; u0 += (uint64_t)step * kAtATime) {
        float v[kAtATime][8];
        uint32_t row[kAtATime];
        int c[kAtATime];
#pragma unroll
        for (int k = 0; k < kAtATime; ++k) {
            const uint64_t u = u0 + (uint64_t)k * step;
            if (u >= total) break;
            row[k] = (uint32_t)u / (uint32_t)per_row;
            c[k] = (int)((uint32_t)u - row[k] * (uint32_t)per_row) * 8;
            load_eight<T, ALIGN>(src + (int64_t)row[k] * prm.src_row, c[k], (int)prm.cols, v[k]);
        }
#pragma unroll
        for (int k = 0; k < kAtATime; ++k) {
            if (u0 + (uint64_t)k * step >= total) break;
            store_parts<T>(dst + (int64_t)row[k] * prm.dst_row + c[k], prm.dst_plane, v[k]);
        }
    }
}

// Joins the (maximum, sum) pairs of a row's vocabulary tiles: a CTA for ROWS rows, whose pairs of a tile lie together, and 32 / ROWS tiles to a
// warp at a time.  The sum over a worker's rows is made of the CTAs' sums by the one that finishes last, always in the same order.  8 rows
// fill the SMs where 32 would not (4096 rows of 512 tiles 16 us against 25, 2048 of 196 6.0 against 10.4); where they would, fewer CTAs
// to wait for are better (8192 rows of 32 tiles 13.1 against 7.7).
// TOP: a row's loss is its divergence from the teacher, with the logits z of its entries, q their probabilities, and the largest logit and the sum of
// exponentials: tau^2 sum q (log (q sum) + (top - z) / tau).  Entry by entry, as terms of different sizes, lse's next to z's or q's entropy
// next to theirs, would cancel (with logits that are all larger by 1024 to 6e-5).
template <int ROWS, bool TOP>
__global__ void __launch_bounds__(kMergeThreads) rps_lce_merge_kernel(const LceParams prm)
{
    after_the_kernel_before();
    constexpr int kSets = kMergeThreads / ROWS;  // of tiles
    __shared__ float2 parts[kMergeThreads / 32][ROWS];
    const int w = blockIdx.y, count = prm.count[w], lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int blocks = (count + ROWS - 1) / ROWS;
    if ((int)blockIdx.x >= blocks) return;
    const int i = blockIdx.x * ROWS + threadIdx.x % ROWS;
    float top = -INFINITY, sum = 0.0f;
    const auto join = [&](float2 p) {
        const float m = fmaxf(top, p.x), at = m == -INFINITY ? 0.0f : m;
        const float factor = TOP ? prm.sharpness : 1.0f;
        sum = sum * __expf((top - at) * factor) + p.y * __expf((p.x - at) * factor);
        top = m;
    };
    if (i < count) {
        const float2* part = prm.part + w * prm.stat_tiles * prm.tokens_padded + i;
        constexpr int kAtATime = 8;
        for (int64_t v = threadIdx.x / ROWS; v < prm.stat_tiles; v += kSets * kAtATime) {
            float2 p[kAtATime];
#pragma unroll
            for (int k = 0; k < kAtATime; ++k)
                p[k] = v + k * kSets < prm.stat_tiles ? __ldcs(part + (v + k * kSets) * prm.tokens_padded) : make_float2(-INFINITY, 0.0f);
#pragma unroll
            for (int k = 0; k < kAtATime; ++k) join(p[k]);
        }
    }
#pragma unroll
    for (int s = ROWS; s < 32; s *= 2) join(make_float2(__shfl_xor_sync(0xFFFFFFFFu, top, s), __shfl_xor_sync(0xFFFFFFFFu, sum, s)));
    if (lane < ROWS) parts[warp][lane] = make_float2(top, sum);
    __syncthreads();
    if (warp != 0) return;
    // each lane some of the warps' pairs of a row, then the lanes of the row
    top = -INFINITY, sum = 0.0f;
#pragma unroll
    for (int k = 0; k < ROWS * kMergeThreads / 32 / 32; ++k) join(parts[lane / ROWS + k * (32 / ROWS)][lane % ROWS]);
#pragma unroll
    for (int s = ROWS; s < 32; s *= 2) join(make_float2(__shfl_xor_sync(0xFFFFFFFFu, top, s), __shfl_xor_sync(0xFFFFFFFFu, sum, s)));
    float loss = 0.0f, apart = 0.0f;
    const float lse = TOP ? top + prm.factor * logf(sum) : top + logf(sum);
    if constexpr (TOP) {
        // the lanes of a row share its entries
        if (i < count) {
            const int64_t first = (w * prm.tokens + prm.rows[w * prm.tokens + i]) * prm.top;
#pragma unroll 4
            for (int e = lane / ROWS; e < prm.top; e += 32 / ROWS) {
                const float q = prm.entry_weight[first + e], z = prm.entry_logit[first + e];
                apart = q != 0.0f ? fmaf(q, fmaf(top - z, prm.sharpness, logf(q * sum)), apart) : apart;  // the logits of the others are not there
            }
        }
#pragma unroll
        for (int s = ROWS; s < 32; s *= 2) apart += __shfl_xor_sync(0xFFFFFFFFu, apart, s);
    }
    if (i < count && lane < ROWS) {
        const int64_t t = prm.rows[w * prm.tokens + i];
        loss = TOP ? prm.factor * prm.factor * apart : lse - prm.hit[w * prm.tokens_padded + i];
        if (TOP && prm.targets[w * prm.tokens + t] < 0) loss = nanf("");  // its entries are no distribution
        prm.lse[w * prm.tokens + t] = lse;
        if (prm.reduction == RPS_REDUCE_NONE) prm.loss[w * prm.tokens + t] = loss;
    }
    if (prm.reduction == RPS_REDUCE_NONE) return;
    for (int s = 16; s > 0; s /= 2) loss += __shfl_xor_sync(0xFFFFFFFFu, loss, s);
    float* sums = prm.sums + w * gridDim.x;
    int before = 0;
    if (lane == 0) {
        sums[blockIdx.x] = loss;
        __threadfence();
        before = atomicAdd(&prm.done[w], 1);
        __threadfence();
    }
    if (__shfl_sync(0xFFFFFFFFu, before, 0) != blocks - 1) return;
    double all = 0.0;
    for (int b = lane; b < blocks; b += 32) all += (double)__ldcg(&sums[b]);
    for (int s = 16; s > 0; s /= 2) all += __shfl_xor_sync(0xFFFFFFFFu, all, s);
    if (prm.reduction == RPS_REDUCE_MEAN) all /= (double)count;
    if (lane == 0) prm.loss[w] = (float)all;
}

template <typename T, bool SELECT>
cudaError_t gather(const LceParams& prm, cudaStream_t stream)
{
    const int64_t rows = ceil_div(round_up(prm.tokens, kTokenBlock), kRowThreads / 32), places = kSms * 4;
    // few rows share their columns out, instead of a warp's turns along each (4 workers of 42 rows of 2530 fp32: 25 -> 6.5 us)
    const int64_t along = std::max<int64_t>(1, std::min(ceil_div(prm.cols_padded, 256), places / (rows * prm.n)));
    const dim3 grid((unsigned)rows, (unsigned)prm.n, (unsigned)along);
    const int align = aligned_source<T>(prm.hidden, prm.cols, prm.hidden_row, prm.hidden_worker);
    const auto kernel = align == 16  ? rps_lce_gather_kernel<T, 16, SELECT>
                        : align == 4 ? rps_lce_gather_kernel<T, 4, SELECT>
                                     : rps_lce_gather_kernel<T, sizeof(T), SELECT>;
    return launch_after(kernel, grid, kRowThreads, 0, stream, 1, prm);
}

template <typename T>
cudaError_t planes(const PlanesParams& prm, cudaStream_t stream)
{
    int sms = 0;
    cudaError_t err = sm_count(&sms);
    if (err != cudaSuccess) return err;
    const int64_t blocks = ceil_div(prm.rows * (prm.dst_row / 8), kRowThreads), resident = ceil_div((int64_t)sms * 8, prm.n);
    const dim3 grid((unsigned)(blocks < resident ? blocks : resident), (unsigned)prm.n);
    const int align = aligned_source<T>(prm.src, prm.cols, prm.src_row, prm.src_worker);
    const auto kernel = align == 16 ? rps_planes_kernel<T, 16> : align == 4 ? rps_planes_kernel<T, 4> : rps_planes_kernel<T, sizeof(T)>;
    return launch_after(kernel, grid, kRowThreads, 0, stream, 1, prm);
}

}  // namespace

cudaError_t launch_lce_rows(const LceParams& prm, cudaStream_t stream)
{
    if (prm.tokens > 0 && prm.tokens <= kFewTokens) return prm.f32 ? gather<float, true>(prm, stream) : gather<bf16, true>(prm, stream);
    const cudaError_t err = launch_after(rps_lce_select_kernel, dim3((unsigned)prm.n), kSelectThreads, 0, stream, 1, prm);
    if (err != cudaSuccess || prm.tokens == 0) return err;
    return prm.f32 ? gather<float, false>(prm, stream) : gather<bf16, false>(prm, stream);
}

int64_t lce_merge_blocks(int64_t tokens) { return ceil_div(tokens, kMergeRows); }

cudaError_t launch_lce_merge(const LceParams& prm, cudaStream_t stream)
{
    const int64_t many = ceil_div(prm.tokens, kManyMergeRows);
    if (many * prm.n >= kSms) {
        const auto kernel = prm.top > 0 ? rps_lce_merge_kernel<kManyMergeRows, true> : rps_lce_merge_kernel<kManyMergeRows, false>;
        return launch_after(kernel, dim3((unsigned)many, (unsigned)prm.n), kMergeThreads, 0, stream, 1, prm);
    }
    const auto kernel = prm.top > 0 ? rps_lce_merge_kernel<kMergeRows, true> : rps_lce_merge_kernel<kMergeRows, false>;
    return launch_after(kernel, dim3((unsigned)lce_merge_blocks(prm.tokens), (unsigned)prm.n), kMergeThreads, 0, stream, 1, prm);
}

// A launch counts its pieces of 16 bytes in 32 bits, so a matrix of 64 GiB and more takes several.
cudaError_t launch_planes(const PlanesParams& prm, cudaStream_t stream)
{
    const int64_t most = ((1ll << 32) - 1) / (prm.dst_row / 8);
    for (int64_t row = 0; row < prm.rows; row += most) {
        PlanesParams q = prm;
        q.rows = std::min(most, prm.rows - row);
        q.src = static_cast<const unsigned char*>(prm.src) + row * prm.src_row * (prm.f32 ? 4 : 2), q.dst = prm.dst + row * prm.dst_row;
        const cudaError_t err = q.f32 ? planes<float>(q, stream) : planes<bf16>(q, stream);
        if (err != cudaSuccess) return err;
    }
    return cudaSuccess;
}

}  // namespace rps_ops
