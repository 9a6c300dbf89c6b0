// The loss of a few tokens.  Logits of a few tokens a worker are dot products of the weight's rows with their hidden states, and
// their gradients are multiples of rows: each pass reads (or writes) the weight as it is, once, and memory bounds it.  The tensor
// cores would make 128 rows for them, and would have fp32 weights and rows that no 16 bytes divide laid out anew first.
//
// Up to 4 tokens of bf16 and 8 of fp32 (forward and backward, tensor cores / here, us): 1 token x 131072 x 2048 bf16 467 / 409, 4 tokens
// 467 / 451; 8 workers of 3 x 5000 x 4096 bf16 303 / 307, of 3 x 1000 x 256 39 / 25; 4 of 1 x 31046 x 1313 bf16 764 / 347; 4 of 8 x 17081 x
// 1000 fp32 800 / 322; 1 x 1000 x 256 fp32 60 / 20.  More tokens would hold more sums than registers allow, for less gain.
// Logits run at 5.0 TB/s (1 token) to 4.7 (4), the gradients' pass over weight and gradient at 5.6.
#include "rps_kernels.h"
#include "rps_lce.cuh"

namespace rps_ops {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMostTokens = 4, kMostTokensF32 = 8;  // see above
constexpr int kMostHiddenBytes = 100 * 1024;  // of hidden states in shared memory, of two CTAs on an SM

// 16 bytes of a row for each lane: a lane's columns are next to each other, or (rows that are not 16-byte aligned) a warp's
// width apart, so that the lanes of each load are next to each other.
template <typename T>
constexpr int kCols = 16 / (int)sizeof(T);
template <typename T>
constexpr int kChunk = 32 * kCols<T>;  // of a warp

template <typename T, bool WIDE>
struct RowPart {  // as loaded: what lies ahead takes few registers
    uint4 bits;
    __device__ __forceinline__ void load(const T* row, int c0, int lane, int cols)
    {
        const int c = c0 + lane * kCols<T>;
        bits = c < cols ? __ldg(reinterpret_cast<const uint4*>(row + c)) : make_uint4(0, 0, 0, 0);
    }
    __device__ __forceinline__ void values(Pair (&v)[kCols<T> / 2]) const { widen(bits, v); }
};

template <typename T>
struct RowPart<T, false> {
    T e[kCols<T>];
    __device__ __forceinline__ void load(const T* row, int c0, int lane, int cols)
    {
#pragma unroll
        for (int j = 0; j < kCols<T>; ++j) {
            const int c = c0 + lane + 32 * j;
            e[j] = c < cols ? __ldg(row + c) : from_float<T>(0.0f);
        }
    }
    __device__ __forceinline__ void values(Pair (&v)[kCols<T> / 2]) const
    {
#pragma unroll
        for (int j = 0; j < kCols<T> / 2; ++j) v[j] = Pair(to_float<T>(e[2 * j]), to_float<T>(e[2 * j + 1]));
    }
};

template <typename T, bool WIDE>
__device__ __forceinline__ void store_columns(T* row, int c0, int lane, int cols, const Pair (&v)[kCols<T> / 2])
{
    if constexpr (WIDE) {
        const int c = c0 + lane * kCols<T>;
        if (c < cols) __stcs(reinterpret_cast<uint4*>(row + c), narrow(v));
    } else {
#pragma unroll
        for (int j = 0; j < kCols<T>; ++j) {
            float e[2];
            v[j / 2].get(e[0], e[1]);
            const int c = c0 + lane + 32 * j;
            if (c < cols) row[c] = from_float<T>(e[j % 2]);
        }
    }
}

// The same columns of a token's hidden state, zero for token -1.
template <typename T, bool WIDE>
__device__ __forceinline__ void hidden_columns(const LceParams& prm, int w, int token, int c0, int lane, float (&e)[kCols<T>])
{
    const T* row = static_cast<const T*>(prm.hidden) + w * prm.hidden_worker + max(token, 0) * prm.hidden_row;
#pragma unroll
    for (int j = 0; j < kCols<T>; ++j) {
        const int c = WIDE ? c0 + lane * kCols<T> + j : c0 + lane + 32 * j;
        e[j] = token >= 0 && c < prm.cols ? to_float<T>(__ldg(row + c)) : 0.0f;
    }
}

// Sums over the lanes of N values of each, a power of two of at most 32: half of the values to each half of the lanes, and so
// on.  Lane l has number l / (32 / N)'s in x[0].
template <int N>
__device__ __forceinline__ void sum_over_lanes(float (&x)[N], int lane)
{
    int left = N;
#pragma unroll
    for (int s = 16; s > 0; s /= 2) {
        if (left > 1) {
            left /= 2;
            const bool upper = (lane & s) != 0;
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                if (i >= left) break;
                const float mine = upper ? x[i + left] : x[i], other = upper ? x[i] : x[i + left];
                x[i] = mine + __shfl_xor_sync(0xFFFFFFFFu, other, s);
            }
        } else {
            x[0] += __shfl_xor_sync(0xFFFFFFFFu, x[0], s);
        }
    }
}

// Of the weight, by a warp: with 8 a worker of 5000 rows leaves most warps waiting in the last turn (8 workers of 2 tokens x 4096: 98 us
// against 74), and the next rows' loads on their way under the sums take registers that more warps use better (67 against 74).
constexpr int kRowsAtATime = 4;
template <int ROWS>
constexpr int kResident = ROWS <= 2 ? 3 : 2;  // CTAs on an SM

// A warp takes rows of the weight, all tokens' products with each at once; the hidden states lie in shared memory as fp32.  Forward: the
// CTA's maximum and sum of exponentials of each token for rps_lce_merge_kernel; backward: dl.
template <typename T, bool WIDE, int ROWS, bool BACKWARD>
__global__ void __launch_bounds__(kThreads, kResident<ROWS>) rps_lce_dot_kernel(const LceParams prm)
{
    constexpr int kR = kRowsAtATime, kValues = kR * ROWS, kPairs = kCols<T> / 2;
    extern __shared__ float4 hidden[];  // [ROWS][chunk][kCols / 4][lane]
    __shared__ int row_of[ROWS];
    __shared__ float2 statistics[kWarps][kValues];
    after_the_kernel_before();
    const int w = blockIdx.y, lane = threadIdx.x % 32, warp = threadIdx.x / 32, D = (int)prm.cols, V = (int)prm.vocab;
    const int chunks = (D + kChunk<T> - 1) / kChunk<T>;
    const int count = select_tokens<kThreads>(prm, w, blockIdx.x == 0, row_of);
#pragma unroll 2
    for (int i = warp; i < ROWS * chunks; i += kWarps) {
        const int q = i / chunks, c0 = (i - q * chunks) * kChunk<T>;
        float e[kCols<T>];
        hidden_columns<T, WIDE>(prm, w, q < count ? row_of[q] : -1, c0, lane, e);
#pragma unroll
        for (int p = 0; p < kCols<T>; p += 4) hidden[(i * (kCols<T> / 4) + p / 4) * 32 + lane] = make_float4(e[p], e[p + 1], e[p + 2], e[p + 3]);
    }
    if (BACKWARD && blockIdx.x == 0) {  // ignored tokens' gradients
        for (int i = count; i < prm.tokens; ++i)
            for (int c = threadIdx.x; c < D; c += kThreads) static_cast<T*>(prm.dhidden)[(w * prm.tokens + row_of[i]) * prm.cols + c] = from_float<T>(0.0f);
    }
    // this lane's share of the sums: token t's product with row r of those that the warp has in hand
    const int value = lane / (32 / kValues), r = value / ROWS, t = value % ROWS;
    const bool first = lane % (32 / kValues) == 0, in = t < count;
    const int64_t token = in ? w * prm.tokens + row_of[t] : 0;
    const int64_t y = in ? prm.targets[token] : 0;
    const int target = in && y >= 0 && y < V ? (int)y : -1;
    float lse = 0.0f, g = 0.0f, top = -INFINITY, sum = 0.0f;
    if (BACKWARD && in) {
        lse = prm.lse_in[token];
        g = target < 0 ? nanf("") : prm.reduction == RPS_REDUCE_NONE ? prm.dloss[token] : 1.0f;
    }
    __syncthreads();
    const T* weight = static_cast<const T*>(prm.weight) + w * prm.weight_worker;
    const int each = (V + gridDim.x * kWarps - 1) / (gridDim.x * kWarps), start = min(V, (blockIdx.x * kWarps + warp) * each), end = min(V, start + each);
    for (int v0 = start; v0 < end; v0 += kR) {
        Pair acc[kValues];
#pragma unroll
        for (int i = 0; i < kValues; ++i) acc[i] = Pair(0.0f);
#pragma unroll 2
        for (int k = 0; k < chunks; ++k) {
            RowPart<T, WIDE> part[kR];
#pragma unroll
            for (int i = 0; i < kR; ++i) part[i].load(weight + min(v0 + i, end - 1) * prm.weight_row, k * kChunk<T>, lane, D);
            Pair h[ROWS][kPairs];
#pragma unroll
            for (int q = 0; q < ROWS; ++q)
#pragma unroll
                for (int p = 0; p < kPairs; p += 2) {
                    const float4 s = hidden[((q * chunks + k) * (kPairs / 2) + p / 2) * 32 + lane];
                    h[q][p] = Pair(s.x, s.y), h[q][p + 1] = Pair(s.z, s.w);
                }
#pragma unroll
            for (int i = 0; i < kR; ++i) {
                Pair v[kPairs];
                part[i].values(v);
#pragma unroll
                for (int q = 0; q < ROWS; ++q)
#pragma unroll
                    for (int p = 0; p < kPairs; ++p) acc[i * ROWS + q] = fma(v[p], h[q][p], acc[i * ROWS + q]);
            }
        }
        float logit[kValues];
#pragma unroll
        for (int i = 0; i < kValues; ++i) logit[i] = acc[i].sum();
        sum_over_lanes(logit, lane);
        const int at = v0 + r;
        const float l = logit[0];
        if (at >= end) continue;
        if constexpr (BACKWARD) {
            const float p = exp_of_difference(l, lse) - (at == target ? 1.0f : 0.0f);
            if (first) prm.dot_dl[((int64_t)w * V + at) * ROWS + t] = in ? g * p : 0.0f;
        } else if (in) {
            if (at == target && first) const_cast<float*>(prm.hit)[w * prm.tokens_padded + t] = l;
            const float m = fmaxf(top, l), from = m == -INFINITY ? 0.0f : m;
            sum = fmaf(sum, __expf(top - from), __expf(l - from));
            top = m;
        }
    }
    if constexpr (!BACKWARD) {
        if (first) statistics[warp][value] = make_float2(top, sum);
        __syncthreads();
        if (threadIdx.x < count) {
            top = -INFINITY, sum = 0.0f;
            for (int i = 0; i < kWarps * kR; ++i) {
                const float2 p = statistics[i / kR][i % kR * ROWS + threadIdx.x];
                const float m = fmaxf(top, p.x), from = m == -INFINITY ? 0.0f : m;
                sum = sum * __expf(top - from) + p.y * __expf(p.x - from);
                top = m;
            }
            const_cast<float2*>(prm.part)[((int64_t)w * prm.stat_tiles + blockIdx.x) * prm.tokens_padded + threadIdx.x] = make_float2(top, sum);
        }
    }
}

template <int ROWS>
__device__ __forceinline__ void load_dl(const float* p, float (&d)[ROWS])
{
    if constexpr (ROWS == 1) {
        d[0] = __ldg(p);
    } else if constexpr (ROWS == 2) {
        const float2 a = __ldg(reinterpret_cast<const float2*>(p));
        d[0] = a.x, d[1] = a.y;
    } else {
#pragma unroll
        for (int i = 0; i < ROWS; i += 4) {
            const float4 a = __ldg(reinterpret_cast<const float4*>(p + i));
            d[i] = a.x, d[i + 1] = a.y, d[i + 2] = a.z, d[i + 3] = a.w;
        }
    }
}

// Both gradients in one pass over a range of the vocabulary.  A lane keeps its columns of the hidden states and of dhidden's sum; warps side
// by side along the rows, the others take rows in turn.
template <typename T, bool WIDE, int ROWS>
__global__ void __launch_bounds__(kThreads, 2) rps_lce_dot_grads_kernel(const LceParams prm)
{
    constexpr int kPairs = kCols<T> / 2, kAtATime = ROWS == 8 ? 2 : 4;
    __shared__ float sums[kWarps][kChunk<T>];
    after_the_kernel_before();
    const int w = blockIdx.z, lane = threadIdx.x % 32, warp = threadIdx.x / 32, D = (int)prm.cols;
    const int beside = warp % prm.dot_wide, turn = warp / prm.dot_wide, high = prm.dot_high;
    const int c0 = (blockIdx.x * prm.dot_wide + beside) * kChunk<T>;  // may be past the last column
    const int range = ((int)prm.vocab + gridDim.y - 1) / gridDim.y, end = min((int)prm.vocab, ((int)blockIdx.y + 1) * range);
    const int count = prm.count[w];
    const float scale = prm.scale[w];
    Pair h[ROWS][kPairs], acc[ROWS][kPairs];
#pragma unroll
    for (int q = 0; q < ROWS; ++q) {
        float e[kCols<T>];
        hidden_columns<T, WIDE>(prm, w, q < count ? prm.rows[w * prm.tokens + q] : -1, c0, lane, e);
#pragma unroll
        for (int j = 0; j < kPairs; ++j) h[q][j] = Pair(e[2 * j], e[2 * j + 1]), acc[q][j] = Pair(0.0f);
    }
    const T* weight = static_cast<const T*>(prm.weight) + w * prm.weight_worker;
    T* dweight = static_cast<T*>(prm.dweight) + w * prm.dweight_worker;
    const float* dl = prm.dot_dl + w * prm.vocab * ROWS;
    for (int v0 = blockIdx.y * range + turn; v0 < end; v0 += kAtATime * high) {
        RowPart<T, WIDE> from[kAtATime];
        float d[kAtATime][ROWS];
#pragma unroll
        for (int i = 0; i < kAtATime; ++i) {
            const int at = v0 + i * high;
            from[i].load(weight + min(at, end - 1) * prm.weight_row, c0, lane, at < end ? D : 0);
            load_dl(dl + (int64_t)min(at, end - 1) * ROWS, d[i]);
        }
#pragma unroll
        for (int i = 0; i < kAtATime; ++i) {
            const int at = v0 + i * high;
            if (at >= end) break;
            Pair v[kPairs], out[kPairs];
            from[i].values(v);
#pragma unroll
            for (int j = 0; j < kPairs; ++j) {
                out[j] = Pair(d[i][0]) * h[0][j];
                acc[0][j] = fma(Pair(d[i][0]), v[j], acc[0][j]);
#pragma unroll
                for (int q = 1; q < ROWS; ++q) {
                    out[j] = fma(Pair(d[i][q]), h[q][j], out[j]);
                    acc[q][j] = fma(Pair(d[i][q]), v[j], acc[q][j]);
                }
                out[j] = out[j] * Pair(scale);
            }
            store_columns<T, WIDE>(dweight + at * prm.dweight_row, c0, lane, D, out);
        }
    }
    const int64_t part_row = (prm.cols + 3) / 4 * 4;
#pragma unroll
    for (int q = 0; q < ROWS; ++q) {
        float e[kCols<T>];
#pragma unroll
        for (int j = 0; j < kPairs; ++j) acc[q][j].get(e[2 * j], e[2 * j + 1]);
        if (high > 1) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < kCols<T>; ++j) sums[warp][j * 32 + lane] = e[j];
            __syncthreads();
            if (turn > 0) continue;
            for (int k = 1; k < high; ++k)
#pragma unroll
                for (int j = 0; j < kCols<T>; ++j) e[j] += sums[beside + k * prm.dot_wide][j * 32 + lane];
        }
        if (q >= count) continue;
        float* part = prm.dot_parts + (((int64_t)blockIdx.y * prm.n + w) * ROWS + q) * part_row;
#pragma unroll
        for (int j = 0; j < kCols<T>; ++j) {
            const int c = WIDE ? c0 + lane * kCols<T> + j : c0 + lane + 32 * j;
            if (c < D) part[c] = e[j];
        }
    }
}

template <typename T>
int chunks_of(int64_t cols)
{
    return (int)ceil_div(cols, kChunk<T>);
}

template <typename T, bool WIDE, int ROWS, bool BACKWARD>
cudaError_t logits(const LceParams& prm, cudaStream_t stream)
{
    static rps::LaunchState state;
    const size_t bytes = (size_t)ROWS * chunks_of<T>(prm.cols) * kChunk<T> * sizeof(float);
    const cudaError_t err = rps::grant_smem(state, rps_lce_dot_kernel<T, WIDE, ROWS, BACKWARD>, (uint32_t)bytes);
    if (err != cudaSuccess) return err;
    return launch_after(rps_lce_dot_kernel<T, WIDE, ROWS, BACKWARD>, dim3((unsigned)prm.dot_blocks, (unsigned)prm.n), kThreads, bytes, stream, 1, prm);
}

template <typename T, int ROWS>
cudaError_t logits(const LceParams& prm, cudaStream_t stream)
{
    const bool wide = aligned_source<T>(prm.weight, prm.cols, prm.weight_row, prm.weight_worker) == 16;
    if (prm.backward) return wide ? logits<T, true, ROWS, true>(prm, stream) : logits<T, false, ROWS, true>(prm, stream);
    return wide ? logits<T, true, ROWS, false>(prm, stream) : logits<T, false, ROWS, false>(prm, stream);
}

template <typename T, int ROWS>
cudaError_t grads(const LceParams& prm, cudaStream_t stream)
{
    const bool wide = aligned_source<T>(prm.weight, prm.cols, prm.weight_row, prm.weight_worker) == 16 &&
                      aligned_source<T>(prm.dweight, prm.cols, prm.dweight_row, prm.dweight_worker) == 16;
    const dim3 grid((unsigned)ceil_div(chunks_of<T>(prm.cols), prm.dot_wide), (unsigned)prm.dot_ranges, (unsigned)prm.n);
    const auto kernel = wide ? rps_lce_dot_grads_kernel<T, true, ROWS> : rps_lce_dot_grads_kernel<T, false, ROWS>;
    return launch_after(kernel, grid, 32 * prm.dot_wide * prm.dot_high, 0, stream, 1, prm);
}

}  // namespace

void plan_lce_dot(LceParams* prm)
{
    prm->dot_rows = 0;
    const int rows = prm->tokens <= 1 ? 1 : prm->tokens <= 2 ? 2 : prm->tokens <= 4 ? 4 : 8;
    const int chunks = prm->f32 ? chunks_of<float>(prm->cols) : chunks_of<bf16>(prm->cols), chunk = prm->f32 ? kChunk<float> : kChunk<bf16>;
    if (prm->tokens < 1 || prm->tokens > (prm->f32 ? kMostTokensF32 : kMostTokens) || (int64_t)rows * chunks * chunk * 4 > kMostHiddenBytes) return;
    const auto within = [](int64_t x, int64_t most) { return (int)std::max<int64_t>(1, std::min(x, most)); };
    prm->dot_rows = rows;
    prm->dot_blocks = within(ceil_div(prm->vocab, kWarps * kRowsAtATime), kSms * (rows <= 2 ? kResident<1> : kResident<4>) / prm->n);
    const int across = (int)ceil_div(chunks, kWarps);
    prm->dot_wide = (int)ceil_div(chunks, across), prm->dot_high = kWarps / prm->dot_wide;
    prm->dot_ranges = within(ceil_div(prm->vocab, 16 * prm->dot_high), 2 * kSms / (across * prm->n));
}

cudaError_t launch_lce_dot(const LceParams& prm, cudaStream_t stream)
{
    switch (prm.dot_rows) {
        case 1: return prm.f32 ? logits<float, 1>(prm, stream) : logits<bf16, 1>(prm, stream);
        case 2: return prm.f32 ? logits<float, 2>(prm, stream) : logits<bf16, 2>(prm, stream);
        case 4: return prm.f32 ? logits<float, 4>(prm, stream) : logits<bf16, 4>(prm, stream);
        default: return logits<float, 8>(prm, stream);
    }
}

cudaError_t launch_lce_dot_grads(const LceParams& prm, cudaStream_t stream)
{
    switch (prm.dot_rows) {
        case 1: return prm.f32 ? grads<float, 1>(prm, stream) : grads<bf16, 1>(prm, stream);
        case 2: return prm.f32 ? grads<float, 2>(prm, stream) : grads<bf16, 2>(prm, stream);
        case 4: return prm.f32 ? grads<float, 4>(prm, stream) : grads<bf16, 4>(prm, stream);
        default: return grads<float, 8>(prm, stream);
    }
}

}  // namespace rps_ops
