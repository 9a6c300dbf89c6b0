// The step between two blocks of a network: norm, gate, residual scale, residual sum, norm; forward and backward.
#include "rps_ops_kernels.h"

namespace rps_ops {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float block_sum(float v, float* buf)
{
    for (int s = 16; s > 0; s /= 2) v += __shfl_xor_sync(0xFFFFFFFFu, v, s);
    __syncthreads();
    if (threadIdx.x % 32 == 0) buf[threadIdx.x / 32] = v;
    __syncthreads();
    v = 0.0f;
    for (int i = 0; i < kThreads / 32; ++i) v += buf[i];
    return v;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) rps_norm_forward_kernel(const NormParams prm)
{
    extern __shared__ float hrow[];
    __shared__ float buf[kThreads / 32];
    const int64_t row = blockIdx.x, w = row / prm.tokens, t = row % prm.tokens, D = prm.cols;
    const T* x = static_cast<const T*>(prm.x) + row * D;
    const T* f = static_cast<const T*>(prm.f) + row * D;
    const T* gate = static_cast<const T*>(prm.gate) + w * prm.gate_worker + t / prm.rows_per_gate * D;
    const T* post = static_cast<const T*>(prm.post) + w * prm.post_worker;
    const T* pre = static_cast<const T*>(prm.pre) + w * prm.pre_worker;
    float s = 0.0f;
    for (int64_t c = threadIdx.x; c < D; c += kThreads) {
        const float v = to_float<T>(f[c]);
        s = fmaf(v, v, s);
    }
    const float r_f = rsqrtf(block_sum(s, buf) / (float)D + prm.eps);
    s = 0.0f;
    for (int64_t c = threadIdx.x; c < D; c += kThreads) {
        const float u = to_float<T>(f[c]) * r_f * to_float<T>(post[c]);
        const float h = fmaf(prm.scale * to_float<T>(gate[c]), u, to_float<T>(x[c]));
        static_cast<T*>(prm.h)[row * D + c] = from_float<T>(h);
        hrow[c] = h;
        s = fmaf(h, h, s);
    }
    const float r_h = rsqrtf(block_sum(s, buf) / (float)D + prm.eps);
    for (int64_t c = threadIdx.x; c < D; c += kThreads)
        static_cast<T*>(prm.y)[row * D + c] = from_float<T>(hrow[c] * r_h * to_float<T>(pre[c]));
    if (threadIdx.x == 0 && prm.r_f != nullptr) {
        prm.r_f[row] = r_f;
        prm.r_h[row] = r_h;
    }
}

template <typename T>
__device__ __forceinline__ float kept(const void* values, const float* scales, const NormParams& prm, int64_t row, int64_t c)
{
    if (scales == nullptr) return to_float<T>(static_cast<const T*>(values)[row * prm.cols + c]);
    return (float)static_cast<const int8_t*>(values)[row * prm.pitch + c] * scales[row * prm.groups + c / RPS_PACK_GROUP];
}

template <typename T>
__global__ void __launch_bounds__(kThreads) rps_norm_backward_kernel(const NormParams prm)
{
    extern __shared__ float trow[];
    __shared__ float buf[kThreads / 32];
    const int64_t D = prm.cols, w = blockIdx.y, block = blockIdx.x;
    int64_t first, end;
    if (prm.chunks > 0) {
        const int64_t g = block / prm.chunks;
        first = g * prm.rows_per_gate + block % prm.chunks * prm.rows_per_block;
        end = min(first + prm.rows_per_block, (g + 1) * prm.rows_per_gate);
    } else {
        first = block * prm.rows_per_block;
        end = min(first + prm.rows_per_block, prm.tokens);
    }
    const T* post = static_cast<const T*>(prm.post) + w * prm.post_worker;
    const T* pre = static_cast<const T*>(prm.pre) + w * prm.pre_worker;
    float* partial = prm.partial + (w * prm.blocks + block) * 3 * D;
    for (int64_t c = threadIdx.x; c < 3 * D; c += kThreads) partial[c] = 0.0f;
    __syncthreads();
    for (int64_t t = first; t < end; ++t) {
        const int64_t row = w * prm.tokens + t;
        const T* gate = static_cast<const T*>(prm.gate) + w * prm.gate_worker + t / prm.rows_per_gate * D;
        const float r_f = prm.r_f[row], r_h = prm.r_h[row];
        float s = 0.0f;
        for (int64_t c = threadIdx.x; c < D; c += kThreads)
            s = fmaf(to_float<T>(static_cast<const T*>(prm.dy)[row * D + c]) * to_float<T>(pre[c]), kept<T>(prm.h_in, prm.h_scales, prm, row, c), s);
        const float mean_h = block_sum(s, buf) / (float)D * r_h * r_h;
        s = 0.0f;
        for (int64_t c = threadIdx.x; c < D; c += kThreads) {
            const float h = kept<T>(prm.h_in, prm.h_scales, prm, row, c), f = kept<T>(prm.f, prm.f_scales, prm, row, c);
            const float dy = to_float<T>(static_cast<const T*>(prm.dy)[row * D + c]);
            float v = r_h * (dy * to_float<T>(pre[c]) - h * mean_h);
            if (prm.dh != nullptr) v += to_float<T>(static_cast<const T*>(prm.dh)[row * D + c]);
            static_cast<T*>(prm.dx)[row * D + c] = from_float<T>(v);
            trow[c] = v;
            const float du = prm.scale * to_float<T>(gate[c]) * v;
            s = fmaf(du * to_float<T>(post[c]), f, s);
            partial[c] += du * f * r_f;
            partial[D + c] += dy * h * r_h;
            partial[2 * D + c] += prm.scale * v * f * r_f * to_float<T>(post[c]);
        }
        const float mean_f = block_sum(s, buf) / (float)D * r_f * r_f;
        for (int64_t c = threadIdx.x; c < D; c += kThreads) {
            const float f = kept<T>(prm.f, prm.f_scales, prm, row, c);
            const float b = prm.scale * to_float<T>(gate[c]) * trow[c] * to_float<T>(post[c]);
            static_cast<T*>(prm.df)[row * D + c] = from_float<T>(r_f * (b - f * mean_f));
        }
        if (prm.chunks == 0 && (t + 1) % prm.rows_per_gate == 0) {  // the block holds the whole gate group
            for (int64_t c = threadIdx.x; c < D; c += kThreads) {
                static_cast<T*>(prm.dgate)[(w * prm.gates + t / prm.rows_per_gate) * D + c] = from_float<T>(partial[2 * D + c]);
                partial[2 * D + c] = 0.0f;
            }
        }
    }
}

// Sums of the blocks' partial sums, a thread for each column, always in the same order.
template <typename T>
__global__ void __launch_bounds__(128) rps_norm_reduce_kernel(const NormParams prm)
{
    const int64_t c = (int64_t)blockIdx.x * 128 + threadIdx.x, w = blockIdx.y, D = prm.cols, job = blockIdx.z;
    if (c >= D) return;
    const float* partial = prm.partial + w * prm.blocks * 3 * D + c;
    float s = 0.0f;
    if (job < 2) {
        for (int64_t b = 0; b < prm.blocks; ++b) s += partial[(3 * b + job) * D];
        static_cast<T*>(job == 0 ? prm.dpost : prm.dpre)[w * D + c] = from_float<T>(s);
    } else {
        const int64_t g = job - 2;
        for (int64_t b = g * prm.chunks; b < (g + 1) * prm.chunks; ++b) s += partial[(3 * b + 2) * D];
        static_cast<T*>(prm.dgate)[(w * prm.gates + g) * D + c] = from_float<T>(s);
    }
}

template <typename T>
cudaError_t backward(const NormParams& prm, cudaStream_t stream)
{
    cudaError_t err = cudaFuncSetAttribute(rps_norm_backward_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, RPS_MAX_NORM_COLS * 4);
    if (err != cudaSuccess) return err;
    rps_norm_backward_kernel<T><<<dim3((unsigned)prm.blocks, (unsigned)prm.n), kThreads, prm.cols * 4, stream>>>(prm);
    rps_norm_reduce_kernel<T><<<dim3((unsigned)ceil_div(prm.cols, 128), (unsigned)prm.n, (unsigned)(2 + (prm.chunks > 0 ? prm.gates : 0))), 128, 0, stream>>>(prm);
    return cudaGetLastError();
}

template <typename T>
cudaError_t forward(const NormParams& prm, cudaStream_t stream)
{
    cudaError_t err = cudaFuncSetAttribute(rps_norm_forward_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, RPS_MAX_NORM_COLS * 4);
    if (err != cudaSuccess) return err;
    rps_norm_forward_kernel<T><<<(unsigned)(prm.n * prm.tokens), kThreads, prm.cols * 4, stream>>>(prm);
    if ((err = cudaGetLastError()) != cudaSuccess || prm.f_codes == nullptr) return err;
    PackParams pack{};
    pack.f32 = prm.f32;
    pack.rows = prm.n * prm.tokens;
    pack.cols = pack.x_row = prm.cols;
    pack.pitch = prm.pitch;
    pack.groups = prm.groups;
    pack.x = prm.f, pack.codes = prm.f_codes, pack.scales = prm.f_scales;
    if ((err = launch_pack(pack, stream)) != cudaSuccess) return err;
    pack.x = prm.h, pack.codes = prm.h_codes, pack.scales = prm.h_scales;
    return launch_pack(pack, stream);
}

}  // namespace

void plan_norm_backward(NormParams* prm)
{
    // about four blocks per SM over all workers
    const int64_t want = ceil_div(148 * 4, prm->n), rows = prm->rows_per_gate;
    const int64_t target = prm->tokens / want > 0 ? prm->tokens / want : 1;
    if (rows <= target) {
        prm->chunks = 0;
        prm->rows_per_block = target / rows * rows;
        prm->blocks = ceil_div(prm->tokens, prm->rows_per_block);
    } else {
        prm->rows_per_block = target;
        prm->chunks = ceil_div(rows, target);
        prm->blocks = prm->gates * prm->chunks;
    }
}

cudaError_t launch_norm_forward(const NormParams& prm, cudaStream_t stream)
{
    return prm.f32 ? forward<float>(prm, stream) : forward<bf16>(prm, stream);
}

cudaError_t launch_norm_backward(const NormParams& prm, cudaStream_t stream)
{
    return prm.f32 ? backward<float>(prm, stream) : backward<bf16>(prm, stream);
}

}  // namespace rps_ops
