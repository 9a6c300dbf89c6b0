// Activations in 8 bits: a scale for each 128 columns of a row.
#include "rps_ops_kernels.h"

namespace rps_ops {
namespace {

constexpr int kGroup = RPS_PACK_GROUP;
constexpr float kSmallest = 0x1p-100f;  // a group with nothing larger is kept as zeros: 127 / max stays finite

// One warp per group, four columns a lane.
template <typename T>
__global__ void __launch_bounds__(256) rps_pack_kernel(const PackParams prm)
{
    const int64_t g = (int64_t)blockIdx.x * 8 + threadIdx.x / 32;
    if (g >= prm.rows * prm.groups) return;
    const int lane = threadIdx.x % 32;
    const int64_t row = g / prm.groups, c0 = g % prm.groups * kGroup + lane * 4;
    const T* x = static_cast<const T*>(prm.x) + row * prm.x_row;
    float v[4], top = 0.0f;
    bool finite = true;
    for (int j = 0; j < 4; ++j) {
        v[j] = c0 + j < prm.cols ? to_float<T>(x[c0 + j]) : 0.0f;
        finite &= fabsf(v[j]) <= 3.402823466e38f;
        top = fmaxf(top, fabsf(v[j]));
    }
    for (int s = 16; s > 0; s /= 2) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, s));
    finite = __all_sync(0xFFFFFFFFu, finite);
    const bool zero = !finite || top < kSmallest;
    const float factor = zero ? 0.0f : __fdiv_rn(127.0f, top);
    for (int j = 0; j < 4; ++j)
        if (c0 + j < prm.pitch) prm.codes[row * prm.pitch + c0 + j] = zero ? 0 : (int8_t)__float2int_rn(__fmul_rn(v[j], factor));
    if (lane == 0) prm.scales[g] = !finite ? nanf("") : zero ? 0.0f : __fmul_rn(top, 1.0f / 127.0f);
}

template <typename T>
__global__ void __launch_bounds__(256) rps_unpack_kernel(const PackParams prm)
{
    const int64_t row = blockIdx.x;
    for (int64_t c = threadIdx.x; c < prm.cols; c += blockDim.x)
        static_cast<T*>(prm.out)[row * prm.x_row + c] =
            from_float<T>(__fmul_rn((float)prm.codes[row * prm.pitch + c], prm.scales[row * prm.groups + c / kGroup]));
}

__global__ void __launch_bounds__(256) rps_unpack_planes_kernel(const PackParams prm)
{
    const int64_t row = blockIdx.x, w = row / prm.tokens;
    bf16* dst = prm.planes_out + w * prm.dst_worker + row % prm.tokens * prm.dst_row;
    for (int64_t c = threadIdx.x; c < prm.dst_row; c += blockDim.x) {
        const float v = c < prm.cols ? __fmul_rn((float)prm.codes[row * prm.pitch + c], prm.scales[row * prm.groups + c / kGroup]) : 0.0f;
        if (prm.planes == 1) {
            dst[c] = __float2bfloat16_rn(v);
        } else {
            bf16 p[3];
            split_planes(v, p);
            for (int q = 0; q < 3; ++q) dst[q * prm.dst_plane + c] = p[q];
        }
    }
}

}  // namespace

cudaError_t launch_pack(const PackParams& prm, cudaStream_t stream)
{
    const unsigned grid = (unsigned)ceil_div(prm.rows * prm.groups, 8);
    if (prm.f32)
        rps_pack_kernel<float><<<grid, 256, 0, stream>>>(prm);
    else
        rps_pack_kernel<bf16><<<grid, 256, 0, stream>>>(prm);
    return cudaGetLastError();
}

cudaError_t launch_unpack(const PackParams& prm, cudaStream_t stream)
{
    if (prm.f32)
        rps_unpack_kernel<float><<<(unsigned)prm.rows, 256, 0, stream>>>(prm);
    else
        rps_unpack_kernel<bf16><<<(unsigned)prm.rows, 256, 0, stream>>>(prm);
    return cudaGetLastError();
}

cudaError_t launch_unpack_planes(const PackParams& prm, cudaStream_t stream)
{
    rps_unpack_planes_kernel<<<(unsigned)prm.rows, 256, 0, stream>>>(prm);
    return cudaGetLastError();
}

}  // namespace rps_ops
