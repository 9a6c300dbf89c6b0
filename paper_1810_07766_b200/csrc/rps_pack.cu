// Activations in 8 bits: a scale for each 128 columns of a row.
//
// Bound by memory.  A unit of work is a warp's worth of slices of one row (256 columns of bf16, 128 of fp32); a warp takes
// kUnits of them at a time, so that their loads are all on their way before the first is used.
#include "rps_rows.cuh"

namespace rps_ops {
namespace {

constexpr int kThreads = 256, kUnits = 4;

struct Place {
    int64_t row;
    int c;
};

// Column of this lane in unit u; units_per_row of them to a row.
template <int W>
__device__ __forceinline__ Place place(uint32_t u, uint32_t units_per_row)
{
    const uint32_t row = u / units_per_row;
    return {row, (int)((u - row * units_per_row) * 32 + threadIdx.x % 32) * W};
}

template <typename T, int ALIGN>
__global__ void __launch_bounds__(kThreads) rps_pack_kernel(const PackParams prm, uint32_t units, uint32_t units_per_row)
{
    after_the_kernel_before();
    constexpr int W = Slice<T>::kWidth;
    const int D = (int)prm.cols;
    const uint32_t warp = blockIdx.x * (kThreads / 32) + threadIdx.x / 32, step = gridDim.x * (kThreads / 32);
    for (uint64_t u0 = warp; u0 < units; u0 += (uint64_t)step * kUnits) {
        uint4 x[kUnits];
        Place at[kUnits];
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
            const uint64_t u = u0 + (uint64_t)i * step;
            if (u >= units) break;
            at[i] = place<W>((uint32_t)u, units_per_row);
            x[i] = load_slice<T, ALIGN, true>(static_cast<const T*>(prm.x) + at[i].row * prm.x_row, at[i].c, D);
        }
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
            if (u0 + (uint64_t)i * step >= units) break;
            const int c = at[i].c;
            float v[W];
            widen(x[i], v);
            pack_slice(v, c < prm.pitch ? prm.codes + at[i].row * prm.pitch + c : nullptr,
                       c < D ? prm.scales + at[i].row * prm.groups + c / RPS_PACK_GROUP : nullptr);
        }
    }
}

template <int W>
__device__ __forceinline__ void load_codes(const PackParams& prm, const Place& at, Codes<W>& codes, float& scale)
{
    codes.clear(), scale = 0.0f;
    if (at.c < prm.cols) {
        codes.load(prm.codes + at.row * prm.pitch + at.c);
        scale = __ldg(prm.scales + at.row * prm.groups + at.c / RPS_PACK_GROUP);
    }
}

template <typename T, int ALIGN>
__global__ void __launch_bounds__(kThreads) rps_unpack_kernel(const PackParams prm, uint32_t units, uint32_t units_per_row)
{
    after_the_kernel_before();
    constexpr int W = Slice<T>::kWidth;
    const uint32_t warp = blockIdx.x * (kThreads / 32) + threadIdx.x / 32, step = gridDim.x * (kThreads / 32);
    for (uint64_t u0 = warp; u0 < units; u0 += (uint64_t)step * kUnits) {
        Codes<W> codes[kUnits];
        float scale[kUnits];
        Place at[kUnits];
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
            const uint64_t u = u0 + (uint64_t)i * step;
            if (u >= units) break;
            at[i] = place<W>((uint32_t)u, units_per_row);
            load_codes(prm, at[i], codes[i], scale[i]);
        }
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
            if (u0 + (uint64_t)i * step >= units) break;
            float v[W];
            codes[i].values(scale[i], v);
            store_slice<T, ALIGN>(static_cast<T*>(prm.out) + at[i].row * prm.x_row, at[i].c, (int)prm.cols, narrow(v));
        }
    }
}

// The values as operands of a product: bf16, or the three bf16 parts of fp32 values; rows of dst_row columns, zero behind the last.
template <typename T>
__global__ void __launch_bounds__(kThreads) rps_unpack_planes_kernel(const PackParams prm, uint32_t units, uint32_t units_per_row)
{
    after_the_kernel_before();
    constexpr int W = 8;
    const uint32_t warp = blockIdx.x * (kThreads / 32) + threadIdx.x / 32, step = gridDim.x * (kThreads / 32);
    for (uint64_t u0 = warp; u0 < units; u0 += (uint64_t)step * kUnits) {
        Codes<W> codes[kUnits];
        float scale[kUnits];
        Place at[kUnits];
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
            const uint64_t u = u0 + (uint64_t)i * step;
            if (u >= units) break;
            at[i] = place<W>((uint32_t)u, units_per_row);
            load_codes(prm, at[i], codes[i], scale[i]);
        }
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
            if (u0 + (uint64_t)i * step >= units) break;
            if (at[i].c >= prm.dst_row) continue;
            const int64_t w = at[i].row / prm.tokens;
            bf16* dst = prm.planes_out + w * prm.dst_worker + (at[i].row - w * prm.tokens) * prm.dst_row + at[i].c;
            float v[W];
            codes[i].values(scale[i], v);
            if constexpr (sizeof(T) == 2) {
                *reinterpret_cast<uint4*>(dst) = narrow(v);
            } else {
                uint4 parts[3];
                split_slice(v, parts);
#pragma unroll
                for (int q = 0; q < 3; ++q) *reinterpret_cast<uint4*>(dst + q * prm.dst_plane) = parts[q];
            }
        }
    }
}

template <typename Kernel>
cudaError_t launch_units(Kernel kernel, const PackParams& prm, int64_t row_cols, int width, cudaStream_t stream)
{
    int sms = 0;
    cudaError_t err = sm_count(&sms);
    if (err != cudaSuccess) return err;
    const int64_t units_per_row = ceil_div(row_cols, 32 * width), units = prm.rows * units_per_row;
    if (units >= 1ll << 32) return cudaErrorInvalidValue;  // 2 TB of activations
    const int64_t blocks = ceil_div(units, kThreads / 32), resident = (int64_t)sms * 8;
    return launch_after(kernel, dim3((unsigned)(blocks < resident ? blocks : resident)), kThreads, 0, stream, 1, prm, (uint32_t)units,
                        (uint32_t)units_per_row);
}

template <typename T>
cudaError_t pack(const PackParams& prm, cudaStream_t stream)
{
    const int align = alignment<T>(prm.x, prm.cols, prm.x_row);
    return launch_units(align == 16 ? rps_pack_kernel<T, 16> : align == 4 ? rps_pack_kernel<T, 4> : rps_pack_kernel<T, sizeof(T)>, prm, prm.pitch,
                        Slice<T>::kWidth, stream);
}

template <typename T>
cudaError_t unpack(const PackParams& prm, cudaStream_t stream)
{
    const int align = alignment<T>(prm.out, prm.cols, prm.x_row);
    return launch_units(align == 16 ? rps_unpack_kernel<T, 16> : align == 4 ? rps_unpack_kernel<T, 4> : rps_unpack_kernel<T, sizeof(T)>, prm,
                        prm.cols, Slice<T>::kWidth, stream);
}

}  // namespace

cudaError_t launch_pack(const PackParams& prm, cudaStream_t stream)
{
    return prm.f32 ? pack<float>(prm, stream) : pack<bf16>(prm, stream);
}

cudaError_t launch_unpack(const PackParams& prm, cudaStream_t stream)
{
    return prm.f32 ? unpack<float>(prm, stream) : unpack<bf16>(prm, stream);
}

cudaError_t launch_unpack_planes(const PackParams& prm, cudaStream_t stream)
{
    return prm.f32 ? launch_units(rps_unpack_planes_kernel<float>, prm, prm.dst_row, 8, stream)
                   : launch_units(rps_unpack_planes_kernel<bf16>, prm, prm.dst_row, 8, stream);
}

}  // namespace rps_ops
