// Activations in 8 bits: a scale for each 128 columns of a row.
//
// Bound by memory, and close to it by instructions: packing gives a group of 128 columns to as many lanes as make four slices each
// (8 lanes of fp32, 4 of bf16), so that one maximum over lanes, one division and one address serve 16 or 32 values.  (A
// slice a lane took 213 us for 32768 x 5000 fp32, this 172 us.)
#include "rps_rows.cuh"

namespace rps_ops {
namespace {

constexpr int kThreads = 256, kUnits = 4;

// n / d for any 32-bit n, without a division (Granlund and Montgomery, "Division by invariant integers using multiplication").
struct Divisor {
    uint32_t d, factor, shift;
    explicit Divisor(uint32_t by) : d(by)
    {
        uint32_t bits = 0;
        while (bits < 32 && (1ull << bits) < by) ++bits;
        factor = (uint32_t)((((1ull << bits) - by) << 32) / by + 1);
        shift = bits;
    }
    __device__ __forceinline__ uint32_t divide(uint32_t n) const
    {
        const uint32_t t = __umulhi(n, factor);
        return shift == 0 ? n : (t + ((n - t) >> 1)) >> (shift - 1);
    }
};

template <typename T, int ALIGN>
__global__ void __launch_bounds__(kThreads) rps_pack_kernel(const PackParams prm, uint32_t groups, Divisor groups_per_row)
{
    after_the_kernel_before();
    constexpr int W = Slice<T>::kWidth, kSlices = 4, kLanes = RPS_PACK_GROUP / (W * kSlices), kGroups = kThreads / kLanes;
    const int D = (int)prm.cols, lane = threadIdx.x % kLanes;
    for (uint64_t g0 = (uint64_t)blockIdx.x * kGroups + threadIdx.x / kLanes; g0 - threadIdx.x / kLanes < groups; g0 += (uint64_t)gridDim.x * kGroups) {
        const bool there = g0 < groups;  // all lanes of a warp go on, for the sake of the exchange
        const uint32_t g = there ? (uint32_t)g0 : 0, row = groups_per_row.divide(g);
        const int c0 = (int)(g - row * groups_per_row.d) * RPS_PACK_GROUP + lane * W;
        const T* x = static_cast<const T*>(prm.x) + row * prm.x_row;
        uint4 slice[kSlices];
#pragma unroll
        for (int i = 0; i < kSlices; ++i) slice[i] = load_slice<T, ALIGN, true>(x, c0 + i * kLanes * W, there ? D : 0);
        float v[kSlices][W];
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < kSlices; ++i) {
            widen(slice[i], v[i]);
            top = max(top, largest(v[i]));
        }
#pragma unroll
        for (int s = kLanes / 2; s > 0; s /= 2) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, s));
        const Quantiser q(top);
        int8_t* codes = prm.codes + row * prm.pitch;
#pragma unroll
        for (int i = 0; i < kSlices; ++i) {
            const int c = c0 + i * kLanes * W;
            if (there && c < prm.pitch) q.store(v[i], codes + c);
        }
        if (there && lane == 0) prm.scales[g] = q.scale();
    }
}

struct Place {
    int64_t row;
    int c;
};

// Reading back, a unit of work is a warp's worth of slices of one row (256 columns of bf16, 128 of fp32); a warp takes kUnits
// of them at a time, so that their loads are all on their way before the first is used.
template <int W>
__device__ __forceinline__ Place place(uint32_t u, const Divisor& units_per_row)
{
    const uint32_t row = units_per_row.divide(u);
    return {row, (int)((u - row * units_per_row.d) * 32 + threadIdx.x % 32) * W};
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
__global__ void __launch_bounds__(kThreads) rps_unpack_kernel(const PackParams prm, uint32_t units, Divisor units_per_row)
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
__global__ void __launch_bounds__(kThreads) rps_unpack_planes_kernel(const PackParams prm, uint32_t units, Divisor units_per_row)
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
            const uint32_t row = (uint32_t)at[i].row, w = row / (uint32_t)prm.tokens;  // both below 2^32
            bf16* dst = prm.planes_out + w * prm.dst_worker + (int64_t)(row - w * (uint32_t)prm.tokens) * prm.dst_row + at[i].c;
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

// `count` pieces of work, `per_row` to a row and `per_block` to a CTA.
template <typename Kernel>
cudaError_t launch_pieces(Kernel kernel, const PackParams& prm, int64_t per_row, int per_block, cudaStream_t stream)
{
    int sms = 0;
    cudaError_t err = sm_count(&sms);
    if (err != cudaSuccess) return err;
    const int64_t count = prm.rows * per_row;
    if (count >= 1ll << 32) return cudaErrorInvalidValue;  // terabytes of activations
    const int64_t blocks = ceil_div(count, per_block), resident = (int64_t)sms * 8;
    return launch_after(kernel, dim3((unsigned)(blocks < resident ? blocks : resident)), kThreads, 0, stream, 1, prm, (uint32_t)count,
                        Divisor((uint32_t)per_row));
}

template <typename Kernel>
cudaError_t launch_units(Kernel kernel, const PackParams& prm, int64_t row_cols, int width, cudaStream_t stream)
{
    return launch_pieces(kernel, prm, ceil_div(row_cols, 32 * width), kThreads / 32, stream);
}

template <typename T>
cudaError_t pack(const PackParams& prm, cudaStream_t stream)
{
    const int align = alignment<T>(prm.x, prm.cols, prm.x_row);
    return launch_pieces(align == 16 ? rps_pack_kernel<T, 16> : align == 4 ? rps_pack_kernel<T, 4> : rps_pack_kernel<T, sizeof(T)>, prm, prm.groups,
                         kThreads * 4 * Slice<T>::kWidth / RPS_PACK_GROUP, stream);
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
