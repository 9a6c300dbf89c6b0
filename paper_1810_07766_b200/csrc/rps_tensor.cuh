// The tensor cores' instructions (tcgen05) and the descriptors that they take.
#pragma once

#include <atomic>

#include "rps_cluster.cuh"

namespace rps_ops {
namespace {

// One lane of a converged warp.  Behind a branch on this, products' operands that are the same for all lanes are issued as such: 42 cycles each at most,
// where behind `lane == 0` every one takes 110 (measured for tiles of 64 to 128 columns, which the tensor cores take 48 to 64 for).
__device__ __forceinline__ bool elect_one()
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}

// Descriptor of a shared-memory tile with the 128-byte swizzle: start address and two strides in units of 16 bytes, the constant 1 at
// bit 46, layout 2 (128-byte swizzle) at bit 61.  Summed axis contiguous: the stride at bit 32 leads from 8 rows to the next 8.
// Other axis contiguous: it leads from 8 steps of the summed axis to the next 8, and the one at bit 16 from one 64-wide box to the
// next.  The upper word is the same for all, and in the lower one tiles and their parts lie a constant apart.
constexpr uint32_t kDescriptorHigh = 1024 / 16 | 1u << 14 | 2u << 29;

__device__ __forceinline__ uint32_t descriptor_low(uint32_t addr, bool other, uint32_t box_bytes) { return addr >> 4 | (other ? box_bytes / 16 : 1) << 16; }

// fp32 sums of bf16 products, rows x tile_n.
__device__ __forceinline__ uint32_t instruction_descriptor(bool a_other, bool b_other, int rows, int tile_n)
{
    return 1u << 4 | 1u << 7 | 1u << 10 | (a_other ? 1u : 0u) << 15 | (b_other ? 1u : 0u) << 16 | (uint32_t)(tile_n / 8) << 17 | (uint32_t)(rows / 16) << 24;
}

// `a`, `b`: lower words of the descriptors.
template <int CTAS>
__device__ __forceinline__ void multiply(uint32_t sum, uint32_t a, uint32_t b, uint32_t descriptor, bool add)
{
    if constexpr (CTAS == 2)
        asm volatile(
            "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tsetp.ne.u32 p, %5, 0;\n\tmov.b64 da, {%1, %3};\n\tmov.b64 db, {%2, %3};\n\t"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %4, p;\n\t}" ::"r"(sum),
            "r"(a), "r"(b), "n"(kDescriptorHigh), "r"(descriptor), "r"((uint32_t)add)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tsetp.ne.u32 p, %5, 0;\n\tmov.b64 da, {%1, %3};\n\tmov.b64 db, {%2, %3};\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %4, p;\n\t}" ::"r"(sum),
            "r"(a), "r"(b), "n"(kDescriptorHigh), "r"(descriptor), "r"((uint32_t)add)
            : "memory");
}

// Arrives on the barrier at this offset (in both CTAs of a pair) once the products issued so far are done.
template <int CTAS>
__device__ __forceinline__ void commit(uint32_t bar)
{
    if constexpr (CTAS == 2)
        asm volatile(
            "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3)
            : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// All 512 columns of tensor memory, for the whole kernel.
template <int CTAS>
__device__ __forceinline__ void take_tensor_memory(uint32_t address_to)
{
    if constexpr (CTAS == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(address_to) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    } else {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(address_to) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
}

template <int CTAS>
__device__ __forceinline__ void free_tensor_memory(uint32_t address)
{
    if constexpr (CTAS == 2)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(address) : "memory");
    else
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(address) : "memory");
}

// 16 columns of this lane's row.
__device__ __forceinline__ void load_sums(float* v, uint32_t addr)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]),
          "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
        : "r"(addr)
        : "memory");
}

// Whether the kernel was compiled to the registers that its warps share out anew: it would wait for ever for those that a smaller launch does not have.
// `known` keeps the number once it has been asked for; a question that fails is asked again.
template <typename Kernel>
cudaError_t check_registers(std::atomic<int>& known, Kernel kernel, int expected)
{
    int registers = known.load(std::memory_order_relaxed);
    if (registers == 0) {
        cudaFuncAttributes attributes{};
        const cudaError_t err = cudaFuncGetAttributes(&attributes, kernel);
        if (err != cudaSuccess) return err;
        known.store(registers = attributes.numRegs, std::memory_order_relaxed);
    }
    return registers == expected ? cudaSuccess : cudaErrorInvalidKernelImage;
}

}  // namespace
}  // namespace rps_ops
