// Slices of rows: what a lane owns of a row is 16 bytes of values (8 bf16 or 4 fp32 consecutive columns).  128 columns, which
// share a scale in 8-bit form, are then 16 or 32 neighbouring lanes.  ALIGN says what a slice is moved in: 16 bytes where every
// row starts on such a boundary, else 4 (two bf16 of an even row, or one fp32), else 2.
#pragma once

#include "rps_ops_kernels.h"

namespace rps_ops {
namespace {

template <typename T>
struct Slice;
template <>
struct Slice<float> {
    static constexpr int kWidth = 4;
    static constexpr int kGroupLanes = RPS_PACK_GROUP / 4;
};
template <>
struct Slice<bf16> {
    static constexpr int kWidth = 8;
    static constexpr int kGroupLanes = RPS_PACK_GROUP / 8;
};

__device__ __forceinline__ uint4 load_streaming(const void* p)
{
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

// The 16 bytes of columns c..c+width-1, zero from `cols` on.
template <typename T, int ALIGN, bool STREAM>
__device__ __forceinline__ uint4 load_slice(const T* row, int c, int cols)
{
    if constexpr (ALIGN == 16) {
        if (c >= cols) return make_uint4(0, 0, 0, 0);
        return STREAM ? load_streaming(row + c) : *reinterpret_cast<const uint4*>(row + c);
    } else if constexpr (ALIGN == 4) {
        constexpr int kPer = 4 / sizeof(T);
        uint32_t r[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) r[j] = c + j * kPer < cols ? __ldg(reinterpret_cast<const uint32_t*>(row + c + j * kPer)) : 0u;
        return make_uint4(r[0], r[1], r[2], r[3]);
    } else {
        const unsigned short* half = reinterpret_cast<const unsigned short*>(row);
        uint32_t r[4] = {};
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (c + j < cols) r[j / 2] |= (uint32_t)__ldg(half + c + j) << (j % 2 * 16);
        return make_uint4(r[0], r[1], r[2], r[3]);
    }
}

template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t slot, const void* from, bool there)
{
    const uint32_t bytes = there ? BYTES : 0;  // what is not there becomes zero
    if constexpr (BYTES == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(slot), "l"(from), "r"(bytes) : "memory");
    else
        asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(slot), "l"(from), "n"(BYTES), "r"(bytes) : "memory");
}

// load_slice into this thread's slot of shared memory, without waiting for it where the alignment allows.
template <typename T, int ALIGN>
__device__ __forceinline__ void copy_slice(uint32_t slot, const T* row, int c, int cols)
{
    if constexpr (ALIGN == 16) {
        copy_async<16>(slot, c < cols ? row + c : row, c < cols);
    } else if constexpr (ALIGN == 4) {
        constexpr int kPer = 4 / sizeof(T);
#pragma unroll
        for (int j = 0; j < 4; ++j) copy_async<4>(slot + 4 * j, c + j * kPer < cols ? row + c + j * kPer : row, c + j * kPer < cols);
    } else {
        const uint4 v = load_slice<T, 2, true>(row, c, cols);
        asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(slot), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
    }
}

__device__ __forceinline__ void copies_sent() { asm volatile("cp.async.commit_group;" ::: "memory"); }

// All but the last N groups of this thread's copies have arrived.
template <int N>
__device__ __forceinline__ void copies_arrived()
{
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

__device__ __forceinline__ uint4 read_slot(uint32_t slot)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(slot) : "memory");
    return v;
}

__device__ __forceinline__ void widen(const uint4& s, float (&v)[4])
{
    v[0] = __uint_as_float(s.x), v[1] = __uint_as_float(s.y), v[2] = __uint_as_float(s.z), v[3] = __uint_as_float(s.w);
}

__device__ __forceinline__ void widen(const uint4& s, float (&v)[8])
{
    const uint32_t r[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(r[i] << 16);
        v[2 * i + 1] = __uint_as_float(r[i] & 0xFFFF0000u);
    }
}

// Two fp32 values that one instruction works on (fma.rn.f32x2 and its like round each as the single instructions do).
struct Pair {
    uint64_t bits;
    __device__ __forceinline__ Pair() {}
    __device__ __forceinline__ Pair(float a, float b) { asm("mov.b64 %0, {%1, %2};" : "=l"(bits) : "f"(a), "f"(b)); }
    __device__ __forceinline__ explicit Pair(float a) : Pair(a, a) {}
    __device__ __forceinline__ void get(float& a, float& b) const { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(bits)); }
    __device__ __forceinline__ float sum() const
    {
        float a, b;
        get(a, b);
        return a + b;
    }
};

__device__ __forceinline__ Pair operator*(const Pair& a, const Pair& b)
{
    Pair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.bits) : "l"(a.bits), "l"(b.bits));
    return r;
}

__device__ __forceinline__ Pair fma(const Pair& a, const Pair& b, const Pair& c)
{
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.bits) : "l"(a.bits), "l"(b.bits), "l"(c.bits));
    return r;
}

__device__ __forceinline__ Pair operator+(const Pair& a, const Pair& b)
{
    Pair r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.bits) : "l"(a.bits), "l"(b.bits));
    return r;
}

// exp(v - at).  The difference comes before the factor: v * log2(e) - at * log2(e) is off by a unit of the products' last place, which beyond 2^30
// is outside the exponent's range, so that a row's largest logit gave infinity or zero instead of one.
__device__ __forceinline__ float exp_of_difference(float v, float at) { return exp2_fast((v - at) * kLog2e); }

// The same of two values.
__device__ __forceinline__ Pair exp_of_difference(const Pair& v, float at)
{
    float a, b;
    ((v + Pair(-at)) * Pair(kLog2e)).get(a, b);
    return Pair(exp2_fast(a), exp2_fast(b));
}

__device__ __forceinline__ void widen(const uint4& s, Pair (&v)[2])
{
    v[0] = Pair(__uint_as_float(s.x), __uint_as_float(s.y)), v[1] = Pair(__uint_as_float(s.z), __uint_as_float(s.w));
}

__device__ __forceinline__ void widen(const uint4& s, Pair (&v)[4])
{
    const uint32_t r[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = Pair(__uint_as_float(r[i] << 16), __uint_as_float(r[i] & 0xFFFF0000u));
}

__device__ __forceinline__ uint4 narrow(const Pair (&v)[2])
{
    float a, b, c, d;
    v[0].get(a, b), v[1].get(c, d);
    return make_uint4(__float_as_uint(a), __float_as_uint(b), __float_as_uint(c), __float_as_uint(d));
}

__device__ __forceinline__ uint4 narrow(const Pair (&v)[4])
{
    uint32_t r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a, b;
        v[i].get(a, b);
        const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
        r[i] = *reinterpret_cast<const uint32_t*>(&p);
    }
    return make_uint4(r[0], r[1], r[2], r[3]);
}

__device__ __forceinline__ uint4 narrow(const float (&v)[4])
{
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
}

__device__ __forceinline__ uint4 narrow(const float (&v)[8])
{
    uint32_t r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 p = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        r[i] = *reinterpret_cast<const uint32_t*>(&p);
    }
    return make_uint4(r[0], r[1], r[2], r[3]);
}

template <typename T, int ALIGN>
__device__ __forceinline__ void store_slice(T* row, int c, int cols, const uint4& v)
{
    const uint32_t r[4] = {v.x, v.y, v.z, v.w};
    if constexpr (ALIGN == 16) {
        if (c < cols) *reinterpret_cast<uint4*>(row + c) = v;
    } else if constexpr (ALIGN == 4) {
        constexpr int kPer = 4 / sizeof(T);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (c + j * kPer < cols) *reinterpret_cast<uint32_t*>(row + c + j * kPer) = r[j];
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (c + j < cols) reinterpret_cast<unsigned short*>(row)[c + j] = (unsigned short)(r[j / 2] >> (j % 2 * 16));
    }
}

// What rows that start at `p` and are `stride` elements apart (of `cols` elements) can be moved in.
template <typename T>
int alignment(const void* p, int64_t cols, int64_t stride)
{
    const uint64_t bits = reinterpret_cast<uintptr_t>(p) | (uint64_t)cols * sizeof(T) | (uint64_t)stride * sizeof(T);
    return bits % 16 == 0 ? 16 : bits % 4 == 0 ? 4 : 2;
}

// Eight fp32 values as three slices of bf16 parts that add up to them.
__device__ __forceinline__ void split_slice(const float (&v)[8], uint4 (&parts)[3])
{
    uint32_t r[4][3];
#pragma unroll
    for (int j = 0; j < 4; ++j) split_two(v[2 * j], v[2 * j + 1], r[j]);
#pragma unroll
    for (int q = 0; q < 3; ++q) parts[q] = make_uint4(r[0][q], r[1][q], r[2][q], r[3][q]);
}

constexpr float kSmallestPacked = 0x1p-100f;  // a group with nothing larger is kept as zeros: 127 / max stays finite

// The largest size among a lane's values, as bits: as integers, finite < infinity < NaN.
template <int WIDTH>
__device__ __forceinline__ uint32_t largest(const float (&v)[WIDTH])
{
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < WIDTH; ++j) top = max(top, __float_as_uint(v[j]) & 0x7FFFFFFFu);
    return top;
}

// Codes and scale of a group whose largest size is `top`.
struct Quantiser {
    float largest, factor;
    bool finite, zero;
    __device__ __forceinline__ explicit Quantiser(uint32_t top)
    {
        largest = __uint_as_float(top);
        finite = top < 0x7F800000u, zero = !finite || largest < kSmallestPacked;
        factor = zero ? 0.0f : __fdiv_rn(127.0f, largest);
    }
    __device__ __forceinline__ float scale() const { return !finite ? __int_as_float(0x7FFFFFFF) : zero ? 0.0f : __fmul_rn(largest, 1.0f / 127.0f); }
    // 1.5 * 2^23 has units of one in its last place, so adding it rounds to an integer, ties to even, and leaves it in the low bits
    template <int WIDTH>
    __device__ __forceinline__ void store(const float (&v)[WIDTH], int8_t* codes) const
    {
        uint32_t word[WIDTH / 4];
#pragma unroll
        for (int i = 0; i < WIDTH / 4; ++i) {
            uint32_t q[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) q[j] = __float_as_uint(__fadd_rn(__fmul_rn(v[4 * i + j], factor), 12582912.0f));
            word[i] = __byte_perm(__byte_perm(q[0], q[1], 0x0040), __byte_perm(q[2], q[3], 0x0040), 0x5410);
            if (zero) word[i] = 0;  // infinities and NaN times zero
        }
        if constexpr (WIDTH == 8)
            *reinterpret_cast<uint2*>(codes) = make_uint2(word[0], word[1]);
        else
            *reinterpret_cast<uint32_t*>(codes) = word[0];
    }
};

// A lane's slice of a group in 8 bits: all lanes of the warp call it.  Columns past the end hold zeros.  The scale goes out from
// the group's first lane (`scale` NULL in lanes that are past the end), the codes where `codes` is not NULL.
template <int WIDTH>
__device__ __forceinline__ void pack_slice(const float (&v)[WIDTH], int8_t* codes, float* scale)
{
    constexpr int kLanes = RPS_PACK_GROUP / WIDTH;
    uint32_t top = largest(v);
#pragma unroll
    for (int s = kLanes / 2; s > 0; s /= 2) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, s));
    const Quantiser q(top);
    if (codes != nullptr) q.store(v, codes);
    if (scale != nullptr && threadIdx.x % kLanes == 0) *scale = q.scale();
}

// The values of four codes: a byte with its sign bit turned over, put under the bits of 2^23, is 2^23 + 128 + code.
__device__ __forceinline__ void code_values(uint32_t word, float scale, float* v)
{
    const uint32_t w = word ^ 0x80808080u;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = __fmul_rn(__uint_as_float(__byte_perm(w, 0x4B000000u, 0x7540u + j)) - 8388736.0f, scale);
}

// Codes of a slice as they lie in memory, and their values.
template <int WIDTH>
struct Codes {
    uint32_t w[WIDTH / 4];
    __device__ __forceinline__ void load(const int8_t* p)
    {
        if constexpr (WIDTH == 8) {
            const uint2 v = __ldg(reinterpret_cast<const uint2*>(p));
            w[0] = v.x, w[1] = v.y;
        } else {
            w[0] = __ldg(reinterpret_cast<const uint32_t*>(p));
        }
    }
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < WIDTH / 4; ++i) w[i] = 0;
    }
    __device__ __forceinline__ void values(float scale, float (&v)[WIDTH]) const
    {
#pragma unroll
        for (int i = 0; i < WIDTH / 4; ++i) code_values(w[i], scale, v + 4 * i);
    }
};

}  // namespace
}  // namespace rps_ops
