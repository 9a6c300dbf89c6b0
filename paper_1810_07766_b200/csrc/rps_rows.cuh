// Slices of rows: what a lane owns of a row is 16 bytes of values (8 bf16 or 4 fp32 consecutive columns), read and written in one piece
// where everything is aligned and element by element otherwise.  128 columns, which share a scale in 8-bit form, are then
// 16 or 32 neighbouring lanes.
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
template <typename T, bool ALIGNED, bool STREAM>
__device__ __forceinline__ uint4 load_slice(const T* row, int c, int cols)
{
    if constexpr (ALIGNED) {
        if (c >= cols) return make_uint4(0, 0, 0, 0);
        return STREAM ? load_streaming(row + c) : *reinterpret_cast<const uint4*>(row + c);
    } else {
        uint4 v = make_uint4(0, 0, 0, 0);
        T* e = reinterpret_cast<T*>(&v);
#pragma unroll
        for (int j = 0; j < Slice<T>::kWidth; ++j)
            if (c + j < cols) e[j] = row[c + j];
        return v;
    }
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

template <typename T, bool ALIGNED>
__device__ __forceinline__ void store_slice(T* row, int c, int cols, const uint4& v)
{
    if constexpr (ALIGNED) {
        if (c < cols) *reinterpret_cast<uint4*>(row + c) = v;
    } else {
        const T* e = reinterpret_cast<const T*>(&v);
#pragma unroll
        for (int j = 0; j < Slice<T>::kWidth; ++j)
            if (c + j < cols) row[c + j] = e[j];
    }
}

// Eight fp32 values as three slices of bf16 parts that add up to them.
__device__ __forceinline__ void split_slice(const float (&v)[8], uint4 (&parts)[3])
{
    uint32_t r[3][4];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        bf16 p[3];
        split_planes(v[j], p);
#pragma unroll
        for (int q = 0; q < 3; ++q) {
            const uint32_t bits = __bfloat16_as_ushort(p[q]);
            r[q][j / 2] = j % 2 == 0 ? bits : r[q][j / 2] | bits << 16;
        }
    }
#pragma unroll
    for (int q = 0; q < 3; ++q) parts[q] = make_uint4(r[q][0], r[q][1], r[q][2], r[q][3]);
}

constexpr float kSmallestPacked = 0x1p-100f;  // a group with nothing larger is kept as zeros: 127 / max stays finite

// A lane's part of a group in 8 bits: all lanes of the warp call it.  Columns past the end hold zeros.  The scale goes out from
// the group's first lane (`scale` NULL in lanes that are past the end), the codes where `codes` is not NULL.
template <int WIDTH>
__device__ __forceinline__ void pack_slice(const float (&v)[WIDTH], int8_t* codes, float* scale)
{
    constexpr int kLanes = RPS_PACK_GROUP / WIDTH;
    float top = 0.0f;
    bool finite = true;
#pragma unroll
    for (int j = 0; j < WIDTH; ++j) {
        finite &= fabsf(v[j]) <= 3.402823466e38f;
        top = fmaxf(top, fabsf(v[j]));
    }
    if (!finite) top = INFINITY;  // a NaN that the maximum does not see
#pragma unroll
    for (int s = kLanes / 2; s > 0; s /= 2) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, s));
    finite = top <= 3.402823466e38f;
    const bool zero = !finite || top < kSmallestPacked;
    const float factor = zero ? 0.0f : __fdiv_rn(127.0f, top);
    uint32_t word[WIDTH / 4];
#pragma unroll
    for (int i = 0; i < WIDTH / 4; ++i) {
        word[i] = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int q = zero ? 0 : __float2int_rn(__fmul_rn(v[4 * i + j], factor));
            word[i] |= (uint32_t)(q & 0xFF) << (8 * j);
        }
    }
    if (codes != nullptr) {
        if constexpr (WIDTH == 8)
            *reinterpret_cast<uint2*>(codes) = make_uint2(word[0], word[1]);
        else
            *reinterpret_cast<uint32_t*>(codes) = word[0];
    }
    if (scale != nullptr && threadIdx.x % kLanes == 0) *scale = !finite ? __int_as_float(0x7FFFFFFF) : zero ? 0.0f : __fmul_rn(top, 1.0f / 127.0f);
}

// Codes as they lie in memory, and their values.
template <int WIDTH>
struct Codes;
template <>
struct Codes<8> {
    uint2 w;
    __device__ __forceinline__ void load(const int8_t* p) { w = __ldg(reinterpret_cast<const uint2*>(p)); }
    __device__ __forceinline__ void clear() { w = make_uint2(0, 0); }
    __device__ __forceinline__ void values(float scale, float (&v)[8]) const
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[j] = __fmul_rn((float)(int8_t)(w.x >> (8 * j)), scale);
            v[4 + j] = __fmul_rn((float)(int8_t)(w.y >> (8 * j)), scale);
        }
    }
};
template <>
struct Codes<4> {
    uint32_t w;
    __device__ __forceinline__ void load(const int8_t* p) { w = __ldg(reinterpret_cast<const uint32_t*>(p)); }
    __device__ __forceinline__ void clear() { w = 0; }
    __device__ __forceinline__ void values(float scale, float (&v)[4]) const
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = __fmul_rn((float)(int8_t)(w >> (8 * j)), scale);
    }
};

}  // namespace
}  // namespace rps_ops
