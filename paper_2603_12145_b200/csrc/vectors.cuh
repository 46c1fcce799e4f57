// vectors.cuh -- runs of neighbouring elements as they lie in memory: one access, and taken apart where they are needed
// (an extraction right behind a load would wait for it).
#pragma once

#include <cstdint>

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

namespace {

template <typename T, int V>
struct Packed {
    static constexpr int kBytes = static_cast<int>(sizeof(T)) * V;
    static constexpr int kWords = (kBytes + 3) / 4;
    uint32_t w[kWords];
};

template <typename T, int V>
__device__ __forceinline__ Packed<T, V> packed_zero()
{
    Packed<T, V> v;
#pragma unroll
    for (int i = 0; i < Packed<T, V>::kWords; ++i) v.w[i] = 0;
    return v;
}

// Read once: no place in L1.  (Written as instructions, so that they stay ahead of the arithmetic.)
template <typename T, int V>
__device__ __forceinline__ Packed<T, V> packed_load(const T *p)
{
    Packed<T, V> v;
    if constexpr (Packed<T, V>::kBytes == 16)
        asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(v.w[0]), "=r"(v.w[1]), "=r"(v.w[2]), "=r"(v.w[3])
                     : "l"(p)
                     : "memory");
    else if constexpr (Packed<T, V>::kBytes == 8)
        asm volatile("ld.global.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(v.w[0]), "=r"(v.w[1]) : "l"(p) : "memory");
    else if constexpr (Packed<T, V>::kBytes == 4)
        asm volatile("ld.global.L1::no_allocate.u32 %0, [%1];" : "=r"(v.w[0]) : "l"(p) : "memory");
    else {
        static_assert(Packed<T, V>::kBytes == 2, "runs of 2, 4, 8 or 16 bytes");
        uint16_t h;
        asm volatile("ld.global.L1::no_allocate.u16 %0, [%1];" : "=h"(h) : "l"(p) : "memory");
        v.w[0] = h;
    }
    return v;
}

template <typename T, int V>
__device__ __forceinline__ void packed_store(T *p, const Packed<T, V> &v)
{
    if constexpr (Packed<T, V>::kBytes == 16)
        *reinterpret_cast<uint4 *>(p) = make_uint4(v.w[0], v.w[1], v.w[2], v.w[3]);
    else if constexpr (Packed<T, V>::kBytes == 8)
        *reinterpret_cast<uint2 *>(p) = make_uint2(v.w[0], v.w[1]);
    else if constexpr (Packed<T, V>::kBytes == 4)
        *reinterpret_cast<uint32_t *>(p) = v.w[0];
    else
        *reinterpret_cast<uint16_t *>(p) = static_cast<uint16_t>(v.w[0]);
}

template <typename T>
__device__ __forceinline__ float half_of(uint32_t w, int upper);
template <>
__device__ __forceinline__ float half_of<__nv_bfloat16>(uint32_t w, int upper)
{
    return __uint_as_float(upper ? w & 0xFFFF0000u : w << 16);
}
template <>
__device__ __forceinline__ float half_of<__half>(uint32_t w, int upper)
{
    return __half2float(__ushort_as_half(static_cast<unsigned short>(upper ? w >> 16 : w)));
}

template <typename T, int V>
__device__ __forceinline__ float packed_get(const Packed<T, V> &v, int e)
{
    if constexpr (sizeof(T) == 4)
        return __uint_as_float(v.w[e]);
    else
        return half_of<T>(v.w[e / 2], e & 1);
}

template <typename T>
__device__ __forceinline__ uint32_t pack_halves(float lo, float hi);
template <>
__device__ __forceinline__ uint32_t pack_halves<__nv_bfloat16>(float lo, float hi)
{
    const __nv_bfloat162 r = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&r);
}
template <>
__device__ __forceinline__ uint32_t pack_halves<__half>(float lo, float hi)
{
    const __half2 r = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&r);
}

template <typename T, int V>
__device__ __forceinline__ Packed<T, V> packed_of(const float (&f)[V])
{
    Packed<T, V> v;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < V; ++e) v.w[e] = __float_as_uint(f[e]);
    } else {
#pragma unroll
        for (int e = 0; e < V; e += 2) v.w[e / 2] = pack_halves<T>(f[e], e + 1 < V ? f[e + 1 < V ? e + 1 : e] : 0.0f);
    }
    return v;
}

}  // namespace
