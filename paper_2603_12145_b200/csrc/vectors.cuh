// vectors.cuh -- runs of neighbouring elements as they lie in memory: one access, and taken apart where they are needed
// (an extraction right behind a load would wait for it).
#pragma once

#include <cstdint>

#include <type_traits>

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "ssm_common.cuh"

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

// Of runs of 16-bit elements: those [from, to), one by one; the others are neither read (zeros) nor written.
template <typename T, int V>
__device__ __forceinline__ Packed<T, V> packed_load_part(const T *p, int from, int to)
{
    static_assert(sizeof(T) == 2, "halves of words");
    Packed<T, V> v = packed_zero<T, V>();
#pragma unroll
    for (int e = 0; e < V; ++e)
        if (e >= from && e < to) v.w[e / 2] |= packed_load<T, 1>(p + e).w[0] << (e & 1 ? 16 : 0);
    return v;
}

template <typename T, int V>
__device__ __forceinline__ void packed_store_part(T *p, const Packed<T, V> &v, int from, int to)
{
    static_assert(sizeof(T) == 2, "halves of words");
#pragma unroll
    for (int e = 0; e < V; ++e)
        if (e >= from && e < to) *reinterpret_cast<uint16_t *>(p + e) = static_cast<uint16_t>(v.w[e / 2] >> (e & 1 ? 16 : 0));
}

// Zeros but for elements [from, to).
template <typename T, int V>
__device__ __forceinline__ void packed_trim(Packed<T, V> &v, int from, int to)
{
    static_assert(sizeof(T) == 2, "halves of words");
#pragma unroll
    for (int e = 0; e < V; ++e) v.w[e / 2] &= e >= from && e < to ? 0xFFFFFFFFu : e & 1 ? 0x0000FFFFu : 0xFFFF0000u;
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

// ---- values of one element, or of a pair that one instruction works on.  (In a namespace of their own: among the names of
// the file that includes this, fma and its like would hide those of binary64.)

namespace vals {

using ssm_k::add;
using ssm_k::ex2;
using ssm_k::fma;
using ssm_k::hi;
using ssm_k::lo;
using ssm_k::mul;
using ssm_k::Pair;
using ssm_k::pair;
using ssm_k::rcp;

template <int V>
using Vals = std::conditional_t<V == 1, float, Pair>;

__device__ __forceinline__ float add(float a, float b) { return __fadd_rn(a, b); }
__device__ __forceinline__ float mul(float a, float b) { return __fmul_rn(a, b); }
__device__ __forceinline__ float fma(float a, float b, float c) { return fmaf(a, b, c); }

template <int V>
__device__ __forceinline__ Vals<V> all(float v)
{
    if constexpr (V == 1)
        return v;
    else
        return pair(v, v);
}

// f on each channel
template <typename F>
__device__ __forceinline__ float each(F f, float a) { return f(a); }
template <typename F>
__device__ __forceinline__ Pair each(F f, Pair a) { return pair(f(lo(a)), f(hi(a))); }
template <typename F>
__device__ __forceinline__ float each(F f, float a, float b) { return f(a, b); }
template <typename F>
__device__ __forceinline__ Pair each(F f, Pair a, Pair b) { return pair(f(lo(a), lo(b)), f(hi(a), hi(b))); }
template <typename F>
__device__ __forceinline__ float each(F f, float a, float b, float c) { return f(a, b, c); }
template <typename F>
__device__ __forceinline__ Pair each(F f, Pair a, Pair b, Pair c) { return pair(f(lo(a), lo(b), lo(c)), f(hi(a), hi(b), hi(c))); }

template <typename T>
__device__ __forceinline__ float widen(const Packed<T, 1> &v) { return packed_get<T, 1>(v, 0); }
template <typename T>
__device__ __forceinline__ Pair widen(const Packed<T, 2> &v) { return pair(packed_get<T, 2>(v, 0), packed_get<T, 2>(v, 1)); }

template <typename T>
__device__ __forceinline__ Packed<T, 1> narrow(float v)
{
    const float f[1] = {v};
    return packed_of<T, 1>(f);
}
template <typename T>
__device__ __forceinline__ Packed<T, 2> narrow(Pair v)
{
    const float f[2] = {lo(v), hi(v)};
    return packed_of<T, 2>(f);
}

// Of V elements, the i-th pair (of one, the element itself).
template <typename T, int V>
__device__ __forceinline__ Vals<V == 1 ? 1 : 2> widen_at(const Packed<T, V> &v, int i)
{
    if constexpr (V == 1)
        return packed_get<T, 1>(v, 0);
    else
        return pair(packed_get<T, V>(v, 2 * i), packed_get<T, V>(v, 2 * i + 1));
}

template <typename T>
__device__ __forceinline__ void narrow_at(Packed<T, 1> &v, int, float f) { v = narrow<T>(f); }
template <typename T, int V>
__device__ __forceinline__ void narrow_at(Packed<T, V> &v, int i, Pair f)
{
    if constexpr (sizeof(T) == 4) {
        v.w[2 * i] = __float_as_uint(lo(f));
        v.w[2 * i + 1] = __float_as_uint(hi(f));
    } else {
        v.w[i] = pack_halves<T>(lo(f), hi(f));
    }
}

__device__ __forceinline__ float sum_of(float v) { return v; }
__device__ __forceinline__ float sum_of(Pair v) { return lo(v) + hi(v); }

}  // namespace vals
}  // namespace
