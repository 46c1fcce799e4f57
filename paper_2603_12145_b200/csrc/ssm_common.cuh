// ssm_common.cuh -- what the kernels behind ssm.h share: element types, the
// scalar functions of the recurrence, packed binary32 pairs.
#pragma once

#include <cstdint>

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "../../include/ssm.h"

namespace ssm_k {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// ---- element types

template <typename T>
__device__ __forceinline__ float to_f32(T v);
template <>
__device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <>
__device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }

template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// A sequence with its element type; the innermost stride is 1.
template <typename T>
struct Seq {
    T *ptr;
    int64_t sb, st;
    __device__ __forceinline__ T *row(int64_t b, int64_t t) const { return ptr + b * sb + t * st; }
};

template <typename T>
Seq<T> seq_of(const ssm_seq &s)
{
    return Seq<T>{static_cast<T *>(s.ptr), s.stride_b, s.stride_t};
}

// ---- scalar functions (binary32)

__device__ __forceinline__ float ex2(float v)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

__device__ __forceinline__ float rcp(float v)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

// 1 / (1 + e^-v).  2^(-v log2 e) overflows to infinity for v < -88, whose reciprocal is the limit 0.
__device__ __forceinline__ float sigmoid(float v) { return rcp(1.0f + ex2(-kLog2e * v)); }

// log(1 + e^v) = max(v, 0) + log1p(e), e = e^-|v| in [0, 1].  log1p(e) = 2 artanh(s) with
// s = e / (2 + e) <= 1/3, summed as s + s^3/3 + ... + s^13/13: the rest is below s * 3e-8.
// Unlike log(1 + e) this keeps the relative precision of small steps (e near 0).
__device__ __forceinline__ float softplus(float v)
{
    const float e = ex2(-kLog2e * fabsf(v));
    const float s = e * rcp(2.0f + e);
    const float q = s * s;
    float p = 1.0f / 13.0f;
    p = fmaf(p, q, 1.0f / 11.0f);
    p = fmaf(p, q, 1.0f / 9.0f);
    p = fmaf(p, q, 1.0f / 7.0f);
    p = fmaf(p, q, 1.0f / 5.0f);
    p = fmaf(p, q, 1.0f / 3.0f);
    p = fmaf(p * q, s, s);
    return fmaxf(v, 0.0f) + 2.0f * p;
}

// ---- pairs of binary32 numbers: one instruction for both

struct Pair {
    unsigned long long v;
};

__device__ __forceinline__ Pair pair(float lo, float hi)
{
    Pair r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(lo), "f"(hi));
    return r;
}

__device__ __forceinline__ float lo(Pair p)
{
    float a, b;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p.v));
    return a;
}

__device__ __forceinline__ float hi(Pair p)
{
    float a, b;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p.v));
    return b;
}

__device__ __forceinline__ Pair mul(Pair a, Pair b)
{
    Pair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}

__device__ __forceinline__ Pair add(Pair a, Pair b)
{
    Pair r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}

__device__ __forceinline__ Pair fma(Pair a, Pair b, Pair c)
{
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}

__device__ __forceinline__ Pair ex2(Pair a) { return pair(ex2(lo(a)), ex2(hi(a))); }

}  // namespace ssm_k
