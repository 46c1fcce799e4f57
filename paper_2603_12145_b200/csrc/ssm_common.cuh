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

// An element as the low bits of a register, to be widened when it is needed: kept as a 16-bit variable it
// would be packed with another one right behind its load, which waits for it.  The sequences are read
// once: they need no place in L1.  (Written as an instruction: as a plain load the compiler moves it
// next to its use, 2.53 against 2.11 ms in the backward kernel at 512 x 128 x 1152.)
template <typename T>
__device__ __forceinline__ uint32_t load_bits(const T *p)
{
    if (sizeof(T) == 4) {
        uint32_t v;
        asm volatile("ld.global.L1::no_allocate.u32 %0, [%1];" : "=r"(v) : "l"(p));
        return v;
    }
    uint16_t v;
    asm volatile("ld.global.L1::no_allocate.u16 %0, [%1];" : "=h"(v) : "l"(p));
    return v;
}

template <typename T>
__device__ __forceinline__ float from_bits(uint32_t w);
template <>
__device__ __forceinline__ float from_bits<float>(uint32_t w) { return __uint_as_float(w); }
template <>
__device__ __forceinline__ float from_bits<__nv_bfloat16>(uint32_t w) { return __uint_as_float(w << 16); }
template <>
__device__ __forceinline__ float from_bits<__half>(uint32_t w)
{
    return __half2float(__ushort_as_half(static_cast<unsigned short>(w)));
}

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

// e^v.  v log2 e is formed in two parts: rounded to one binary32 number its error would be that
// of the exponent, |v| 2^-24 relative in the result.
__device__ __forceinline__ float exp_of(float v)
{
    constexpr float kLog2eLow = 1.9259629911e-8f;   // log2 e - float(log2 e)
    const float t = v * kLog2e;
    const float r = fmaf(v, kLog2eLow, fmaf(v, kLog2e, -t));
    const float e = ex2(t);
    return fmaf(e * kLn2, r, e);
}

// Bounds that let a NaN through.
__device__ __forceinline__ float at_least(float v, float bound)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(v), "f"(bound));
    return r;
}

__device__ __forceinline__ float at_most(float v, float bound)
{
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(v), "f"(bound));
    return r;
}

// 1 / (1 + e^-v).  Below v = -88 the result stays at its value there, 0 (e^88 has a subnormal
// reciprocal): the correction term of an infinite exponential would be a NaN.
__device__ __forceinline__ float sigmoid(float v) { return rcp(1.0f + exp_of(at_most(-v, 88.0f))); }

// log(1 + e^v) = max(v, 0) + log1p(e), e = e^-|v| in [0, 1].  log1p(e) = 2 artanh(s) with
// s = e / (2 + e) <= 1/3, summed as s + s^3/3 + ... + s^13/13: the rest is below s * 3e-8.
// Unlike log(1 + e) this keeps the relative precision of small steps (e near 0).
__device__ __forceinline__ float softplus(float v)
{
    const float e = exp_of(at_least(-fabsf(v), -104.0f));
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

// ---- sums over lanes

// v[0..3] over the four lanes that share lane >> 2: lane gets the total of v[lane & 3].
__device__ __forceinline__ float spread4(const float (&v)[4], int lane)
{
    const bool b1 = lane & 2, b0 = lane & 1;
    const float s0 = b1 ? v[0] : v[2], s1 = b1 ? v[1] : v[3];
    const float k0 = (b1 ? v[2] : v[0]) + __shfl_xor_sync(0xFFFFFFFFu, s0, 2);
    const float k1 = (b1 ? v[3] : v[1]) + __shfl_xor_sync(0xFFFFFFFFu, s1, 2);
    return (b0 ? k1 : k0) + __shfl_xor_sync(0xFFFFFFFFu, b0 ? k0 : k1, 1);
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

// The decay 2^(rate delta) of one step, rate = A log2 e.  A state that decays slowly is multiplied by
// numbers just below one step after step, so that a bias of the exponential adds up over the
// sequence.  The hardware's result is low, in units of 2^-23 and on average, by 0.04 to 0.1 for arguments
// up to 2^-8 and by 0.07 to 0.26 from there to a half (measured; the spread is 0.25 to 0.3 units, as that
// of a correctly rounded result).  The multiply-add that forms the argument adds 0.15 of them back, which
// leaves 0.11 either way: 1,000 steps at 0.999 end 1.3e-5 high, the final state of 128 training steps is off by
// 5.8e-7 (1.3e-6 without the addend; with 0.2 units 1.9e-5 and 8.0e-7).  Where the argument is so large that the
// addend disappears in its rounding, the state forgets within a few steps.
//
// Every form of the recurrence uses it, so that a rollout taken in single tokens and its training pass go through
// the same states.
constexpr float kDecayBias = 0.15f * 1.1920929e-7f * kLog2e;

__device__ __forceinline__ float decay(float rate, float delta) { return ex2(fmaf(rate, delta, kDecayBias)); }

__device__ __forceinline__ Pair decay(Pair rate, Pair delta) { return ex2(fma(rate, delta, pair(kDecayBias, kDecayBias))); }

// ---- the scalar functions on pairs (two steps of a channel): the same arithmetic in half the instructions

__device__ __forceinline__ Pair exp_of(Pair v)
{
    constexpr float kLog2eLow = 1.9259629911e-8f;
    const Pair t = mul(v, pair(kLog2e, kLog2e)), minus_t = mul(v, pair(-kLog2e, -kLog2e));
    const Pair r = fma(v, pair(kLog2eLow, kLog2eLow), fma(v, pair(kLog2e, kLog2e), minus_t));
    const Pair e = ex2(t);
    return fma(mul(e, pair(kLn2, kLn2)), r, e);
}

__device__ __forceinline__ Pair rcp(Pair v) { return pair(rcp(lo(v)), rcp(hi(v))); }

// The gate's sigmoid: for a 16-bit result the exponent's rounding (|v| 2^-24 relative) is far below the result's.
template <typename T>
__device__ __forceinline__ Pair gate_sigmoid(Pair v)
{
    const Pair one = pair(1.0f, 1.0f);
    if (sizeof(T) == 2) return rcp(add(ex2(mul(v, pair(-kLog2e, -kLog2e))), one));
    return rcp(add(exp_of(pair(at_most(-lo(v), 88.0f), at_most(-hi(v), 88.0f))), one));
}

// softplus, and its slope sigmoid(v) from the same exponential
__device__ __forceinline__ Pair softplus(Pair v, Pair *slope = nullptr)
{
    const Pair e = exp_of(pair(at_least(-fabsf(lo(v)), -104.0f), at_least(-fabsf(hi(v)), -104.0f)));
    const Pair s = mul(e, rcp(add(e, pair(2.0f, 2.0f))));
    const Pair q = mul(s, s);
    Pair p = pair(1.0f / 13.0f, 1.0f / 13.0f);
    p = fma(p, q, pair(1.0f / 11.0f, 1.0f / 11.0f));
    p = fma(p, q, pair(1.0f / 9.0f, 1.0f / 9.0f));
    p = fma(p, q, pair(1.0f / 7.0f, 1.0f / 7.0f));
    p = fma(p, q, pair(1.0f / 5.0f, 1.0f / 5.0f));
    p = fma(p, q, pair(1.0f / 3.0f, 1.0f / 3.0f));
    p = fma(mul(p, q), s, s);
    if (slope != nullptr) {
        const Pair r = rcp(add(e, pair(1.0f, 1.0f))), er = mul(e, r);
        *slope = pair(lo(v) >= 0.0f ? lo(r) : lo(er), hi(v) >= 0.0f ? hi(r) : hi(er));
    }
    return fma(p, pair(2.0f, 2.0f), pair(fmaxf(lo(v), 0.0f), fmaxf(hi(v), 0.0f)));
}

}  // namespace ssm_k
