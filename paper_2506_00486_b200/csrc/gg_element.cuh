// Element types of the training kernels: storage in fp32 or bf16 (as uint16_t), arithmetic in fp32.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace gg {

template <typename T> __device__ __forceinline__ float widen(T v);
template <> __device__ __forceinline__ float widen<float>(float v) { return v; }
template <> __device__ __forceinline__ float widen<uint16_t>(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
template <typename T> __device__ __forceinline__ T narrow(float v);
template <> __device__ __forceinline__ float narrow<float>(float v) { return v; }
template <> __device__ __forceinline__ uint16_t narrow<uint16_t>(float v) { return __bfloat16_as_ushort(__float2bfloat16_rn(v)); }

// Two fp32 values in one register pair: one instruction does both (mul, add and fma of sm_100).  None of these is
// contracted with another by the compiler.
using f32x2 = unsigned long long;
__device__ __forceinline__ f32x2 pair(float lo, float hi)
{
    f32x2 d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
    return d;
}
__device__ __forceinline__ f32x2 both(float v) { return pair(v, v); }
__device__ __forceinline__ float2 halves(f32x2 v)
{
    float2 d;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(d.x), "=f"(d.y) : "l"(v));
    return d;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b)
{
    f32x2 d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b)
{
    f32x2 d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c)
{
    f32x2 d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
// The two bf16 values of a word, and back (to nearest).
__device__ __forceinline__ f32x2 widen2(uint32_t w) { return pair(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)); }
__device__ __forceinline__ uint32_t narrow2(f32x2 v)
{
    const float2 f = halves(v);
    uint32_t d;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(f.y), "f"(f.x));
    return d;
}

// Eight consecutive elements as four pairs; fp32 at a 32-byte boundary, bf16 at 16.  Streamed past L1.
template <typename T> struct Eight;
template <> struct Eight<float> {
    f32x2 v[4];
    __device__ __forceinline__ void zero() { v[0] = v[1] = v[2] = v[3] = 0; }
    __device__ __forceinline__ void load(const float *p)
    {
        asm volatile("ld.global.L1::no_allocate.v4.b64 {%0, %1, %2, %3}, [%4];" : "=l"(v[0]), "=l"(v[1]), "=l"(v[2]), "=l"(v[3]) : "l"(p));
    }
    __device__ __forceinline__ f32x2 get(int i) const { return v[i]; }
    static __device__ __forceinline__ void store(float *p, const f32x2 (&x)[4])
    {
        asm volatile("st.global.L1::no_allocate.v4.b64 [%0], {%1, %2, %3, %4};" ::"l"(p), "l"(x[0]), "l"(x[1]), "l"(x[2]), "l"(x[3]) : "memory");
    }
};
template <> struct Eight<uint16_t> {
    uint4 v;
    __device__ __forceinline__ void zero() { v = make_uint4(0u, 0u, 0u, 0u); }
    __device__ __forceinline__ void load(const uint16_t *p)
    {
        asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    }
    __device__ __forceinline__ f32x2 get(int i) const { return widen2(i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w); }
    static __device__ __forceinline__ void store_words(uint16_t *p, uint32_t a, uint32_t b, uint32_t c, uint32_t d)
    {
        asm volatile("st.global.L1::no_allocate.v4.u32 [%0], {%1, %2, %3, %4};" ::"l"(p), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
    }
    static __device__ __forceinline__ void store(uint16_t *p, const f32x2 (&x)[4])
    {
        store_words(p, narrow2(x[0]), narrow2(x[1]), narrow2(x[2]), narrow2(x[3]));
    }
};

}  // namespace gg
