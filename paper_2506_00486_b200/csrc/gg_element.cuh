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

// Two fp32 values in one register pair: one instruction does both (mul, add and fma of sm_100).  The assembler may fuse a
// mul2 and an add2 into a multiply-add, in spite of their .rn (nvcc 12.9, -fmad=false or not): add2_apart is the sum that
// is never fused.
using f32x2 = unsigned long long;
__device__ __forceinline__ f32x2 pair(float lo, float hi)
{
    f32x2 d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
    return d;
}
__device__ __forceinline__ f32x2 both(float v) { return pair(v, v); }
__device__ __forceinline__ f32x2 pair(const float2 &v) { return pair(v.x, v.y); }
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
__device__ __forceinline__ f32x2 add2_apart(f32x2 a, f32x2 b)
{
    const float2 x = halves(a), y = halves(b);
    return pair(__fadd_rn(x.x, y.x), __fadd_rn(x.y, y.y));
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

// Asynchronous copies into shared memory (its 32-bit address).
__device__ __forceinline__ void copy16(uint32_t to, const void *from)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copy8(uint32_t to, const void *from)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void zero16(uint32_t to) { asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(to), "r"(0u) : "memory"); }
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory"); }

// 16 bytes of consecutive elements as pairs: read from shared memory, or through L1 (what every row reads), and streamed
// out past L1.
template <typename T> struct Few;
template <> struct Few<float> {
    static constexpr int kPairs = 2;
    f32x2 v[2];
    __device__ __forceinline__ void read(uint32_t at)
    {
        asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(v[0]), "=l"(v[1]) : "r"(at) : "memory");
    }
    __device__ __forceinline__ void read(const float *p)
    {
        const float4 t = __ldg(reinterpret_cast<const float4 *>(p));
        v[0] = pair(t.x, t.y);
        v[1] = pair(t.z, t.w);
    }
    __device__ __forceinline__ f32x2 get(int i) const { return v[i]; }
    static __device__ __forceinline__ void store(float *p, const f32x2 (&x)[2])
    {
        asm volatile("st.global.L1::no_allocate.v2.b64 [%0], {%1, %2};" ::"l"(p), "l"(x[0]), "l"(x[1]) : "memory");
    }
};
template <> struct Few<uint16_t> {
    static constexpr int kPairs = 4;
    uint32_t v[4];
    __device__ __forceinline__ void read(uint32_t at)
    {
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(at) : "memory");
    }
    __device__ __forceinline__ void read(const uint16_t *p)
    {
        const uint4 t = __ldg(reinterpret_cast<const uint4 *>(p));
        v[0] = t.x; v[1] = t.y; v[2] = t.z; v[3] = t.w;
    }
    __device__ __forceinline__ f32x2 get(int i) const { return widen2(v[i]); }
    static __device__ __forceinline__ void store(uint16_t *p, const f32x2 (&x)[4])
    {
        asm volatile("st.global.L1::no_allocate.v4.u32 [%0], {%1, %2, %3, %4};" ::"l"(p), "r"(narrow2(x[0])), "r"(narrow2(x[1])), "r"(narrow2(x[2])),
                     "r"(narrow2(x[3])) : "memory");
    }
};
// kPairs pairs of a vector that every row reads, from element p on (a 16-byte boundary).
template <typename TW, int kPairs>
__device__ __forceinline__ void read_vector(const TW *p, f32x2 (&x)[kPairs])
{
    constexpr int kEach = Few<TW>::kPairs;
    if constexpr (kEach > kPairs) {      // fp32 rows, bf16 vector: 8 bytes of it
        const uint2 t = __ldg(reinterpret_cast<const uint2 *>(p));
        x[0] = widen2(t.x);
        x[1] = widen2(t.y);
    } else {
#pragma unroll
        for (int i = 0; i < kPairs; i += kEach) {
            Few<TW> t;
            t.read(p + 2 * i);
#pragma unroll
            for (int j = 0; j < kEach; ++j) x[i + j] = t.get(j);
        }
    }
}

// Eight consecutive elements as four pairs; fp32 at a 32-byte boundary, bf16 at 16, codes of one byte at 8.  They come in
// by asynchronous copies through a warp's place in shared memory (kSlot bytes a lane), and go out past L1.  A copy
// instruction of the warp reads consecutive bytes: with two 16-byte pieces 32 bytes apart per lane, as an fp32 vector of
// eight has them, L2 would see every sector twice (2.89 against 2.25 ms for the step of a decoder with fp32 states).  So piece c
// of the 64 comes in by lane c modulo 32, and lies at c ^ (c / 8 & 1), where the reads of a quarter warp hit all banks.
template <typename T> struct Eight;
template <> struct Eight<float> {
    static constexpr int kSlot = 32;
    f32x2 v[4];
    // p: the lane's eight elements of the warp's 256, of which the first n are there (the rest reads as 0)
    static __device__ __forceinline__ void fetch(uint32_t slot, int lane, const float *p, int n)
    {
        p -= 4 * lane;
        const uint32_t to = slot + (uint32_t)(lane ^ (lane >> 3 & 1)) * 16u;
        if (n >= 256) {
            copy16(to, p);
            copy16(to + 512u, p + 128);
            return;
        }
        some(to, p, n - 4 * lane);
        some(to + 512u, p + 128, n - 4 * lane - 128);
    }
    static __device__ __forceinline__ void some(uint32_t to, const float *p, int n)
    {
        if (n >= 4) {
            copy16(to, p);
            return;
        }
        zero16(to);
        for (int i = 0; i < n; ++i) asm volatile("st.shared.f32 [%0], %1;" ::"r"(to + 4u * i), "f"(p[i]) : "memory");
    }
    __device__ __forceinline__ void read(uint32_t slot, int lane)
    {
        const uint32_t from = slot + (uint32_t)lane * 32u, odd = (uint32_t)(lane >> 2 & 1) * 16u;
        asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(v[0]), "=l"(v[1]) : "r"(from + odd) : "memory");
        asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(v[2]), "=l"(v[3]) : "r"(from + 16u - odd) : "memory");
    }
    __device__ __forceinline__ f32x2 get(int i) const { return v[i]; }
    static __device__ __forceinline__ void store(float *p, const f32x2 (&x)[4])
    {
        asm volatile("st.global.L1::no_allocate.v4.b64 [%0], {%1, %2, %3, %4};" ::"l"(p), "l"(x[0]), "l"(x[1]), "l"(x[2]), "l"(x[3]) : "memory");
    }
    // the first n of them, one by one
    static __device__ __forceinline__ void store_some(float *p, const f32x2 (&x)[4], int n)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = halves(x[i]);
            if (2 * i < n) p[2 * i] = f.x;
            if (2 * i + 1 < n) p[2 * i + 1] = f.y;
        }
    }
};
template <> struct Eight<uint16_t> {
    static constexpr int kSlot = 16;
    uint4 v;
    static __device__ __forceinline__ void fetch(uint32_t slot, int lane, const uint16_t *p, int n)
    {
        const uint32_t to = slot + lane * 16;
        if (n >= 256 || n >= 8 * lane + 8) {      // (256: known when the code is compiled)
            copy16(to, p);
            return;
        }
        n -= 8 * lane;
        zero16(to);
        for (int i = 0; i < n; ++i) asm volatile("st.shared.u16 [%0], %1;" ::"r"(to + 2u * i), "h"(p[i]) : "memory");
    }
    __device__ __forceinline__ void read(uint32_t slot, int lane)
    {
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(slot + lane * 16) : "memory");
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
    static __device__ __forceinline__ void store_some_words(uint16_t *p, uint32_t a, uint32_t b, uint32_t c, uint32_t d, int n)
    {
        const uint32_t w[4] = {a, b, c, d};
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = (uint16_t)(w[i / 2] >> 16 * (i & 1));
    }
    static __device__ __forceinline__ void store_some(uint16_t *p, const f32x2 (&x)[4], int n)
    {
        store_some_words(p, narrow2(x[0]), narrow2(x[1]), narrow2(x[2]), narrow2(x[3]), n);
    }
};
template <> struct Eight<uint8_t> {
    static constexpr int kSlot = 8;
    uint2 v;
    static __device__ __forceinline__ void fetch(uint32_t slot, int lane, const uint8_t *p, int n)
    {
        const uint32_t to = slot + lane * 8;
        if (n >= 256 || n >= 8 * lane + 8) {
            copy8(to, p);
            return;
        }
        n -= 8 * lane;
        asm volatile("st.shared.v2.u32 [%0], {%1, %1};" ::"r"(to), "r"(0u) : "memory");
        for (int i = 0; i < n; ++i) asm volatile("st.shared.u8 [%0], %1;" ::"r"(to + i), "r"((uint32_t)p[i]) : "memory");
    }
    __device__ __forceinline__ void read(uint32_t slot, int lane)
    {
        asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(slot + lane * 8) : "memory");
    }
    static __device__ __forceinline__ void store(uint8_t *p, uint32_t a, uint32_t b)
    {
        asm volatile("st.global.L1::no_allocate.v2.u32 [%0], {%1, %2};" ::"l"(p), "r"(a), "r"(b) : "memory");
    }
};

}  // namespace gg
