// The AdamW step over a list of tensors, with its states in fp32 or in 8 bits, and the global norm of the gradient.
//
//     m <- b1 m + (1 - b1) g        v <- b2 v + (1 - b2) g^2
//     w <- w (1 - lr decay) - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// Every product and sum of m and v is one fp32 rounding, none contracted: the 8-bit codes then depend on the definition
// alone.
//
// 8-bit states: m and r = sqrt(v) are held as e4m3 codes with one fp32 scale for each kBlock elements of a tensor
// (from its start), the largest magnitude of the block at 448.  e4m3 spans 2^18 from that down, so r spans 2^36 of
// v, which a format for v itself would need twice the exponent bits for; and r is what the step divides by.  A code
// is 6 to 12 % from the next one while one step moves v by 0.1 % (b2 = 0.999): rounding to nearest would leave most
// codes where they are for ever.  So the codes are rounded up or down with the probabilities that keep the mean, from
// 16 random bits each (8 bits would resolve 1/256 of a code, about one step's change).  bf16 weights without an fp32
// copy lose small updates in the same way and are rounded in the same way.
// The random bits come from Philox4x32-10 at counter (j, j / 2^32, t, tensor) and key = seed; a block serves the
// elements 8 j .. 8 j + 7 of a tensor with 16 bits u each: element e takes u[e] for m, u[e + 4] for r and u[e + 2]
// for w (indices modulo 8), so that the three roundings of one element are independent.
#include <cuda_fp16.h>

#include "gg_adamw.cuh"
#include "gg_device.cuh"
#include "gg_element.cuh"
#include "gg_internal.h"
#include "gg_philox.cuh"

namespace gg {
namespace {

constexpr int kThreads = kStepWarps * 32;
constexpr int kPerLane = kBlock / 32;
constexpr float kZeroRoot = 0x1p-62f;      // roots of v up to this count as 0 (see sqrt2)
constexpr int kDepth = 3;                  // blocks of a warp in flight or at work

// The entry of the table that owns tile t: the lanes look at N / 32 evenly spaced entries each.  (All lanes of a warp at
// once: a search by halves would wait for the parameters six to nine times over, about 2 us of a small step's 6.)
template <int N>
__device__ __forceinline__ int find_entry(const StepTable<N> &tab, int32_t t)
{
    constexpr int kStride = N / 32;
    const int lane = threadIdx.x & 31;
    const int coarse = 31 - __clz(__ballot_sync(0xFFFFFFFFu, tab.tile0[lane * kStride] <= t));      // (entry 0 starts at tile 0)
    const int fine = __ballot_sync(0xFFFFFFFFu, lane < kStride && tab.tile0[coarse * kStride + (lane & (kStride - 1))] <= t);
    return coarse * kStride + 31 - __clz(fine);
}

struct Element { float w, m, v, r; };

// One element with fp32 states: gradient g and states (m, v) in, new weight (before its rounding), states and root out.
// The root and the quotient come from the approximate reciprocal root and reciprocal, the root with one Newton step (see
// sqrt2): the weight is within a few units of the step's rounding, and no branch keeps eight elements from overlapping
// (the correctly rounded root and division take 4.3 against 2.4 us for 49 vectors of 896).  A v below 2^-126 counts as 0.
__device__ __forceinline__ Element adamw_element(const StepScalars &c, float keep, float w, float g, float m, float v)
{
    Element e;
    e.m = __fadd_rn(__fmul_rn(c.b1.x, m), __fmul_rn(c.one_b1.x, g));
    e.v = __fadd_rn(__fmul_rn(c.b2.x, v), __fmul_rn(c.one_b2.x, __fmul_rn(g, g)));
    float y;
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(e.v));
    const float s = __fmul_rn(e.v, y), r = __fmaf_rn(__fmaf_rn(-s, s, e.v), 0.5f * y, s);
    e.r = e.v >= 0x1p-126f ? (e.v < INFINITY ? r : e.v) : (e.v >= 0.0f ? 0.0f : e.v);       // (nan stays nan)
    e.w = __fmaf_rn(c.step.x, __fmul_rn(e.m, rcp_approx(__fmaf_rn(e.r, c.root.x, c.eps.x))), __fmul_rn(w, keep));
    return e;
}

// The same for 8-bit states, bit for bit what step_eight does with pairs.
__device__ __forceinline__ Element adamw_element_narrow(const StepScalars &c, float keep, float w, float g, float m, float v)
{
    Element e;
    e.m = __fadd_rn(__fmul_rn(c.b1.x, m), __fmul_rn(c.one_b1.x, g));
    e.v = __fadd_rn(__fmul_rn(c.b2.x, v), __fmul_rn(c.one_b2.x, __fmul_rn(g, g)));
    const float v1 = __fadd_rn(e.v, 0x1p-126f);
    float y;
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(v1));
    const float r = __fmul_rn(v1, y);
    e.r = e.v < INFINITY ? __fmaf_rn(__fmaf_rn(-r, r, v1), 0.5f * y, r) : e.v;
    e.w = __fmaf_rn(c.step.x, __fmul_rn(e.m, rcp_approx(__fmaf_rn(e.r, c.root.x, c.eps.x))), __fmul_rn(w, keep));
    return e;
}

__device__ __forceinline__ uint16_t bf16_stochastic(float x, uint32_t u)
{
    const uint32_t b = __float_as_uint(x);
    if ((b & 0x7F800000u) == 0x7F800000u) return narrow<uint16_t>(x);      // inf and nan stay what they are
    return (uint16_t)((b + u) >> 16);
}

// The largest |x| of the block over the warp, inf and nan left out.
__device__ __forceinline__ float block_top(const float (&x)[kPerLane])
{
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < kPerLane; ++k) {
        const uint32_t b = __float_as_uint(x[k]) & 0x7FFFFFFFu;
        if (b < 0x7F800000u && b > top) top = b;
    }
    return __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, top));
}

// The scales of a block's states and what their values are multiplied by, 448 / top: a quotient from the approximate reciprocal with
// one Newton step on its remainder, which rounds to nearest (but for about one in a million).
constexpr float kLargeTop = 16384.0f;
__device__ __forceinline__ float2 block_scales(float m_top, float r_top, float2 &scale)
{
    const f32x2 top = pair(m_top, r_top), y = pair(rcp_approx(m_top), rcp_approx(r_top)), q = mul2(y, both(448.0f));
    const f32x2 rest = fma2(pair(-m_top, -r_top), q, both(448.0f));
    const float2 inv = halves(fma2(rest, y, q)), s = halves(mul2(top, both(1.0f / 448.0f)));
    const bool m_fits = m_top > 0x1p-110f, r_fits = r_top > kZeroRoot;
    scale = make_float2(m_fits ? s.x : 0.0f, r_fits ? s.y : 0.0f);
    return make_float2(m_fits ? inv.x : 0.0f, r_fits ? inv.y : 0.0f);
}

// x times `inv` (448 / top, or 0) as an e4m3 code.  Below 2^-6 the codes are spaced like the binade above it: adding
// 2^-6 puts both cases on one grid of 2^20 units of the fp32 pattern.  A value that was inf or nan becomes nan.
__device__ __forceinline__ uint8_t e4m3_stochastic(float x, float inv, uint32_t u, bool keep_above_zero)
{
    const float y = __fmul_rn(x, inv), a = fabsf(y);
    const bool small = a < 0.015625f;
    const float t = small ? __fadd_rn(a, 0.015625f) : a;
    uint32_t code = ((__float_as_uint(t) + (u * 16u + 8u)) >> 20) - (small ? 968u : 960u);
    code = min(code, 126u);
    if (keep_above_zero && code == 0u && a > 0.0f && x > kZeroRoot) code = 1u;
    if ((__float_as_uint(x) & 0x7F800000u) == 0x7F800000u) code = 127u;
    return (uint8_t)(code | (__float_as_uint(x) >> 31 << 7));
}

__device__ __forceinline__ float e4m3_value(uint8_t code)
{
    const uint32_t k = code & 0x7Fu, s = (uint32_t)(code & 0x80u) << 24;
    if (k == 0x7Fu) return __uint_as_float(0x7FC00000u);
    const float a = k >= 8u ? __uint_as_float((k + 960u) << 20) : (float)k * 0.001953125f;      // 2^-9
    return __uint_as_float(__float_as_uint(a) | s);
}

template <bool kNarrow> struct State { using type = float; };
template <> struct State<true> { using type = uint8_t; };

// Where a warp is in its tensor: each lane points at its eight elements of the block.
template <typename TW, typename TG, bool kNarrow>
struct Place {
    using TS = typename State<kNarrow>::type;
    TW *w;
    const TG *g;
    TS *m, *v;
    uint16_t *copy;            // or null
    uint64_t block;            // of the tensor
    uint32_t id;
#ifdef GG_BOUNDS
    int64_t len;               // of the tensor
#endif

    __device__ __forceinline__ void shift(int elements)
    {
        w += elements;
        g += elements;
        m += elements;
        v += elements;
        if (copy) copy += elements;
    }

    __device__ __forceinline__ void advance()
    {
        shift(kBlock);
        ++block;
    }
    // The noise of the eight elements from 8 * lane on.
    __device__ __forceinline__ Block4 noise(const StepScalars &c, int lane) const
    {
        const uint64_t j = block * 32u + (uint32_t)lane;
        return philox4x32_10((uint32_t)j, (uint32_t)(j >> 32), c.t, id, c.key);
    }
};

// One block of n elements at any alignment, with any values: lane l takes the elements l, l + 32, ...  Takes and returns the
// scales of the block's states in m and in sqrt(v).
template <typename TW, typename TG, bool kNarrow>
__device__ __noinline__ float2 step_block_any(Place<TW, TG, kNarrow> at, int n, const StepScalars &c, float keep, float gscale, float2 scale, uint32_t *noise)
{
    const int lane = threadIdx.x & 31;
    at.shift(-8 * lane);       // all lanes at the block's start
    const uint16_t *u = reinterpret_cast<const uint16_t *>(noise);
    if (kNarrow || sizeof(TW) == 2) {
        const Block4 q = at.noise(c, lane);
        __syncwarp();
        reinterpret_cast<uint4 *>(noise)[lane] = make_uint4(q.w0, q.w1, q.w2, q.w3);
        __syncwarp();
    }
    float mm[kPerLane], rr[kPerLane];
#pragma unroll
    for (int k = 0; k < kPerLane; ++k) {
        const int e = 32 * k + lane;
        mm[k] = rr[k] = 0.0f;
        if (e >= n || !GG_IN_BOUNDS((int64_t)at.block * kBlock + e, at.len)) continue;
        const float wf = widen<TW>(at.w[e]), gf = __fmul_rn(widen<TG>(at.g[e]), gscale);
        Element x;
        if constexpr (kNarrow) {
            const float r = __fmul_rn(e4m3_value(at.v[e]), scale.y);
            x = adamw_element_narrow(c, keep, wf, gf, __fmul_rn(e4m3_value(at.m[e]), scale.x), __fmul_rn(r, r));
            mm[k] = x.m;
            rr[k] = x.r;
        } else {
            x = adamw_element(c, keep, wf, gf, at.m[e], at.v[e]);
            at.m[e] = x.m;
            at.v[e] = x.v;
        }
        if constexpr (sizeof(TW) == 2) at.w[e] = bf16_stochastic(x.w, u[(e & ~7) + ((e + 2) & 7)]);
        else at.w[e] = x.w;
        if (at.copy) at.copy[e] = narrow<uint16_t>(x.w);
    }
    if constexpr (kNarrow) {
        const float m_top = block_top(mm), r_top = block_top(rr);
        float2 inv = block_scales(m_top, r_top, scale);
        if (m_top > kLargeTop) inv.x = __fdiv_rn(448.0f, m_top);       // (the reciprocal of the largest numbers is subnormal)
        if (r_top > kLargeTop) inv.y = __fdiv_rn(448.0f, r_top);
#pragma unroll
        for (int k = 0; k < kPerLane; ++k) {
            const int e = 32 * k + lane;
            if (e >= n || !GG_IN_BOUNDS((int64_t)at.block * kBlock + e, at.len)) continue;
            at.m[e] = e4m3_stochastic(mm[k], inv.x, u[e], false);
            at.v[e] = e4m3_stochastic(rr[k], inv.y, u[(e & ~7) + ((e + 4) & 7)], true);
        }
    }
    return scale;
}

// Blocks at vector boundaries: lane l takes the eight elements from 8 l on, in pairs.  Beyond the end of a tensor's last block
// it computes on zeros and stores nothing.  kRagged: the end is within the eight elements of a lane, and every
// lane stores one by one (it is one block of a tensor at most).  (A case of its own: within the other it takes 1.12 against 1.04 ms for a decoder with 8-bit
// states and bf16 weights.)
template <typename TW, typename TG, bool kNarrow>
struct Operands {
    using TS = typename State<kNarrow>::type;
    static constexpr int kSlot = 32 * (Eight<TW>::kSlot + Eight<TG>::kSlot + 2 * Eight<TS>::kSlot);
    Eight<TW> w;
    Eight<TG> g;
    Eight<TS> m, v;
    // the block `ahead` elements on, n elements of it
    static __device__ __forceinline__ void fetch(uint32_t slot, int lane, const Place<TW, TG, kNarrow> &at, int ahead, int n)
    {
        if (n > 0 && !GG_IN_BOUNDS((int64_t)at.block * kBlock + ahead + min(n, kBlock) - 1, at.len)) return;
        if (n >= kBlock) fetch_from(slot, lane, at.g + ahead, at.w + ahead, at.m + ahead, at.v + ahead, kBlock);
        else if (n > 0) fetch_some(slot, lane, at.g + ahead, at.w + ahead, at.m + ahead, at.v + ahead, n);
    }
    static __device__ __forceinline__ void fetch_from(uint32_t slot, int lane, const TG *g, const TW *w, const TS *m, const TS *v, int n)
    {
        Eight<TG>::fetch(slot, lane, g, n);
        slot += 32 * Eight<TG>::kSlot;
        Eight<TW>::fetch(slot, lane, w, n);
        slot += 32 * Eight<TW>::kSlot;
        Eight<TS>::fetch(slot, lane, m, n);
        slot += 32 * Eight<TS>::kSlot;
        Eight<TS>::fetch(slot, lane, v, n);
    }
    // (a call: its code in the loop would cost the others registers, 1.10 against 1.04 ms for a decoder with 8-bit states)
    static __device__ __noinline__ void fetch_some(uint32_t slot, int lane, const TG *g, const TW *w, const TS *m, const TS *v, int n)
    {
        fetch_from(slot, lane, g, w, m, v, n);
    }
    __device__ __forceinline__ void read(uint32_t slot, int lane)
    {
        g.read(slot, lane);
        slot += 32 * Eight<TG>::kSlot;
        w.read(slot, lane);
        slot += 32 * Eight<TW>::kSlot;
        m.read(slot, lane);
        slot += 32 * Eight<TS>::kSlot;
        v.read(slot, lane);
    }
    // What a step stores of a lane with n <= 8 elements, 8-bit states.
    static __device__ __forceinline__ void put_some(uint32_t slot, const Place<TW, TG, kNarrow> &at, int n, const f32x2 (&wn)[4], const uint32_t (&out)[4],
                                                    const uint32_t (&mc)[2], const uint32_t (&vc)[2])
    {
        const uint32_t lane = threadIdx.x & 31;
        const uint32_t c_at = slot + 16u * lane, w_at = slot + 32u * Eight<TG>::kSlot + Eight<TW>::kSlot * lane;
        const uint32_t m_at = slot + 32u * (Eight<TG>::kSlot + Eight<TW>::kSlot) + 8u * lane, v_at = m_at + 256u;
        asm volatile("st.shared.v2.u32 [%0], {%1, %2};" ::"r"(m_at), "r"(mc[0]), "r"(mc[1]) : "memory");
        asm volatile("st.shared.v2.u32 [%0], {%1, %2};" ::"r"(v_at), "r"(vc[0]), "r"(vc[1]) : "memory");
        if constexpr (sizeof(TW) == 2) {
            asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(w_at), "r"(out[0]), "r"(out[1]), "r"(out[2]), "r"(out[3]) : "memory");
        } else {
            asm volatile("st.shared.v2.b64 [%0], {%1, %2};" ::"r"(w_at), "l"(wn[0]), "l"(wn[1]) : "memory");
            asm volatile("st.shared.v2.b64 [%0], {%1, %2};" ::"r"(w_at + 16u), "l"(wn[2]), "l"(wn[3]) : "memory");
        }
        if (at.copy)
            asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(c_at), "r"(narrow2(wn[0])), "r"(narrow2(wn[1])), "r"(narrow2(wn[2])),
                         "r"(narrow2(wn[3])) : "memory");
#pragma unroll 1
        for (int i = 0; i < n; ++i) {
            uint32_t a, b;
            asm volatile("ld.shared.u8 %0, [%1];" : "=r"(a) : "r"(m_at + i) : "memory");
            asm volatile("ld.shared.u8 %0, [%1];" : "=r"(b) : "r"(v_at + i) : "memory");
            at.m[i] = (TS)a;
            at.v[i] = (TS)b;
            if constexpr (sizeof(TW) == 2) {
                uint16_t h;
                asm volatile("ld.shared.u16 %0, [%1];" : "=h"(h) : "r"(w_at + 2u * i) : "memory");
                at.w[i] = h;
            } else {
                float f;
                asm volatile("ld.shared.f32 %0, [%1];" : "=f"(f) : "r"(w_at + 4u * i) : "memory");
                at.w[i] = f;
            }
            if (at.copy) {
                uint16_t h;
                asm volatile("ld.shared.u16 %0, [%1];" : "=h"(h) : "r"(c_at + 2u * i) : "memory");
                at.copy[i] = h;
            }
        }
    }
};

// The new weights (`out`: rounded, two a word, for bf16), and their copy.
template <typename TW, typename TG, bool kNarrow>
__device__ __forceinline__ void store_weights(const Place<TW, TG, kNarrow> &at, const f32x2 (&wn)[4], const uint32_t (&out)[4])
{
    if constexpr (sizeof(TW) == 2) Eight<uint16_t>::store_words(at.w, out[0], out[1], out[2], out[3]);
    else Eight<float>::store(at.w, wn);
    if (at.copy) Eight<uint16_t>::store(at.copy, wn);
}
template <typename TW, typename TG, bool kNarrow>
__device__ __forceinline__ void store_some_weights(const Place<TW, TG, kNarrow> &at, const f32x2 (&wn)[4], const uint32_t (&out)[4], int n)
{
    if constexpr (sizeof(TW) == 2) Eight<uint16_t>::store_some_words(at.w, out[0], out[1], out[2], out[3], n);
    else Eight<float>::store_some(at.w, wn, n);
    if (at.copy) Eight<uint16_t>::store_some(at.copy, wn, n);
}

// States in fp32: bound by memory with room to spare, so the arithmetic is the plain one.
template <bool kRagged, typename TW, typename TG>
__device__ __forceinline__ float2 step_eight(Operands<TW, TG, false> &x, const Place<TW, TG, false> &at, int n, const StepScalars &c, float keep, float gscale, float2 scale, uint32_t *, uint32_t)
{
    f32x2 wn[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 wf = halves(x.w.get(i)), gf = halves(x.g.get(i)), mf = halves(x.m.get(i)), vf = halves(x.v.get(i));
        const Element a = adamw_element(c, keep, wf.x, __fmul_rn(gf.x, gscale), mf.x, vf.x);
        const Element b = adamw_element(c, keep, wf.y, __fmul_rn(gf.y, gscale), mf.y, vf.y);
        wn[i] = pair(a.w, b.w);
        x.m.v[i] = pair(a.m, b.m);
        x.v.v[i] = pair(a.v, b.v);
    }
    const int mine = n - 8 * (int)(threadIdx.x & 31);
    if (mine <= 0 || !GG_IN_BOUNDS((int64_t)at.block * kBlock + min(8 * (int)(threadIdx.x & 31) + 8, kRagged ? n : kBlock) - 1, at.len)) return scale;
    uint32_t out[4] = {0u, 0u, 0u, 0u};
    if constexpr (sizeof(TW) == 2) {
        const Block4 q = at.noise(c, threadIdx.x & 31);
        const uint32_t word[4] = {q.w1, q.w2, q.w3, q.w0};      // element e takes u[e + 2]
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = halves(wn[i]);
            out[i] = (uint32_t)bf16_stochastic(f.x, word[i] & 0xFFFFu) | ((uint32_t)bf16_stochastic(f.y, word[i] >> 16) << 16);
        }
    }
    if constexpr (kRagged) {
        Eight<float>::store_some(at.m, x.m.v, mine);
        Eight<float>::store_some(at.v, x.v.v, mine);
        store_some_weights(at, wn, out, mine);
    } else {
        Eight<float>::store(at.m, x.m.v);
        Eight<float>::store(at.v, x.v.v);
        store_weights(at, wn, out);
    }
    return scale;
}

// The four e4m3 codes of a word, as two pairs.
__device__ __forceinline__ void e4m3_pairs(uint32_t w, f32x2 &lo, f32x2 &hi)
{
    uint32_t a, b;
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}" : "=r"(a), "=r"(b) : "r"(w));
    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&a)), g = __half22float2(*reinterpret_cast<const __half2 *>(&b));
    lo = pair(f.x, f.y);
    hi = pair(g.x, g.y);
}

// The largest of three; a nan is passed over.
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// sqrt of finite values >= 0 by one Newton step from an approximate reciprocal root y: g = v y, g + (v - g^2) y / 2, the
// remainder v - g^2 exact.  That leaves the rounding of the last sum (and, once in about a million, the neighbour of the
// nearest value; with g (1/2 - g y / 2) for the step, half of the rounding of g stays, one value in ten).  2^-126 is
// added to v, so that y is finite: it changes no v above 2^-102, and the step divides by the root plus eps, beside which
// nothing below that shows (unless eps is below 2^-51 too).  The root of 0 comes out as 2^-63, and roots up to kZeroRoot count as 0.
__device__ __forceinline__ f32x2 sqrt2(f32x2 v)
{
    v = add2(v, both(0x1p-126f));
    const float2 f = halves(v);
    float a, b;
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(a) : "f"(f.x));
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(b) : "f"(f.y));
    const f32x2 y = pair(a, b), g = mul2(v, y);
    return fma2(fma2(mul2(g, both(-1.0f)), g, v), mul2(y, both(0.5f)), g);
}

// The top bytes of four words, in order.
__device__ __forceinline__ uint32_t top_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    return __byte_perm(__byte_perm(a, b, 0x0073), __byte_perm(c, d, 0x0073), 0x5410);
}

// States in 8 bits move 10 to 14 bytes an element, in which time an SM can issue about 50 instructions for it: here the
// arithmetic is what counts, and everything goes in pairs.  Codes: multiplied by 2^-120 the range of e4m3 becomes that
// of the smallest fp32 numbers, subnormals on subnormals, and a code is bits 20 .. 26 of the fp32 pattern; shifted by
// four it is the top byte.  The largest code cannot round up past 126: x (448 / top) exceeds 448 by at most two units
// of its pattern, and the noise stays eight short of a whole code.  A block that holds an inf or nan, or values so
// large that 2^-120 448 / top is not a normal number, goes through step_block_any; nothing is stored before that is known.
template <bool kRagged, typename TW, typename TG>
__device__ __forceinline__ float2 step_eight(Operands<TW, TG, true> &x, const Place<TW, TG, true> &at, int n, const StepScalars &c, float keep, float gscale, float2 scale, uint32_t *noise, uint32_t slot)
{
    using Data = Operands<TW, TG, true>;
    f32x2 wn[4], mn[4], rn[4];
    f32x2 sum = 0;
    float m_top = 0.0f, r_top = 0.0f;
    {
        const f32x2 b1 = pair(c.b1), one_b1 = pair(c.one_b1), b2 = pair(c.b2), one_b2 = pair(c.one_b2), gs = both(gscale);
        const f32x2 ms = both(scale.x), vs = both(scale.y), root = pair(c.root), eps = pair(c.eps), step = pair(c.step), keep2 = both(keep);
        f32x2 m_old[4], r_old[4];
        e4m3_pairs(x.m.v.x, m_old[0], m_old[1]);
        e4m3_pairs(x.m.v.y, m_old[2], m_old[3]);
        e4m3_pairs(x.v.v.x, r_old[0], r_old[1]);
        e4m3_pairs(x.v.v.y, r_old[2], r_old[3]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x2 gi = mul2(x.g.get(i), gs), mo = mul2(m_old[i], ms), ro = mul2(r_old[i], vs);
            mn[i] = add2_apart(mul2(b1, mo), mul2(one_b1, gi));
            rn[i] = sqrt2(add2_apart(mul2(b2, mul2(ro, ro)), mul2(one_b2, mul2(gi, gi))));
            const float2 d = halves(fma2(rn[i], root, eps));
            wn[i] = fma2(step, mul2(mn[i], pair(rcp_approx(d.x), rcp_approx(d.y))), mul2(x.w.get(i), keep2));
            sum = i == 0 ? wn[0] : add2(sum, wn[i]);
            const float2 mf = halves(mn[i]), rf = halves(rn[i]);
            m_top = max3(m_top, fabsf(mf.x), fabsf(mf.y));
            r_top = max3(r_top, rf.x, rf.y);
        }
        // (a maximum passes over a nan, but a nan in m or r is one in w too, and so in the sum)
        const float2 sf = halves(sum);
        if (!isfinite(sf.x + sf.y)) m_top = INFINITY;
    }
    m_top = __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(m_top)));
    r_top = __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(r_top)));
    if (fmaxf(m_top, r_top) > kLargeTop) {
        return step_block_any<TW, TG, true>(at, n, c, keep, gscale, scale, noise);
    }
    const float2 inv = block_scales(m_top, r_top, scale);
    const Block4 q = at.noise(c, threadIdx.x & 31);
    const uint32_t word[4] = {q.w0, q.w1, q.w2, q.w3};
    uint32_t u[8], mt[8], vt[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {       // (u[e] * 16 + 8) * 16
        u[2 * i] = __byte_perm(word[i], 0x80u, 0x5104);
        u[2 * i + 1] = __byte_perm(word[i], 0x80u, 0x5324);
    }
    const f32x2 m_inv = both(inv.x * 0x1p-120f), v_inv = both(inv.y * 0x1p-120f);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 zm = halves(mul2(mn[i], m_inv)), zr = halves(mul2(rn[i], v_inv));
        mt[2 * i] = (__float_as_uint(zm.x) << 4) + u[2 * i];
        mt[2 * i + 1] = (__float_as_uint(zm.y) << 4) + u[2 * i + 1];
        vt[2 * i] = (__float_as_uint(zr.x) << 4) + u[2 * i + 4 & 7];
        vt[2 * i + 1] = (__float_as_uint(zr.y) << 4) + u[2 * i + 5 & 7];
    }
    uint32_t mc[2], vc[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const float2 s0 = halves(mn[2 * h]), s1 = halves(mn[2 * h + 1]);
        const uint32_t sign = top_bytes(__float_as_uint(s0.x), __float_as_uint(s0.y), __float_as_uint(s1.x), __float_as_uint(s1.y));
        mc[h] = top_bytes(mt[4 * h], mt[4 * h + 1], mt[4 * h + 2], mt[4 * h + 3]) | sign & 0x80808080u;
        vc[h] = top_bytes(vt[4 * h], vt[4 * h + 1], vt[4 * h + 2], vt[4 * h + 3]);
        if ((vc[h] - 0x01010101u & ~vc[h] & 0x80808080u) != 0u && inv.y > 0.0f) {       // a code of 0: 1 unless the root is 0
            const float2 r0 = halves(rn[2 * h]), r1 = halves(rn[2 * h + 1]);
            const float r[4] = {r0.x, r0.y, r1.x, r1.y};
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if ((vc[h] >> 8 * i & 0xFFu) == 0u && r[i] > kZeroRoot) vc[h] |= 1u << 8 * i;
        }
    }
    if (8 * (int)(threadIdx.x & 31) >= n || !GG_IN_BOUNDS((int64_t)at.block * kBlock + min(8 * (int)(threadIdx.x & 31) + 8, kRagged ? n : kBlock) - 1, at.len)) return scale;
    if constexpr (!kRagged) {
        Eight<uint8_t>::store(at.m, mc[0], mc[1]);
        Eight<uint8_t>::store(at.v, vc[0], vc[1]);
    }
    uint32_t out[4] = {0u, 0u, 0u, 0u};
    if constexpr (sizeof(TW) == 2)
#pragma unroll
        for (int i = 0; i < 4; ++i) {       // element e takes u[e + 2]
            const float2 f = halves(wn[i]);
            const uint32_t k = word[i + 1 & 3];
            out[i] = __byte_perm(__float_as_uint(f.x) + (k & 0xFFFFu), __float_as_uint(f.y) + (k >> 16), 0x7632);
        }
    // the end of a tensor goes through the warp's places of the ring (all lanes have read them: their maxima are known)
    if constexpr (kRagged) Data::put_some(slot, at, min(n - 8 * (int)(threadIdx.x & 31), 8), wn, out, mc, vc);
    else store_weights(at, wn, out);
    return scale;
}

// (A call, for the loop's registers: inlined, 1.10 against 1.04 ms for a decoder with 8-bit states.)
template <typename TW, typename TG, bool kNarrow>
__device__ __noinline__ float2 step_ragged(uint32_t slot, const Place<TW, TG, kNarrow> at, int n, const StepScalars &c, float keep, float gscale,
                                           float2 scale, uint32_t *noise)
{
    Operands<TW, TG, kNarrow> x;
    x.read(slot, threadIdx.x & 31);
    return step_eight<true>(x, at, n, c, keep, gscale, scale, noise, slot);
}

// A CTA per tile, a warp per run of blocks.  A warp fetches its operands kDepth - 1 blocks ahead into places of shared
// memory that are its own (no barrier of the CTA), so that neither registers nor occupancy limit what is in flight.
template <typename TW, typename TG, bool kNarrow, int N>
__global__ void __launch_bounds__(kThreads, 4) adamw_kernel(const __grid_constant__ StepTable<N> tab, const __grid_constant__ StepScalars c)
{
    using Data = Operands<TW, TG, kNarrow>;
    extern __shared__ __align__(16) unsigned char ring[];
    __shared__ __align__(16) uint32_t noise[kStepWarps][kBlock / 2];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int s = find_entry(tab, (int32_t)blockIdx.x);
    const StepEntry &entry = tab.entry[s];
    const int32_t id = entry.id;
    Place<TW, TG, kNarrow> at;
    at.block = ((uint64_t)(blockIdx.x - tab.tile0[s]) * kStepWarps + warp) * (uint32_t)tab.per_warp;
    at.id = (uint32_t)(id & ~kAligned);
#ifdef GG_BOUNDS
    at.len = entry.len;
#endif
    const int64_t first = (int64_t)at.block * kBlock;
    int left = (int)min((int64_t)tab.per_warp * kBlock, entry.len - first);      // elements of this warp
    if (left <= 0) return;
    at.w = static_cast<TW *>(entry.w);
    at.g = static_cast<const TG *>(entry.g);
    at.m = static_cast<typename State<kNarrow>::type *>(entry.m);
    at.v = static_cast<typename State<kNarrow>::type *>(entry.v);
    at.copy = static_cast<uint16_t *>(entry.copy);
    at.w += first + 8 * lane;
    at.g += first + 8 * lane;
    at.m += first + 8 * lane;
    at.v += first + 8 * lane;
    if (at.copy) at.copy += first + 8 * lane;
    // lane l holds the scales of block l of the run
    const int64_t my_scale = (int64_t)entry.block0 + (int64_t)at.block + lane;
    const bool has_scale = kNarrow && lane * kBlock < left;
    float2 scales = has_scale ? make_float2(c.m_scale[my_scale], c.v_scale[my_scale]) : make_float2(0.0f, 0.0f);

    int fast = id < 0 ? left : 0;        // of these, through the ring
    left -= fast;
    const uint32_t slots = (uint32_t)__cvta_generic_to_shared(ring) + (uint32_t)(warp * kDepth * Data::kSlot);
#pragma unroll
    for (int d = 0; d < kDepth - 1; ++d) {
        Data::fetch(slots + d * Data::kSlot, lane, at, d * kBlock, fast - d * kBlock);
        copies_commit();
    }
    const float gscale = c.grad_scale ? __ldg(c.grad_scale) : 1.0f;
    const float keep = 1.0f - c.lr * (c.decay ? __ldg(c.decay + (id & ~kAligned)) : c.decay_all);
    if (!isfinite(gscale)) {
        copies_wait<0>();
        return;
    }
    int k = 0;
    auto scale_of = [&]() { return kNarrow ? make_float2(__shfl_sync(0xFFFFFFFFu, scales.x, k), __shfl_sync(0xFFFFFFFFu, scales.y, k)) : scales; };
    for (uint32_t d = 0; fast > 0; d = d == kDepth - 1 ? 0 : d + 1) {
        __syncwarp();      // every lane has read the place of the block before this one: the block after the next ones goes there
        Data::fetch(slots + (d == 0 ? kDepth - 1 : d - 1) * Data::kSlot, lane, at, (kDepth - 1) * kBlock, fast - (kDepth - 1) * kBlock);
        copies_commit();
        copies_wait<kDepth - 1>();
        __syncwarp();      // every lane's copies of this block have arrived
        const int n = min(fast, kBlock);
        const uint32_t slot = slots + d * Data::kSlot;
        const float2 scale = scale_of();
        float2 now;
        if (n % 8 == 0) {
            Data x;
            x.read(slot, lane);
            now = step_eight<false>(x, at, n, c, keep, gscale, scale, noise[warp], slot);
        } else {
            now = step_ragged(slot, at, n, c, keep, gscale, scale, noise[warp]);
        }
        if (lane == k) scales = now;
        at.advance();
        fast -= kBlock;
        ++k;
    }
    for (; left > 0; left -= kBlock) {
        const float2 now = step_block_any<TW, TG, kNarrow>(at, min(left, kBlock), c, keep, gscale, scale_of(), noise[warp]);
        if (lane == k) scales = now;
        at.advance();
        ++k;
    }
    if (has_scale) {
        c.m_scale[my_scale] = scales.x;
        c.v_scale[my_scale] = scales.y;
    }
}

template <typename TW, typename TG, bool kNarrow, int N>
cudaError_t launch_one(const StepTable<N> &tab, const StepScalars &c, cudaStream_t st)
{
    constexpr int kBytes = kStepWarps * kDepth * Operands<TW, TG, kNarrow>::kSlot;
    constexpr int kNoise = kNarrow || sizeof(TW) == 2 ? kStepWarps * kBlock * 2 : 0;
    static_assert(kBytes + kNoise <= 48 * 1024, "more would have to be asked for");
    adamw_kernel<TW, TG, kNarrow, N><<<(unsigned)tab.tiles, kThreads, kBytes, st>>>(tab, c);
    return cudaGetLastError();
}

template <int N>
cudaError_t launch_table(const StepTable<N> &tab, const StepScalars &c, int w_dtype, int g_dtype, bool narrow_states, cudaStream_t st)
{
    switch ((w_dtype == GG_BF16 ? 4 : 0) | (g_dtype == GG_BF16 ? 2 : 0) | (narrow_states ? 1 : 0)) {
    case 0: return launch_one<float, float, false>(tab, c, st);
    case 1: return launch_one<float, float, true>(tab, c, st);
    case 2: return launch_one<float, uint16_t, false>(tab, c, st);
    case 3: return launch_one<float, uint16_t, true>(tab, c, st);
    case 4: return launch_one<uint16_t, float, false>(tab, c, st);
    case 5: return launch_one<uint16_t, float, true>(tab, c, st);
    case 6: return launch_one<uint16_t, uint16_t, false>(tab, c, st);
    default: return launch_one<uint16_t, uint16_t, true>(tab, c, st);
    }
}

// The norm from a sum of squares (nan if an entry was not finite), and the factor that brings it down to max_norm.
__device__ __forceinline__ void write_norm(double sum, uint32_t wrong, double max_norm, double *norm, float *scale)
{
    const double r = wrong != 0u ? __longlong_as_double(0x7FF8000000000000ll) : sqrt(sum);
    if (norm) *norm = r;
    if (scale) *scale = r > max_norm ? (float)(max_norm / r) : (r == r ? 1.0f : (float)r);
}

// The norm from the tile sums of a moments sweep.
__global__ void __launch_bounds__(1024) grad_norm_kernel(const double *s2, const uint32_t *bad, int32_t n_tiles, double max_norm,
                                                         double *norm, float *scale)
{
    __shared__ double sh[32];
    __shared__ uint32_t shb[32];
    double s = 0.0;
    uint32_t b = 0;
    for (int32_t t = threadIdx.x; t < n_tiles; t += 1024) { s += s2[t]; b |= bad[t]; }
    s = warp_sum(s);
    b = __reduce_or_sync(0xFFFFFFFFu, b);
    if ((threadIdx.x & 31) == 0) { sh[threadIdx.x >> 5] = s; shb[threadIdx.x >> 5] = b; }
    __syncthreads();
    if (threadIdx.x != 0) return;
    for (int w = 1; w < 32; ++w) { s += sh[w]; b |= shb[w]; }
    write_norm(s, b, max_norm, norm, scale);
}

// The norm of few tiles in one launch: a CTA sums the squares of a tile in fp64, and the last CTA to finish adds the tiles in
// order.  `ticket` is 0 between launches.
constexpr int kNormThreads = 512;
template <typename T>
__global__ void __launch_bounds__(kNormThreads) grad_norm_small_kernel(const TileMap map, double *s2, uint32_t *bad, uint32_t *ticket, double max_norm,
                                                                      double *norm, float *scale)
{
    __shared__ double sh[kNormThreads / 32];
    __shared__ uint32_t last;
    const int t = blockIdx.x, s = map.tile_seg[t], warp = threadIdx.x >> 5;
    const int64_t off = (int64_t)(t - map.tile_prefix[s]) * kTile;
    const int n = (int)min((int64_t)kTile, map.seg_len[s] - off);
    const T *g = static_cast<const T *>(map.seg_ptr[s]) + off;
    double sum = 0.0;
    uint32_t wrong = 0;
    auto add = [&](float v) {
        if (isfinite(v)) sum = fma((double)v, (double)v, sum);
        else wrong = 1u;
    };
    constexpr int kVec = 16 / sizeof(T), kMost = kTile / kVec / kNormThreads;
    if (reinterpret_cast<uintptr_t>(g) % 16 == 0) {
        uint4 v[kMost];
#pragma unroll
        for (int i = 0; i < kMost; ++i) {
            const int e = (i * kNormThreads + (int)threadIdx.x) * kVec;
            v[i] = e + kVec <= n ? __ldg(reinterpret_cast<const uint4 *>(g + e)) : make_uint4(0u, 0u, 0u, 0u);
        }
#pragma unroll
        for (int i = 0; i < kMost; ++i)
            for (const uint32_t w : {v[i].x, v[i].y, v[i].z, v[i].w}) {
                if constexpr (sizeof(T) == 4) {
                    add(__uint_as_float(w));
                } else {
                    add(__uint_as_float(w << 16));
                    add(__uint_as_float(w & 0xFFFF0000u));
                }
            }
        for (int e = n / kVec * kVec + threadIdx.x; e < n; e += kNormThreads) add(widen<T>(g[e]));
    } else {
#pragma unroll 8
        for (int e = threadIdx.x; e < n; e += kNormThreads) add(widen<T>(g[e]));
    }
    sum = warp_sum(sum);
    wrong = __syncthreads_or((int)wrong);
    if ((threadIdx.x & 31) == 0) sh[warp] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kNormThreads / 32; ++w) sum += sh[w];
        s2[t] = sum;
        bad[t] = wrong;
        __threadfence();
        last = atomicAdd(ticket, 1u) == gridDim.x - 1u;
    }
    __syncthreads();
    if (last == 0u || warp != 0) return;
    __threadfence();
    sum = 0.0;
    wrong = 0;
    for (int i = threadIdx.x; i < (int)gridDim.x; i += 32) {
        sum += __ldcg(s2 + i);
        wrong |= __ldcg(bad + i);
    }
    sum = warp_sum(sum);
    wrong = __reduce_or_sync(0xFFFFFFFFu, wrong);
    if (threadIdx.x != 0) return;
    write_norm(sum, wrong, max_norm, norm, scale);
    *ticket = 0u;
}

}  // namespace

cudaError_t launch_adamw(const StepTable<kTableSmall> &tab, const StepScalars &c, int w_dtype, int g_dtype, bool narrow_states, cudaStream_t st)
{
    return launch_table(tab, c, w_dtype, g_dtype, narrow_states, st);
}

cudaError_t launch_adamw(const StepTable<kTableLarge> &tab, const StepScalars &c, int w_dtype, int g_dtype, bool narrow_states, cudaStream_t st)
{
    return launch_table(tab, c, w_dtype, g_dtype, narrow_states, st);
}

cudaError_t launch_grad_norm(const double *s2, const uint32_t *bad, int32_t n_tiles, double max_norm, double *norm, float *scale, cudaStream_t st)
{
    grad_norm_kernel<<<1, 1024, 0, st>>>(s2, bad, n_tiles, max_norm, norm, scale);
    return cudaGetLastError();
}

cudaError_t launch_grad_norm_small(const TileMap &map, int dtype, double *s2, uint32_t *bad, uint32_t *ticket, double max_norm, double *norm,
                                   float *scale, cudaStream_t st)
{
    const unsigned grid = (unsigned)map.n_tiles;
    if (dtype == GG_F32) grad_norm_small_kernel<float><<<grid, kNormThreads, 0, st>>>(map, s2, bad, ticket, max_norm, norm, scale);
    else grad_norm_small_kernel<uint16_t><<<grid, kNormThreads, 0, st>>>(map, s2, bad, ticket, max_norm, norm, scale);
    return cudaGetLastError();
}

}  // namespace gg
