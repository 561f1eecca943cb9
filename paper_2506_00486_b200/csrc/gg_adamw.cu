// The AdamW step over a list of tensors, with its states in fp32 or in 8 bits, and the global norm of the gradient.
//
//     m <- b1 m + (1 - b1) g        v <- b2 v + (1 - b2) g^2
//     w <- w (1 - lr decay) - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// Every product and sum is one fp32 rounding, none contracted: the 8-bit codes then depend on the definition alone.
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
#include "gg_adamw.cuh"
#include "gg_device.cuh"
#include "gg_element.cuh"
#include "gg_internal.h"
#include "gg_philox.cuh"

namespace gg {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kPerLane = kBlock / 32;

// The entry of the table that owns tile t.
template <int N>
__device__ __forceinline__ int find_entry(const StepTable<N> &tab, int32_t t)
{
    int lo = 0, hi = tab.n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (tab.tile0[mid] <= t) lo = mid;
        else hi = mid;
    }
    return lo;
}

struct Element { float w, m, v, r; };

// One element: gradient g and states (m, v) in, new weight (before its rounding), states and root out.
__device__ __forceinline__ Element adamw_element(const StepScalars &c, float keep, float w, float g, float m, float v)
{
    Element e;
    e.m = __fadd_rn(__fmul_rn(c.b1, m), __fmul_rn(c.one_b1, g));
    e.v = __fadd_rn(__fmul_rn(c.b2, v), __fmul_rn(c.one_b2, __fmul_rn(g, g)));
    e.r = __fsqrt_rn(e.v);
    e.w = __fmul_rn(w, keep) - c.step * (e.m / (e.r * c.root + c.eps));
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

// x times `inv` (448 / top, or 0) as an e4m3 code.  Below 2^-6 the codes are spaced like the binade above it: adding
// 2^-6 puts both cases on one grid of 2^20 units of the fp32 pattern.  A value that was inf or nan becomes nan.
__device__ __forceinline__ uint8_t e4m3_stochastic(float x, float inv, uint32_t u, bool keep_above_zero)
{
    const float y = __fmul_rn(x, inv), a = fabsf(y);
    const bool small = a < 0.015625f;
    const float t = small ? __fadd_rn(a, 0.015625f) : a;
    uint32_t code = ((__float_as_uint(t) + (u * 16u + 8u)) >> 20) - (small ? 968u : 960u);
    code = min(code, 126u);
    if (keep_above_zero && code == 0u && a > 0.0f) code = 1u;
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

// One warp per block of kBlock elements, lane l at elements l, l + 32, ...: any alignment.
template <typename TW, typename TG, bool kNarrow, int N>
__global__ void __launch_bounds__(kThreads) adamw_kernel(const __grid_constant__ StepTable<N> tab, const StepScalars c)
{
    __shared__ uint32_t noise[kWarps][kBlock / 2];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const float gscale = c.grad_scale ? __ldg(c.grad_scale) : 1.0f;
    if (!isfinite(gscale)) return;
    const int s = find_entry(tab, (int32_t)blockIdx.x);
    const int64_t len = tab.len[s];
    const float keep = 1.0f - c.lr * (c.decay ? __ldg(c.decay + tab.id[s]) : c.decay_all);
    TW *w = static_cast<TW *>(tab.w[s]);
    const TG *g = static_cast<const TG *>(tab.g[s]);
    uint16_t *copy = static_cast<uint16_t *>(tab.copy[s]);
    constexpr bool kNoise = kNarrow || sizeof(TW) == 2;
    const uint16_t *u = reinterpret_cast<const uint16_t *>(noise[warp]);

    for (int b = warp; b < kTileBlocks; b += kWarps) {
        const int64_t block = (int64_t)(blockIdx.x - tab.tile0[s]) * kTileBlocks + b;      // of the tensor
        const int64_t i0 = block * kBlock;
        if (i0 >= len) break;
        const int n = (int)min((int64_t)kBlock, len - i0);
        if (kNoise) {
            const uint64_t j = (uint64_t)block * 32u + lane;
            const Block4 q = philox4x32_10((uint32_t)j, (uint32_t)(j >> 32), c.t, (uint32_t)tab.id[s], c.seed_lo, c.seed_hi);
            __syncwarp();
            reinterpret_cast<uint4 *>(noise[warp])[lane] = make_uint4(q.w0, q.w1, q.w2, q.w3);
            __syncwarp();
        }
        float m_scale = 1.0f, v_scale = 1.0f;
        if (kNarrow) {
            m_scale = c.m_scale[tab.block0[s] + block];
            v_scale = c.v_scale[tab.block0[s] + block];
        }
        float mm[kPerLane], rr[kPerLane];
#pragma unroll
        for (int k = 0; k < kPerLane; ++k) {
            const int e = 32 * k + lane;
            mm[k] = rr[k] = 0.0f;
            if (e >= n) continue;
            const int64_t i = i0 + e;
            float m, v;
            if (kNarrow) {
                m = __fmul_rn(e4m3_value(static_cast<const uint8_t *>(tab.m[s])[i]), m_scale);
                v = __fmul_rn(e4m3_value(static_cast<const uint8_t *>(tab.v[s])[i]), v_scale);
                v = __fmul_rn(v, v);
            } else {
                m = static_cast<const float *>(tab.m[s])[i];
                v = static_cast<const float *>(tab.v[s])[i];
            }
            const Element x = adamw_element(c, keep, widen<TW>(w[i]), __fmul_rn(widen<TG>(g[i]), gscale), m, v);
            if (sizeof(TW) == 2) reinterpret_cast<uint16_t *>(w)[i] = bf16_stochastic(x.w, u[(e & ~7) + ((e + 2) & 7)]);
            else reinterpret_cast<float *>(w)[i] = x.w;
            if (copy) copy[i] = narrow<uint16_t>(x.w);
            if (kNarrow) {
                mm[k] = x.m;
                rr[k] = x.r;
            } else {
                static_cast<float *>(tab.m[s])[i] = x.m;
                static_cast<float *>(tab.v[s])[i] = x.v;
            }
        }
        if (kNarrow) {
            const float m_top = block_top(mm), r_top = block_top(rr);
            const bool m_fits = m_top > 0x1p-110f, r_fits = r_top > 0x1p-110f;
            const float m_inv = m_fits ? __fdiv_rn(448.0f, m_top) : 0.0f, r_inv = r_fits ? __fdiv_rn(448.0f, r_top) : 0.0f;
#pragma unroll
            for (int k = 0; k < kPerLane; ++k) {
                const int e = 32 * k + lane;
                if (e >= n) continue;
                static_cast<uint8_t *>(tab.m[s])[i0 + e] = e4m3_stochastic(mm[k], m_inv, u[e], false);
                static_cast<uint8_t *>(tab.v[s])[i0 + e] = e4m3_stochastic(rr[k], r_inv, u[(e & ~7) + ((e + 4) & 7)], true);
            }
            if (lane == 0) {
                c.m_scale[tab.block0[s] + block] = m_fits ? __fmul_rn(m_top, 1.0f / 448.0f) : 0.0f;
                c.v_scale[tab.block0[s] + block] = r_fits ? __fmul_rn(r_top, 1.0f / 448.0f) : 0.0f;
            }
        }
    }
}

template <int N>
cudaError_t launch_table(const StepTable<N> &tab, const StepScalars &c, int w_dtype, int g_dtype, bool narrow_states, cudaStream_t st)
{
    const dim3 grid((unsigned)tab.tile0[tab.n]), block(kThreads);
    const int which = (w_dtype == GG_BF16 ? 4 : 0) | (g_dtype == GG_BF16 ? 2 : 0) | (narrow_states ? 1 : 0);
    switch (which) {
    case 0: adamw_kernel<float, float, false, N><<<grid, block, 0, st>>>(tab, c); break;
    case 1: adamw_kernel<float, float, true, N><<<grid, block, 0, st>>>(tab, c); break;
    case 2: adamw_kernel<float, uint16_t, false, N><<<grid, block, 0, st>>>(tab, c); break;
    case 3: adamw_kernel<float, uint16_t, true, N><<<grid, block, 0, st>>>(tab, c); break;
    case 4: adamw_kernel<uint16_t, float, false, N><<<grid, block, 0, st>>>(tab, c); break;
    case 5: adamw_kernel<uint16_t, float, true, N><<<grid, block, 0, st>>>(tab, c); break;
    case 6: adamw_kernel<uint16_t, uint16_t, false, N><<<grid, block, 0, st>>>(tab, c); break;
    default: adamw_kernel<uint16_t, uint16_t, true, N><<<grid, block, 0, st>>>(tab, c); break;
    }
    return cudaGetLastError();
}

// sqrt(sum of squares) over the tile sums of a moments sweep, and the factor that brings it down to max_norm.
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
    const double r = b != 0u ? __longlong_as_double(0x7FF8000000000000ll) : sqrt(s);
    if (norm) *norm = r;
    if (scale) *scale = r > max_norm ? (float)(max_norm / r) : (r == r ? 1.0f : (float)r);
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

}  // namespace gg
