// Layer norm over the rows of a matrix and its gradient.
//
//     y = w xhat + b,  xhat = (x - mean) rstd,  mean = sum(x) / n,  rstd = 1 / sqrt(sum((x - mean)^2) / n + eps)
//     d = w dy:  dx = rstd (d - sum(d) / n - xhat sum(d xhat) / n),  dw = sum over rows of dy xhat,  db = sum over rows of dy
//
// n is the row length.  The variance is that of the differences from the mean (two passes over the row), so a large
// mean costs no digits.  Both directions are bound by memory: the forward pass has to read x and write y once, the
// gradient has to read x and dy and write dx once.
#include "gg_device.cuh"
#include "gg_element.cuh"
#include "gg_internal.h"

namespace gg {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

// Sum over the CTA, the same bits in every thread.  `sh` is used again by the next call.
template <int N>
__device__ __forceinline__ void block_sum(double (&v)[N], double (*sh)[kWarps])
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = warp_sum(v[i]);
    __syncthreads();
    if ((threadIdx.x & 31) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) sh[i][threadIdx.x >> 5] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] = 0.0;
        for (int w = 0; w < kWarps; ++w) v[i] += sh[i][w];
    }
}

// Any row length, stride and alignment: one CTA per row, which reads its row three times.
template <typename T, typename TW>
__global__ void __launch_bounds__(kThreads) layer_norm_kernel(const LayerNormArgs a)
{
    __shared__ double sh[1][kWarps];
    const T *x = static_cast<const T *>(a.x);
    const TW *weight = static_cast<const TW *>(a.weight), *bias = static_cast<const TW *>(a.bias);
    T *y = static_cast<T *>(a.y);
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T *xr = x + r * a.x_ld;
        T *yr = y + r * a.y_ld;
        double s[1] = {0.0};
        for (int64_t c = threadIdx.x; c < a.cols; c += kThreads) s[0] += (double)widen<T>(xr[c]);
        block_sum(s, sh);
        const double mean = s[0] / (double)a.cols;
        s[0] = 0.0;
        for (int64_t c = threadIdx.x; c < a.cols; c += kThreads) {
            const double d = (double)widen<T>(xr[c]) - mean;
            s[0] += d * d;
        }
        block_sum(s, sh);
        const float mu = (float)mean, rstd = (float)(1.0 / sqrt(s[0] / (double)a.cols + a.eps));
        for (int64_t c = threadIdx.x; c < a.cols; c += kThreads) {
            const float xhat = (widen<T>(xr[c]) - mu) * rstd;
            yr[c] = narrow<T>(fmaf(xhat, weight ? widen<TW>(weight[c]) : 1.0f, bias ? widen<TW>(bias[c]) : 0.0f));
        }
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[r] = mu;
            if (a.rstd) a.rstd[r] = rstd;
        }
    }
}

// dx for any row length, stride and alignment: one CTA per row, which reads its two rows twice.
template <typename T, typename TW>
__global__ void __launch_bounds__(kThreads) layer_norm_dx_kernel(const LayerNormGradArgs a)
{
    __shared__ double sh[2][kWarps];
    const TW *weight = static_cast<const TW *>(a.weight);
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T *xr = static_cast<const T *>(a.x) + r * a.x_ld, *dyr = static_cast<const T *>(a.dy) + r * a.dy_ld;
        T *dxr = static_cast<T *>(a.dx) + r * a.dx_ld;
        const float mean = a.mean[r], rstd = a.rstd[r];
        double s[2] = {0.0, 0.0};
        for (int64_t c = threadIdx.x; c < a.cols; c += kThreads) {
            const float d = widen<T>(dyr[c]) * (weight ? widen<TW>(weight[c]) : 1.0f);
            s[0] += (double)d;
            s[1] += (double)d * (double)((widen<T>(xr[c]) - mean) * rstd);
        }
        block_sum(s, sh);
        const float c1 = (float)(s[0] / (double)a.cols), c2 = (float)(s[1] / (double)a.cols);
        for (int64_t c = threadIdx.x; c < a.cols; c += kThreads) {
            const float d = widen<T>(dyr[c]) * (weight ? widen<TW>(weight[c]) : 1.0f), xhat = (widen<T>(xr[c]) - mean) * rstd;
            dxr[c] = narrow<T>(rstd * (d - c1 - xhat * c2));
        }
    }
}

// dw and db for any row length, stride and alignment: a CTA takes 32 columns of one slice of the rows, a warp every
// eighth row of it.  part: [2][slices][cols].
template <typename T>
__global__ void __launch_bounds__(kThreads) layer_norm_dw_kernel(const LayerNormGradArgs a, float *part, int slices)
{
    __shared__ double sh[2][kWarps][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t r0 = a.rows * blockIdx.y / slices, r1 = a.rows * (blockIdx.y + 1) / slices;
    for (int64_t c0 = (int64_t)blockIdx.x * 32; c0 < a.cols; c0 += (int64_t)gridDim.x * 32) {
        const int64_t c = c0 + lane;
        double dw = 0.0, db = 0.0;
        if (c < a.cols)
            for (int64_t r = r0 + warp; r < r1; r += kWarps) {
                const float dy = widen<T>(static_cast<const T *>(a.dy)[r * a.dy_ld + c]);
                const float xhat = (widen<T>(static_cast<const T *>(a.x)[r * a.x_ld + c]) - a.mean[r]) * a.rstd[r];
                dw += (double)dy * (double)xhat;
                db += (double)dy;
            }
        sh[0][warp][lane] = dw;
        sh[1][warp][lane] = db;
        __syncthreads();
        if (warp < 2 && c < a.cols) {
            double s = 0.0;
            for (int w = 0; w < kWarps; ++w) s += sh[warp][w][lane];
            part[((int64_t)warp * slices + blockIdx.y) * a.cols + c] = (float)s;
        }
        __syncthreads();
    }
}

// Adds the slices of a column in order.
__global__ void __launch_bounds__(kThreads) layer_norm_dw_finish_kernel(const float *part, int slices, int64_t cols, float *dweight,
                                                                       float *dbias, int accumulate)
{
    float *out = blockIdx.y == 0 ? dweight : dbias;
    if (out == nullptr) return;
    const float *p = part + (int64_t)blockIdx.y * slices * cols;
    for (int64_t c = (int64_t)blockIdx.x * kThreads + threadIdx.x; c < cols; c += (int64_t)gridDim.x * kThreads) {
        double s = 0.0;
        for (int i = 0; i < slices; ++i) s += (double)p[(int64_t)i * cols + c];
        out[c] = (float)(accumulate ? s + (double)out[c] : s);
    }
}

inline unsigned row_grid(int64_t rows) { return (unsigned)(rows < (1 << 20) ? rows : (1 << 20)); }

}  // namespace

cudaError_t launch_layer_norm(const LayerNormArgs &a, cudaStream_t st)
{
    if (a.rows <= 0 || a.cols <= 0) return cudaSuccess;
    const unsigned grid = row_grid(a.rows);
    if (a.dtype == GG_F32 && a.w_dtype == GG_F32) layer_norm_kernel<float, float><<<grid, kThreads, 0, st>>>(a);
    else if (a.dtype == GG_F32) layer_norm_kernel<float, uint16_t><<<grid, kThreads, 0, st>>>(a);
    else if (a.w_dtype == GG_F32) layer_norm_kernel<uint16_t, float><<<grid, kThreads, 0, st>>>(a);
    else layer_norm_kernel<uint16_t, uint16_t><<<grid, kThreads, 0, st>>>(a);
    return cudaGetLastError();
}

int layer_norm_grad_slices(int64_t rows, int64_t cols, int sm_count)
{
    const int64_t strips = (cols + 31) / 32, most = (rows + 63) / 64;
    int64_t s = (4 * (int64_t)sm_count + strips - 1) / strips;
    s = s < most ? s : most;
    return (int)(s < 1 ? 1 : s);
}

cudaError_t launch_layer_norm_grad(const LayerNormGradArgs &a, float *part, int slices, int *launches, cudaStream_t st)
{
    *launches = 0;
    if (a.cols <= 0) return cudaSuccess;
    if (a.dweight != nullptr || a.dbias != nullptr) {      // (first: dx may be written over x or dy)
        const int64_t strips = (a.cols + 31) / 32;
        const dim3 grid((unsigned)(strips < (1 << 20) ? strips : (1 << 20)), (unsigned)slices);
        if (a.dtype == GG_F32) layer_norm_dw_kernel<float><<<grid, kThreads, 0, st>>>(a, part, slices);
        else layer_norm_dw_kernel<uint16_t><<<grid, kThreads, 0, st>>>(a, part, slices);
        const int64_t cb = (a.cols + kThreads - 1) / kThreads;
        layer_norm_dw_finish_kernel<<<dim3((unsigned)(cb < (1 << 20) ? cb : (1 << 20)), 2), kThreads, 0, st>>>(
            part, slices, a.cols, a.dweight, a.dbias, a.accumulate);
        *launches += 2;
    }
    if (a.dx != nullptr && a.rows > 0) {
        const unsigned grid = row_grid(a.rows);
        if (a.dtype == GG_F32 && a.w_dtype == GG_F32) layer_norm_dx_kernel<float, float><<<grid, kThreads, 0, st>>>(a);
        else if (a.dtype == GG_F32) layer_norm_dx_kernel<float, uint16_t><<<grid, kThreads, 0, st>>>(a);
        else if (a.w_dtype == GG_F32) layer_norm_dx_kernel<uint16_t, float><<<grid, kThreads, 0, st>>>(a);
        else layer_norm_dx_kernel<uint16_t, uint16_t><<<grid, kThreads, 0, st>>>(a);
        *launches += 1;
    }
    return cudaGetLastError();
}

}  // namespace gg
