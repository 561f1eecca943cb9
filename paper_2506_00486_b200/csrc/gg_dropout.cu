// Dropout whose mask is drawn again by whoever needs it (gg_dropout).
#include "gg_element.cuh"
#include "gg_internal.h"
#include "gg_philox.cuh"

namespace gg {
namespace {

constexpr int kThreads = 256;

// Eight elements of a row share one block of 128 random bits: one thread makes them and writes the eight.
template <typename T>
__global__ void __launch_bounds__(kThreads) dropout_kernel(const DropoutArgs a, uint32_t least, float scale, int vector)
{
    const int64_t groups = (a.cols + 7) / 8;
    const uint32_t t = (uint32_t)(a.t + (a.t_dev ? *a.t_dev : 0));
    for (int64_t i = blockIdx.x * (int64_t)kThreads + threadIdx.x; i < groups * a.rows; i += gridDim.x * (int64_t)kThreads) {
        const int64_t row = i / groups, col = (i - row * groups) * 8;
        const Block4 b = philox4x32_10((uint32_t)i, (uint32_t)(i >> 32), t, a.tensor_id, (uint32_t)a.seed, (uint32_t)(a.seed >> 32));
        const uint32_t w[4] = {b.w0, b.w1, b.w2, b.w3};
        const T *x = static_cast<const T *>(a.x) + row * a.x_ld + col;
        const T *r = a.residual ? static_cast<const T *>(a.residual) + row * a.residual_ld + col : nullptr;
        T *y = static_cast<T *>(a.y) + row * a.y_ld + col;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (col + j < a.cols) {
                const uint32_t bits = j & 1 ? w[j / 2] >> 16 : w[j / 2] & 0xFFFF;
                float v = bits >= least ? widen<T>(x[j]) * scale : 0.0f;
                if (r) v += widen<T>(r[j]);
                y[j] = narrow<T>(v);
            }
    }
}

}  // namespace

cudaError_t launch_dropout(const DropoutArgs &a, uint32_t least, int sm_count, cudaStream_t st)
{
    const int64_t n = (a.cols + 7) / 8 * a.rows, want = (n + kThreads - 1) / kThreads, most = (int64_t)sm_count * 16;
    const unsigned grid = (unsigned)(want < most ? want : most);
    const float scale = 65536.0f / (float)(65536 - least);
    if (a.dtype == GG_F32) dropout_kernel<float><<<grid, kThreads, 0, st>>>(a, least, scale, 0);
    else dropout_kernel<uint16_t><<<grid, kThreads, 0, st>>>(a, least, scale, 0);
    return cudaGetLastError();
}

}  // namespace gg
