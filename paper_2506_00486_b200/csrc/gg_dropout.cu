// Dropout whose mask is drawn again by whoever needs it (gg_dropout).
//
// Eight elements of a row share one block of 128 random bits.  A warp takes runs of 256 elements of a row: each lane draws the
// eight keep bits of one group, and the lanes then read and write the run side by side, in whatever pieces its alignment allows,
// fetching the bits of their elements from the lane that drew them.
#include "gg_after.cuh"
#include "gg_element.cuh"
#include "gg_internal.h"
#include "gg_philox.cuh"

namespace gg {
namespace {

constexpr int kWarps = 8, kRun = 256;
// Runs that a warp has under way: 4 pieces of 16 bytes a lane (bf16 [16384, 4096] with a residual 65 us; 2 runs 66, 8 runs 82), or two runs of single
// elements (fp32 [4099, 1023] 7.2 us, one run 8.1)
__host__ __device__ constexpr int together(int pieces) { return pieces >= 4 ? 2 : 4 / pieces; }

struct Keys { uint32_t k[20]; };

// The keep bits of the group's eight elements: bit e is element e's.
__device__ __forceinline__ uint32_t keep_bits(int64_t group, uint32_t t, uint32_t tensor, const Keys &keys, uint32_t least)
{
    const Block4 b = philox4x32_10((uint32_t)group, (uint32_t)(group >> 32), t, tensor, keys.k);
    const uint32_t w[4] = {b.w0, b.w1, b.w2, b.w3};
    uint32_t keep = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        keep |= (uint32_t)((w[i] & 0xFFFF) >= least) << (2 * i);
        keep |= (uint32_t)((w[i] >> 16) >= least) << (2 * i + 1);
    }
    return keep;
}

// kEach consecutive elements.
template <typename T, int kEach> struct Piece;
template <typename T> struct Piece<T, 1> {
    T v;
    __device__ __forceinline__ void read(const T *p) { v = *p; }
    __device__ __forceinline__ void write(T *p) const { *p = v; }
    __device__ __forceinline__ float get(int) const { return widen<T>(v); }
    __device__ __forceinline__ void set(const float (&x)[1]) { v = narrow<T>(x[0]); }
};
template <> struct Piece<float, 4> {
    float4 v;
    __device__ __forceinline__ void read(const float *p) { v = *reinterpret_cast<const float4 *>(p); }
    __device__ __forceinline__ void write(float *p) const { *reinterpret_cast<float4 *>(p) = v; }
    __device__ __forceinline__ float get(int i) const { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
    __device__ __forceinline__ void set(const float (&x)[4]) { v = make_float4(x[0], x[1], x[2], x[3]); }
};
template <> struct Piece<uint16_t, 8> {
    uint4 v;
    __device__ __forceinline__ void read(const uint16_t *p) { v = *reinterpret_cast<const uint4 *>(p); }
    __device__ __forceinline__ void write(uint16_t *p) const { *reinterpret_cast<uint4 *>(p) = v; }
    __device__ __forceinline__ float get(int i) const
    {
        const uint32_t w = i < 2 ? v.x : i < 4 ? v.y : i < 6 ? v.z : v.w;
        return __uint_as_float(i & 1 ? w & 0xFFFF0000u : w << 16);
    }
    __device__ __forceinline__ void set(const float (&x)[8])
    {
        v = make_uint4(narrow2(pair(x[0], x[1])), narrow2(pair(x[2], x[3])), narrow2(pair(x[4], x[5])), narrow2(pair(x[6], x[7])));
    }
};

// Pieces of kEach elements: 16 bytes where every row of every operand starts on such a boundary and is a multiple of it long, else one.
template <typename T, int kEach, bool kResidual>
__global__ void __launch_bounds__(kWarps * 32) dropout_runs_kernel(const DropoutArgs a, const Keys keys, uint32_t least, float scale, int64_t runs, int64_t total)
{
    constexpr int kPieces = kRun / (32 * kEach);         // of a lane in a run
    constexpr int kTogether = together(kPieces);
    const int lane = threadIdx.x & 31;
    wait_for_the_one_before();
    const uint32_t t = (uint32_t)(a.t + (a.t_dev ? *a.t_dev : 0));
    const int64_t groups = (a.cols + 7) / 8, first = (blockIdx.x * (int64_t)kWarps + (threadIdx.x >> 5)) * kTogether;
    Piece<T, kEach> x[kTogether][kPieces], r[kResidual ? kTogether : 1][kPieces];
    int64_t row[kTogether], start[kTogether];
#pragma unroll
    for (int u = 0; u < kTogether; ++u) {
        row[u] = total <= 0x7FFFFFFF ? (int64_t)((uint32_t)(first + u) / (uint32_t)runs) : (first + u) / runs;
        start[u] = (first + u - row[u] * runs) * kRun;
        if (first + u >= total) start[u] = a.cols;       // (nothing of it is there)
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int64_t col = start[u] + (i * 32 + lane) * kEach;
            if (col < a.cols) {
                x[u][i].read(static_cast<const T *>(a.x) + row[u] * a.x_ld + col);
                if constexpr (kResidual) r[u][i].read(static_cast<const T *>(a.residual) + row[u] * a.residual_ld + col);
            }
        }
    }
#pragma unroll
    for (int u = 0; u < kTogether; ++u) {
        const uint32_t mine = keep_bits(row[u] * groups + start[u] / 8 + lane, t, a.tensor_id, keys, least);
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int at = (i * 32 + lane) * kEach;
            const uint32_t keep = (kEach == 8 ? mine : __shfl_sync(~0u, mine, at / 8)) >> (at & 7);
            if (start[u] + at < a.cols) {
                float v[kEach];
#pragma unroll
                for (int e = 0; e < kEach; ++e) {
                    v[e] = keep >> e & 1 ? x[u][i].get(e) * scale : 0.0f;
                    if constexpr (kResidual) v[e] += r[u][i].get(e);
                }
                x[u][i].set(v);
                x[u][i].write(static_cast<T *>(a.y) + row[u] * a.y_ld + start[u] + at);
            }
        }
    }
}

// Rows much shorter than a run, with gaps or odd lengths: one thread for a group.
template <typename T>
__global__ void __launch_bounds__(kWarps * 32) dropout_groups_kernel(const DropoutArgs a, const Keys keys, uint32_t least, float scale)
{
    wait_for_the_one_before();
    const int64_t groups = (a.cols + 7) / 8;
    const uint32_t t = (uint32_t)(a.t + (a.t_dev ? *a.t_dev : 0));
    for (int64_t i = blockIdx.x * (int64_t)(kWarps * 32) + threadIdx.x; i < groups * a.rows; i += gridDim.x * (int64_t)(kWarps * 32)) {
        const int64_t row = i / groups, col = (i - row * groups) * 8;
        const uint32_t keep = keep_bits(i, t, a.tensor_id, keys, least);
        const T *x = static_cast<const T *>(a.x) + row * a.x_ld + col;
        const T *r = a.residual ? static_cast<const T *>(a.residual) + row * a.residual_ld + col : nullptr;
        T *y = static_cast<T *>(a.y) + row * a.y_ld + col;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (col + e < a.cols) {
                float v = keep >> e & 1 ? widen<T>(x[e]) * scale : 0.0f;
                if (r) v += widen<T>(r[e]);
                y[e] = narrow<T>(v);
            }
    }
}

bool whole_pieces(const void *p, int64_t rows, int64_t ld, int64_t each)
{
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (rows <= 1 || ld % each == 0);
}

template <typename T>
cudaError_t launch(DropoutArgs a, const Keys &keys, uint32_t least, float scale, int sm_count, cudaStream_t st)
{
    constexpr int kEach = 16 / sizeof(T);
    // rows of whole groups without gaps are one long row: groups are counted the same way
    if (a.cols % 8 == 0 && a.x_ld == a.cols && a.y_ld == a.cols && (!a.residual || a.residual_ld == a.cols)) {
        a.cols *= a.rows;
        a.rows = 1;
    }
    if (a.rows > 1 && a.cols < 96) {
        const int64_t want = ((a.cols + 7) / 8 * a.rows + kWarps * 32 - 1) / (kWarps * 32), most = (int64_t)sm_count * 8;
        return launch_after(st, dim3((unsigned)(want < most ? want : most)), kWarps * 32, 0, dropout_groups_kernel<T>, a, keys, least, scale);
    }
    const bool whole = a.cols % kEach == 0 && whole_pieces(a.x, a.rows, a.x_ld, kEach) && whole_pieces(a.y, a.rows, a.y_ld, kEach) &&
                       (!a.residual || whole_pieces(a.residual, a.rows, a.residual_ld, kEach));
    const int64_t runs = (a.cols + kRun - 1) / kRun, total = runs * a.rows;
    auto go = [&](auto kernel, int pieces) {
        const int64_t each = (int64_t)kWarps * together(pieces), ctas = (total + each - 1) / each;
        if (ctas > 0x7FFFFFFF) return cudaErrorInvalidValue;
        return launch_after(st, dim3((unsigned)ctas), kWarps * 32, 0, kernel, a, keys, least, scale, runs, total);
    };
    if (whole) return a.residual ? go(dropout_runs_kernel<T, kEach, true>, kRun / (32 * kEach)) : go(dropout_runs_kernel<T, kEach, false>, kRun / (32 * kEach));
    return a.residual ? go(dropout_runs_kernel<T, 1, true>, kRun / 32) : go(dropout_runs_kernel<T, 1, false>, kRun / 32);
}

}  // namespace

cudaError_t launch_dropout(const DropoutArgs &a, uint32_t least, int sm_count, cudaStream_t st)
{
    const float scale = 65536.0f / (float)(65536 - least);
    Keys keys;
    for (uint32_t r = 0; r < 10; ++r) {
        keys.k[2 * r] = (uint32_t)a.seed + r * kPhiloxW0;
        keys.k[2 * r + 1] = (uint32_t)(a.seed >> 32) + r * kPhiloxW1;
    }
    return a.dtype == GG_F32 ? launch<float>(a, keys, least, scale, sm_count, st) : launch<uint16_t>(a, keys, least, scale, sm_count, st);
}

}  // namespace gg
