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

// ---- rows that fit the registers of their threads

// A row belongs to `warps` warps: to one warp of four in a CTA, which then need no barrier, or to all warps of its CTA.
// Thread i of a row holds the vectors i, i + T, i + 2 T, ... (T threads a row, kNum vectors each).
constexpr int kSoloWarps = 4;
template <int kNum> constexpr int kMostThreads = kNum == 1 ? 1024 : 512;        // 64 or 128 registers a thread

// Sums over the threads of a row, the same bits in every one.  `sh` alternates between two halves, so that one barrier a
// sum is enough: a thread writes a half again only after a barrier that follows every read of it.
template <int N>
__device__ __forceinline__ void row_sum(float (&v)[N], float (*sh)[N][32], int warps, int &half)
{
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v[i] += __shfl_xor_sync(0xFFFFFFFFu, v[i], o);
    if (warps == 1) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (lane == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) sh[half][i][warp] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] = lane < warps ? sh[half][i][lane] : 0.0f;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v[i] += __shfl_xor_sync(0xFFFFFFFFu, v[i], o);
    }
    half ^= 1;
}

template <typename T, typename TW, int kVec, int kNum>
__global__ void __launch_bounds__(kMostThreads<kNum>) layer_norm_rows_kernel(const LayerNormArgs a, int warps)
{
    __shared__ float sh[2][1][32];
    const int threads = warps * 32, tid = warps == 1 ? threadIdx.x & 31 : threadIdx.x;
    const int64_t row0 = warps == 1 ? (int64_t)blockIdx.x * kSoloWarps + (threadIdx.x >> 5) : blockIdx.x;
    const int64_t stride = warps == 1 ? (int64_t)gridDim.x * kSoloWarps : gridDim.x;
    const int cols = (int)a.cols;
    const float n_inv = 1.0f / (float)cols;
    const TW *weight = static_cast<const TW *>(a.weight), *bias = static_cast<const TW *>(a.bias);
    int half = 0;
    for (int64_t r = row0; r < a.rows; r += stride) {
        const T *xr = static_cast<const T *>(a.x) + r * a.x_ld;
        T *yr = static_cast<T *>(a.y) + r * a.y_ld;
        Few<T, kVec> raw[kNum];
#pragma unroll
        for (int k = 0; k < kNum; ++k) {
            const int c = (k * threads + tid) * kVec;
            if (c < cols) raw[k].load(xr + c);
        }
        float s[1] = {0.0f};
#pragma unroll
        for (int k = 0; k < kNum; ++k)
            if ((k * threads + tid) * kVec < cols) {
                float x[kVec], t = 0.0f;
                raw[k].get(x);
#pragma unroll
                for (int i = 0; i < kVec; ++i) t += x[i];
                s[0] += t;
            }
        row_sum(s, sh, warps, half);
        const float mean = s[0] * n_inv;
        s[0] = 0.0f;
#pragma unroll
        for (int k = 0; k < kNum; ++k)
            if ((k * threads + tid) * kVec < cols) {
                float x[kVec], t = 0.0f;
                raw[k].get(x);
#pragma unroll
                for (int i = 0; i < kVec; ++i) t = fmaf(x[i] - mean, x[i] - mean, t);
                s[0] += t;
            }
        row_sum(s, sh, warps, half);
        const float rstd = 1.0f / sqrtf(s[0] * n_inv + (float)a.eps);
#pragma unroll
        for (int k = 0; k < kNum; ++k) {
            const int c = (k * threads + tid) * kVec;
            if (c < cols) {
                float x[kVec], w[kVec], b[kVec];
                raw[k].get(x);
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    w[i] = 1.0f;
                    b[i] = 0.0f;
                }
                if (weight) read_shared_vector<kVec>(weight + c, w);
                if (bias) read_shared_vector<kVec>(bias + c, b);
#pragma unroll
                for (int i = 0; i < kVec; ++i) x[i] = fmaf((x[i] - mean) * rstd, w[i], b[i]);
                Few<T, kVec>::store(yr + c, x);
            }
        }
        if (tid == 0) {
            if (a.mean) a.mean[r] = mean;
            if (a.rstd) a.rstd[r] = rstd;
        }
    }
}

// The gradient: each thread keeps the sums of its columns over the rows of its CTA and leaves them as slice blockIdx.x of
// `part` ([2][gridDim.x][cols]); layer_norm_dw_finish_kernel adds the slices.
template <typename T, typename TW, int kVec, int kNum>
__global__ void __launch_bounds__(kMostThreads<kNum>) layer_norm_rows_grad_kernel(const LayerNormGradArgs a, float *part, int warps)
{
    __shared__ float sh[2][2][32];
    extern __shared__ float columns[];      // rows of single warps: [2][cols], where the CTA's four warps meet
    const int threads = warps * 32, tid = warps == 1 ? threadIdx.x & 31 : threadIdx.x;
    const int64_t row0 = warps == 1 ? (int64_t)blockIdx.x * kSoloWarps + (threadIdx.x >> 5) : blockIdx.x;
    const int64_t stride = warps == 1 ? (int64_t)gridDim.x * kSoloWarps : gridDim.x;
    const int cols = (int)a.cols;
    const float n_inv = 1.0f / (float)cols;
    const TW *weight = static_cast<const TW *>(a.weight);
    float dw[kNum][kVec], db[kNum][kVec];
#pragma unroll
    for (int k = 0; k < kNum; ++k)
#pragma unroll
        for (int i = 0; i < kVec; ++i) dw[k][i] = db[k][i] = 0.0f;
    int half = 0;
    for (int64_t r = row0; r < a.rows; r += stride) {
        const T *xr = static_cast<const T *>(a.x) + r * a.x_ld, *dyr = static_cast<const T *>(a.dy) + r * a.dy_ld;
        Few<T, kVec> raw_x[kNum], raw_dy[kNum];
#pragma unroll
        for (int k = 0; k < kNum; ++k) {
            const int c = (k * threads + tid) * kVec;
            if (c < cols) {
                raw_dy[k].load(dyr + c);
                raw_x[k].load(xr + c);
            }
        }
        const float mean = __ldg(a.mean + r), rstd = __ldg(a.rstd + r);
        float s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < kNum; ++k) {
            const int c = (k * threads + tid) * kVec;
            if (c < cols) {
                float x[kVec], dy[kVec], w[kVec], t0 = 0.0f, t1 = 0.0f;
                raw_x[k].get(x);
                raw_dy[k].get(dy);
#pragma unroll
                for (int i = 0; i < kVec; ++i) w[i] = 1.0f;
                if (weight) read_shared_vector<kVec>(weight + c, w);
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    const float xhat = (x[i] - mean) * rstd, d = dy[i] * w[i];
                    t0 += d;
                    t1 = fmaf(d, xhat, t1);
                    dw[k][i] = fmaf(dy[i], xhat, dw[k][i]);
                    db[k][i] += dy[i];
                }
                s[0] += t0;
                s[1] += t1;
            }
        }
        if (a.dx == nullptr) continue;
        row_sum(s, sh, warps, half);
        const float c1 = s[0] * n_inv, c2 = s[1] * n_inv;
        T *dxr = static_cast<T *>(a.dx) + r * a.dx_ld;
#pragma unroll
        for (int k = 0; k < kNum; ++k) {
            const int c = (k * threads + tid) * kVec;
            if (c < cols) {
                float x[kVec], dy[kVec], w[kVec];
                raw_x[k].get(x);
                raw_dy[k].get(dy);
#pragma unroll
                for (int i = 0; i < kVec; ++i) w[i] = 1.0f;
                if (weight) read_shared_vector<kVec>(weight + c, w);
#pragma unroll
                for (int i = 0; i < kVec; ++i) x[i] = rstd * (fmaf(dy[i], w[i], -c1) - (x[i] - mean) * rstd * c2);
                Few<T, kVec>::store(dxr + c, x);
            }
        }
    }
    if (part == nullptr) return;
    float *out_w = part + (int64_t)blockIdx.x * cols, *out_b = out_w + (int64_t)gridDim.x * cols;
    if (warps == 1) {
        for (int turn = 0; turn < kSoloWarps; ++turn) {
            if ((int)(threadIdx.x >> 5) == turn)
#pragma unroll
                for (int k = 0; k < kNum; ++k) {
                    const int c = (k * threads + tid) * kVec;
                    if (c < cols)
#pragma unroll
                        for (int i = 0; i < kVec; ++i) {
                            columns[c + i] = turn ? columns[c + i] + dw[k][i] : dw[k][i];
                            columns[cols + c + i] = turn ? columns[cols + c + i] + db[k][i] : db[k][i];
                        }
                }
            __syncthreads();
        }
        for (int c = threadIdx.x; c < cols; c += kSoloWarps * 32) {
            out_w[c] = columns[c];
            out_b[c] = columns[cols + c];
        }
        return;
    }
#pragma unroll
    for (int k = 0; k < kNum; ++k) {
        const int c = (k * threads + tid) * kVec;
        if (c < cols)
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                out_w[c + i] = dw[k][i];
                out_b[c + i] = db[k][i];
            }
    }
}

// ---- any row length

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

// Adds the slices of a column: 32 columns a CTA, a warp for every sixteenth slice, the warps in order.
constexpr int kFinishWarps = 16;
__global__ void __launch_bounds__(kFinishWarps * 32) layer_norm_dw_finish_kernel(const float *part, int slices, int64_t cols, float *dweight,
                                                                                float *dbias, int accumulate)
{
    __shared__ float sh[kFinishWarps][32];
    cudaGridDependencySynchronize();
    float *out = blockIdx.y == 0 ? dweight : dbias;
    if (out == nullptr) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    const float *p = part + (int64_t)blockIdx.y * slices * cols + c;
    float s = 0.0f;
    if (c < cols)
#pragma unroll 8
        for (int i = warp; i < slices; i += kFinishWarps) s += p[(int64_t)i * cols];
    sh[warp][lane] = s;
    __syncthreads();
    if (warp != 0 || c >= cols) return;
    double t = accumulate ? (double)out[c] : 0.0;
    for (int w = 0; w < kFinishWarps; ++w) t += (double)sh[w][lane];
    out[c] = (float)t;
}

inline unsigned row_grid(int64_t rows) { return (unsigned)(rows < (1 << 20) ? rows : (1 << 20)); }

// How the rows of a matrix are laid over threads: elements a vector, vectors a thread, warps a row; num == 0: not at all.
struct RowShape {
    int vec = 1, num = 0, warps = 0;
    unsigned threads() const { return (unsigned)(warps == 1 ? kSoloWarps : warps) * 32; }
};

RowShape row_shape(int64_t rows, int64_t cols, int vec, int most, int sm_count)
{
    RowShape s;
    s.vec = vec;
    const int64_t vecs = cols / vec;
    // few rows: spread each over as many warps as it can use; many: over as few as hold it
    const bool few = rows < 4 * (int64_t)sm_count;
    for (int num = few ? 1 : most; num <= most && num >= 1; num = few ? num * 2 : num / 2) {
        const int64_t warps = (vecs + 32 * num - 1) / (32 * num);
        if (warps * 32 > (num == 1 ? 1024 : 512)) {
            if (few) continue;
            break;
        }
        s.num = num;
        s.warps = (int)warps;
        if (few || vecs > 16 * num) break;      // (many rows: fewer vectors a thread, where a warp would be half empty)
    }
    return s;
}

// CTAs of a launch: one wave, or less if there are fewer rows.
struct RowLaunch {
    const void *kernel = nullptr;
    RowShape shape;
    size_t shared = 0;
    int64_t grid(int64_t rows, int sm_count) const
    {
        // (asking takes microseconds: the answers are kept)
        struct Known { const void *kernel; unsigned threads; size_t shared; int ctas; };
        static thread_local Known known[32];
        static thread_local int n_known = 0, next = 0;
        int ctas = 0;
        for (int i = 0; i < n_known && ctas == 0; ++i)
            if (known[i].kernel == kernel && known[i].threads == shape.threads() && known[i].shared == shared) ctas = known[i].ctas;
        if (ctas == 0) {
            if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&ctas, kernel, (int)shape.threads(), shared) != cudaSuccess || ctas < 1) {
                cudaGetLastError();
                ctas = 1;
            }
            known[next] = Known{kernel, shape.threads(), shared, ctas};
            next = (next + 1) % 32;
            if (n_known < 32) ++n_known;
        }
        const int64_t each = shape.warps == 1 ? kSoloWarps : 1, want = (rows + each - 1) / each, wave = (int64_t)sm_count * ctas;
        return want < wave ? want : wave;
    }
};

bool on_16_bytes(const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// Does every row of the matrix start on a 16-byte boundary?
bool rows_on_16_bytes(const void *p, int64_t rows, int64_t ld, int dtype)
{
    return on_16_bytes(p) && (rows <= 1 || ld * (dtype == GG_F32 ? 4 : 2) % 16 == 0);
}

int forward_vec(const LayerNormArgs &a)
{
    const int vec = a.dtype == GG_F32 ? 4 : 8;
    const bool ok = a.cols % vec == 0 && rows_on_16_bytes(a.x, a.rows, a.x_ld, a.dtype) && rows_on_16_bytes(a.y, a.rows, a.y_ld, a.dtype) &&
                    on_16_bytes(a.weight) && on_16_bytes(a.bias);
    return ok ? vec : 1;
}

int backward_vec(const LayerNormGradArgs &a)
{
    const int vec = a.dtype == GG_F32 ? 4 : 8;
    const bool ok = a.cols % vec == 0 && rows_on_16_bytes(a.x, a.rows, a.x_ld, a.dtype) && rows_on_16_bytes(a.dy, a.rows, a.dy_ld, a.dtype) &&
                    rows_on_16_bytes(a.dx, a.rows, a.dx_ld, a.dtype) && on_16_bytes(a.weight);
    return ok ? vec : 1;
}

constexpr int kMostVec = 4, kMostOne = 16;      // vectors, single elements that a thread may hold of a row

template <typename T, typename TW, int kVec, int kNum>
const void *forward_kernel(int num)
{
    if (num == kNum) return reinterpret_cast<const void *>(layer_norm_rows_kernel<T, TW, kVec, kNum>);
    if constexpr (kNum > 1) return forward_kernel<T, TW, kVec, kNum / 2>(num);
    return nullptr;
}

template <typename T, typename TW, int kVec, int kNum>
const void *backward_kernel(int num)
{
    if (num == kNum) return reinterpret_cast<const void *>(layer_norm_rows_grad_kernel<T, TW, kVec, kNum>);
    if constexpr (kNum > 1) return backward_kernel<T, TW, kVec, kNum / 2>(num);
    return nullptr;
}

template <typename T, typename TW>
cudaError_t forward(const LayerNormArgs &a, int sm_count, cudaStream_t st)
{
    RowLaunch l;
    const int vec = forward_vec(a);
    l.shape = row_shape(a.rows, a.cols, vec, vec == 1 ? kMostOne : kMostVec, sm_count);
    if (l.shape.num == 0) {
        layer_norm_kernel<T, TW><<<row_grid(a.rows), kThreads, 0, st>>>(a);
        return cudaGetLastError();
    }
    l.kernel = vec == 1 ? forward_kernel<T, TW, 1, kMostOne>(l.shape.num) : forward_kernel<T, TW, 16 / sizeof(T), kMostVec>(l.shape.num);
    void *args[] = {const_cast<LayerNormArgs *>(&a), &l.shape.warps};
    return cudaLaunchKernel(l.kernel, dim3((unsigned)l.grid(a.rows, sm_count)), dim3(l.shape.threads()), args, 0, st);
}

template <typename T, typename TW>
RowLaunch backward_launch(const LayerNormGradArgs &a, int sm_count)
{
    RowLaunch l;
    const int vec = backward_vec(a);
    l.shape = row_shape(a.rows, a.cols, vec, vec == 1 ? kMostOne : kMostVec, sm_count);
    if (a.rows == 0) l.shape.num = 0;
    if (l.shape.num == 0) return l;
    l.kernel = vec == 1 ? backward_kernel<T, TW, 1, kMostOne>(l.shape.num) : backward_kernel<T, TW, 16 / sizeof(T), kMostVec>(l.shape.num);
    if (l.shape.warps == 1 && (a.dweight || a.dbias)) l.shared = sizeof(float) * 2 * (size_t)a.cols;
    return l;
}

RowLaunch backward_launch(const LayerNormGradArgs &a, int sm_count)
{
    if (a.dtype == GG_F32 && a.w_dtype == GG_F32) return backward_launch<float, float>(a, sm_count);
    if (a.dtype == GG_F32) return backward_launch<float, uint16_t>(a, sm_count);
    if (a.w_dtype == GG_F32) return backward_launch<uint16_t, float>(a, sm_count);
    return backward_launch<uint16_t, uint16_t>(a, sm_count);
}

// Any row length: the sums first, since dx may be written over x or dy.
template <typename T, typename TW>
cudaError_t backward_any(const LayerNormGradArgs &a, int slices, float *part, int *launches, cudaStream_t st)
{
    if (part != nullptr) {
        const int64_t strips = (a.cols + 31) / 32;
        layer_norm_dw_kernel<T><<<dim3((unsigned)(strips < (1 << 20) ? strips : (1 << 20)), (unsigned)slices), kThreads, 0, st>>>(a, part, slices);
        *launches += 1;
    }
    if (a.dx != nullptr && a.rows > 0) {
        layer_norm_dx_kernel<T, TW><<<row_grid(a.rows), kThreads, 0, st>>>(a);
        *launches += 1;
    }
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_layer_norm(const LayerNormArgs &a, int sm_count, cudaStream_t st)
{
    if (a.rows <= 0 || a.cols <= 0) return cudaSuccess;
    if (a.dtype == GG_F32 && a.w_dtype == GG_F32) return forward<float, float>(a, sm_count, st);
    if (a.dtype == GG_F32) return forward<float, uint16_t>(a, sm_count, st);
    if (a.w_dtype == GG_F32) return forward<uint16_t, float>(a, sm_count, st);
    return forward<uint16_t, uint16_t>(a, sm_count, st);
}

int layer_norm_grad_slices(const LayerNormGradArgs &a, int sm_count)
{
    const RowLaunch l = backward_launch(a, sm_count);
    if (l.kernel != nullptr) return (int)l.grid(a.rows, sm_count);
    const int64_t strips = (a.cols + 31) / 32, most = (a.rows + 63) / 64;
    int64_t n = (4 * (int64_t)sm_count + strips - 1) / strips;
    n = n < most ? n : most;
    return (int)(n < 1 ? 1 : n);
}

cudaError_t launch_layer_norm_grad(const LayerNormGradArgs &a, float *part, int slices, int sm_count, int *launches, cudaStream_t st)
{
    *launches = 0;
    if (a.cols <= 0) return cudaSuccess;
    const bool sums = a.dweight != nullptr || a.dbias != nullptr;
    if (!sums) part = nullptr;
    const RowLaunch l = backward_launch(a, sm_count);
    cudaError_t e;
    if (l.kernel != nullptr) {
        int warps = l.shape.warps;
        void *args[] = {const_cast<LayerNormGradArgs *>(&a), &part, &warps};
        e = cudaLaunchKernel(l.kernel, dim3((unsigned)slices), dim3(l.shape.threads()), args, l.shared, st);
        *launches += 1;
    } else if (a.dtype == GG_F32 && a.w_dtype == GG_F32) {
        e = backward_any<float, float>(a, slices, part, launches, st);
    } else if (a.dtype == GG_F32) {
        e = backward_any<float, uint16_t>(a, slices, part, launches, st);
    } else if (a.w_dtype == GG_F32) {
        e = backward_any<uint16_t, float>(a, slices, part, launches, st);
    } else {
        e = backward_any<uint16_t, uint16_t>(a, slices, part, launches, st);
    }
    if (e != cudaSuccess || !sums) return e;
    // launched while the kernel before it drains: it waits for that kernel's writes by itself
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)((a.cols + 31) / 32), 2);
    cfg.blockDim = dim3(kFinishWarps * 32);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    *launches += 1;
    return cudaLaunchKernelEx(&cfg, layer_norm_dw_finish_kernel, (const float *)part, slices, a.cols, a.dweight, a.dbias, (int)a.accumulate);
}

}  // namespace gg
