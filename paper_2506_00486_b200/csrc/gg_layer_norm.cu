// Layer norm over the rows of a matrix and its gradient.
//
//     y = w xhat + b,  xhat = (x - mean) rstd,  mean = sum(x) / n,  rstd = 1 / sqrt(sum((x - mean)^2) / n + eps)
//     d = w dy:  dx = rstd (d - sum(d) / n - xhat sum(d xhat) / n),  dw = sum over rows of dy xhat,  db = sum over rows of dy
//
// n is the row length.  The variance is that of the differences from the mean (two passes over the row), so a large
// mean costs it no digits beyond those of the mean itself, which is an fp32 sum.  Both directions are bound by memory: the forward pass has to read x and write y once, the
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

// 1 / sqrt(v): the approximate reciprocal root with one Newton step (v is a normal number wherever the result matters: an
// fp32 variance that is not zero, plus eps; zero gives infinity).
__device__ __forceinline__ float rsqrt_of(float v)
{
    const float y = rsqrtf(v), h = 0.5f * v * y;
    return v > 0.0f && v < INFINITY ? fmaf(y, fmaf(-h, y, 0.5f), y) : y;
}

// Few rows: the sums over the rows need no slices.  The launch of the kernel over rows gets one more CTA for each 32 columns
// (of `strips` in all), which reads these columns of all rows again, from cache: one launch instead of two.
template <typename T>
__device__ __forceinline__ void sum_strip(const LayerNormGradArgs &a, int strip, float *shared)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int64_t c = (int64_t)strip * 32 + lane;
    float dw = 0.0f, db = 0.0f;
    if (c < a.cols)
#pragma unroll 4
        for (int r = warp; r < (int)a.rows; r += warps) {
            const float dy = widen<T>(static_cast<const T *>(a.dy)[r * a.dy_ld + c]), x = widen<T>(static_cast<const T *>(a.x)[r * a.x_ld + c]);
            dw = fmaf(dy, (x - __ldg(a.mean + r)) * __ldg(a.rstd + r), dw);
            db += dy;
        }
    shared[warp * 32 + lane] = dw;
    shared[1024 + warp * 32 + lane] = db;
    __syncthreads();
    float *out = warp == 0 ? a.dweight : a.dbias;
    if (warp >= 2 || out == nullptr || c >= a.cols) return;
    double t = a.accumulate ? (double)out[c] : 0.0;
    for (int w = 0; w < warps; ++w) t += (double)shared[warp * 1024 + w * 32 + lane];
    out[c] = (float)t;
}

// ---- rows of 16-byte vectors that fit the registers of their threads

// A row belongs to T threads: to 2^k lanes of a warp (short rows: a CTA of four warps then holds several, and needs no
// barrier), or to all of its CTA.  Thread i of a row holds the vectors i, i + T, i + 2 T, ..., kNum of them at most.  The
// rows come in by asynchronous copies, kDepth - 1 ahead of the one at work, each thread's vectors into places of shared
// memory that are its own: what is in flight then depends neither on registers nor on how long a row's sums take.
// (Loads into registers, one row at a time, measured 60 against 47 us forward and 133 against 77 us backward on bf16 [16384, 4096].)
constexpr int kSoloWarps = 4;
constexpr int kDepth = 3;
template <int kNum> constexpr int kMostThreads = kNum == 1 ? 1024 : 512;        // 64 or 128 registers a thread

// Sums over the threads of a row, the same bits in every one.  kSolo: `threads` lanes of a warp.  Else all of the CTA, over
// `sh`, which alternates between two halves, so that one barrier a sum is enough: a thread writes a half again only after a
// barrier that follows every read of it.
template <bool kSolo>
__device__ __forceinline__ float row_sum(float v, float (*sh)[32], int threads, int &half)
{
    if (kSolo) {
        for (int o = threads >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
        return v;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    if ((threadIdx.x & 31) == 0) sh[half][threadIdx.x >> 5] = v;
    __syncthreads();
    // (the places beyond the last warp are zero)
    const int quads = (threads + 127) >> 7;
    v = 0.0f;
    for (int q = 0; q < quads; ++q) {
        const float4 t = reinterpret_cast<const float4 *>(sh[half])[q];
        v += (t.x + t.y) + (t.z + t.w);
    }
    half ^= 1;
    return v;
}

// Two sums at once.
template <bool kSolo>
__device__ __forceinline__ float2 row_sum2(float v0, float v1, float2 (*sh)[32], int threads, int &half)
{
    if (kSolo) {
        for (int o = threads >> 1; o > 0; o >>= 1) {
            v0 += __shfl_xor_sync(0xFFFFFFFFu, v0, o);
            v1 += __shfl_xor_sync(0xFFFFFFFFu, v1, o);
        }
        return make_float2(v0, v1);
    }
    // the lower half warp goes on with the first, the upper with the second
    const int lane = threadIdx.x & 31;
    const bool upper = lane & 16;
    float v = (upper ? v1 : v0) + __shfl_xor_sync(0xFFFFFFFFu, upper ? v0 : v1, 16);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    if ((lane & 15) == 0) reinterpret_cast<float *>(&sh[half][threadIdx.x >> 5])[lane >> 4] = v;
    __syncthreads();
    const int twos = (threads + 63) >> 6;
    f32x2 t = 0;
    for (int q = 0; q < twos; ++q) {
        const ulonglong2 p = reinterpret_cast<const ulonglong2 *>(sh[half])[q];
        t = add2(t, add2(p.x, p.y));
    }
    half ^= 1;
    return halves(t);
}

// What is known of a launch.  kRagged: nothing.  kFull: every thread has all of its vectors (the widths of models mostly do),
// and nothing is asked.  kKept: besides, weight and bias are there, in the type of x, and a thread keeps its columns of them
// in registers (read from L1 for each row they cost 51 against 47 us on bf16 [16384, 4096]).
enum Known { kRagged, kFull, kKept };

// The rows of a thread and its vectors of them: kOperands rows for each of kDepth stages of the ring.
template <typename T, int kNum, int kOperands, bool kWhole, bool kSolo>
struct Rows {
    static constexpr int kVec = 16 / sizeof(T);
    int threads, tid, cols;
    int64_t first, stride;             // rows of this thread
    uint32_t base, step, stage_bytes;  // in shared memory: this thread's first place, from one vector to the next, a stage
    __device__ __forceinline__ Rows(int t, int c, unsigned ctas, unsigned char *shared) : threads(t), cols(c)
    {
        if (kSolo) {
            const int each = 32 / t;                                           // rows of a warp
            tid = threadIdx.x & (t - 1);
            first = ((int64_t)blockIdx.x * kSoloWarps + (threadIdx.x >> 5)) * each + (threadIdx.x & 31) / t;
            stride = (int64_t)ctas * kSoloWarps * each;
        } else {
            tid = threadIdx.x;
            first = blockIdx.x;
            stride = ctas;
        }
        step = blockDim.x * 16u;
        stage_bytes = kOperands * kNum * step;
        base = (uint32_t)__cvta_generic_to_shared(shared) + threadIdx.x * 16u;
    }
    __device__ __forceinline__ bool has(int k) const { return kWhole || (k * threads + tid) * kVec < cols; }
    __device__ __forceinline__ int column(int k) const { return (k * threads + tid) * kVec; }
    // row: where this thread's first vector of it is, in the matrix at `base`
    __device__ __forceinline__ void fetch(uint32_t slot, int operand, const T *row, const void *base, int64_t n_rows, int64_t ld) const
    {
#pragma unroll
        for (int k = 0; k < kNum; ++k)
            if (has(k) && GG_IN_MATRIX(row + k * threads * kVec, kVec, base, n_rows, cols, ld)) copy16(slot + (operand * kNum + k) * step, row + k * threads * kVec);
    }
    __device__ __forceinline__ void read(uint32_t slot, int operand, Few<T> (&v)[kNum]) const
    {
#pragma unroll
        for (int k = 0; k < kNum; ++k)
            if (has(k)) v[k].read(slot + (operand * kNum + k) * step);
    }
    __device__ __forceinline__ uint32_t after(uint32_t slot) const { return slot == base + (kDepth - 1) * stage_bytes ? base : slot + stage_bytes; }
    __device__ __forceinline__ uint32_t before(uint32_t slot) const { return slot == base ? base + (kDepth - 1) * stage_bytes : slot - stage_bytes; }
    // whether there is another round of rows: the lanes of a warp stay together, since they form their sums together
    __device__ __forceinline__ bool more(int64_t r, int64_t rows) const { return kSolo ? __any_sync(0xFFFFFFFFu, r < rows) : r < rows; }
};

template <typename T, typename TW, int kNum, Known kKnown, bool kSolo>
__global__ void __launch_bounds__(kMostThreads<kNum>) layer_norm_rows_kernel(const __grid_constant__ LayerNormArgs a, int threads)
{
    constexpr int kPairs = Few<T>::kPairs;
    __shared__ __align__(16) float sh[2][32];
    extern __shared__ __align__(16) unsigned char shared[];
    const Rows<T, kNum, 1, kKnown != kRagged, kSolo> rows(threads, (int)a.cols, gridDim.x, shared);
    const float n_inv = 1.0f / (float)rows.cols, eps = (float)a.eps;
    const TW *weight = static_cast<const TW *>(a.weight), *bias = static_cast<const TW *>(a.bias);
    const T *x_ahead = static_cast<const T *>(a.x) + rows.first * a.x_ld + rows.column(0);
    T *y = static_cast<T *>(a.y) + rows.first * a.y_ld + rows.column(0);
    const int64_t x_step = rows.stride * a.x_ld, y_step = rows.stride * a.y_ld;
    Few<TW> kept_w[kNum], kept_b[kNum];
    if constexpr (kKnown == kKept)
#pragma unroll
        for (int k = 0; k < kNum; ++k) {
            if (!GG_IN_BOUNDS(rows.column(k) + rows.kVec - 1, a.cols)) continue;
            kept_w[k].read(weight + rows.column(k));
            kept_b[k].read(bias + rows.column(k));
        }
    int half = 0;
    uint32_t slot = rows.base;
    if (!kSolo) {
        if (threadIdx.x < 64) sh[threadIdx.x >> 5][threadIdx.x & 31] = 0.0f;
        __syncthreads();
    }
    int64_t r_ahead = rows.first;
    for (int d = 0; d < kDepth - 1; ++d) {
        if (r_ahead < a.rows) rows.fetch(rows.base + d * rows.stage_bytes, 0, x_ahead, a.x, a.rows, a.x_ld);
        copies_commit();
        x_ahead += x_step;
        r_ahead += rows.stride;
    }
    for (int64_t r = rows.first; rows.more(r, a.rows); r += rows.stride) {
        if (r_ahead < a.rows) rows.fetch(rows.before(slot), 0, x_ahead, a.x, a.rows, a.x_ld);
        copies_commit();
        x_ahead += x_step;
        r_ahead += rows.stride;
        copies_wait<kDepth - 1>();
        const bool live = !kSolo || r < a.rows;
        f32x2 x[kNum][kPairs], t = 0;
        if (live) {
            Few<T> raw[kNum];
            rows.read(slot, 0, raw);
#pragma unroll
            for (int k = 0; k < kNum; ++k)
                if (rows.has(k))
#pragma unroll
                    for (int i = 0; i < kPairs; ++i) {
                        x[k][i] = raw[k].get(i);
                        t = add2(t, x[k][i]);
                    }
        }
        slot = rows.after(slot);
        float2 f = halves(t);
        const float mean = row_sum<kSolo>(f.x + f.y, sh, threads, half) * n_inv;
        t = 0;
        if (live) {
            const f32x2 minus = both(-mean);
#pragma unroll
            for (int k = 0; k < kNum; ++k)
                if (rows.has(k))
#pragma unroll
                    for (int i = 0; i < kPairs; ++i) {
                        x[k][i] = add2(x[k][i], minus);
                        t = fma2(x[k][i], x[k][i], t);
                    }
        }
        f = halves(t);
        const float rstd = rsqrt_of(fmaf(row_sum<kSolo>(f.x + f.y, sh, threads, half), n_inv, eps));
        if (live) {
            const f32x2 by = both(rstd);
#pragma unroll
            for (int k = 0; k < kNum; ++k)
                if (rows.has(k)) {
                    const int c = rows.column(k);
#pragma unroll
                    for (int i = 0; i < kPairs; ++i) x[k][i] = mul2(x[k][i], by);
                    if constexpr (kKnown == kKept) {
#pragma unroll
                        for (int i = 0; i < kPairs; ++i) x[k][i] = fma2(x[k][i], kept_w[k].get(i), kept_b[k].get(i));
                    } else if (weight && bias && GG_IN_BOUNDS(c + rows.kVec - 1, a.cols)) {
                        f32x2 w[kPairs], b[kPairs];
                        read_vector(weight + c, w);
                        read_vector(bias + c, b);
#pragma unroll
                        for (int i = 0; i < kPairs; ++i) x[k][i] = fma2(x[k][i], w[i], b[i]);
                    } else if (weight || bias) {
                        f32x2 o[kPairs];
                        read_vector((weight ? weight : bias) + c, o);
#pragma unroll
                        for (int i = 0; i < kPairs; ++i) x[k][i] = weight ? mul2(x[k][i], o[i]) : add2(x[k][i], o[i]);
                    }
                    if (GG_IN_MATRIX(y + k * threads * rows.kVec, rows.kVec, a.y, a.rows, a.cols, a.y_ld)) Few<T>::store(y + k * threads * rows.kVec, x[k]);
                }
            if (rows.tid == 0 && GG_IN_BOUNDS(r, a.rows)) {
                if (a.mean) a.mean[r] = mean;
                if (a.rstd) a.rstd[r] = rstd;
            }
        }
        y += y_step;
    }
    copies_wait<0>();
}

// The gradient: each thread keeps the sums of its columns over the rows of its CTA and leaves them as slice blockIdx.x of
// `part` ([2][gridDim.x][cols]); layer_norm_dw_finish_kernel adds the slices.
template <typename T, typename TW, int kNum, Known kKnown, bool kSolo>
__global__ void __launch_bounds__(kMostThreads<kNum>) layer_norm_rows_grad_kernel(const __grid_constant__ LayerNormGradArgs a, float *part, int strips, int threads)
{
    constexpr int kPairs = Few<T>::kPairs;
    __shared__ __align__(16) float2 sh[2][32];
    extern __shared__ __align__(16) unsigned char shared[];
    const unsigned row_ctas = gridDim.x - (unsigned)strips;
    if (blockIdx.x >= row_ctas) {
        sum_strip<T>(a, (int)(blockIdx.x - row_ctas), reinterpret_cast<float *>(shared));
        return;
    }
    const Rows<T, kNum, 2, kKnown != kRagged, kSolo> rows(threads, (int)a.cols, row_ctas, shared);
    cudaTriggerProgrammaticLaunchCompletion();       // (the kernel that adds the slices may take its places as these CTAs leave them)
    const float n_inv = 1.0f / (float)rows.cols;
    const TW *weight = static_cast<const TW *>(a.weight);
    const T *x_ahead = static_cast<const T *>(a.x) + rows.first * a.x_ld + rows.column(0);
    const T *dy_ahead = static_cast<const T *>(a.dy) + rows.first * a.dy_ld + rows.column(0);
    T *dx = static_cast<T *>(a.dx) + rows.first * a.dx_ld + rows.column(0);
    const int64_t x_step = rows.stride * a.x_ld, dy_step = rows.stride * a.dy_ld, dx_step = rows.stride * a.dx_ld;
    f32x2 dw[kNum][kPairs], db[kNum][kPairs];
#pragma unroll
    for (int k = 0; k < kNum; ++k)
#pragma unroll
        for (int i = 0; i < kPairs; ++i) dw[k][i] = db[k][i] = 0;
    int half = 0;
    uint32_t slot = rows.base;
    if (!kSolo) {
        if (threadIdx.x < 64) sh[threadIdx.x >> 5][threadIdx.x & 31] = make_float2(0.0f, 0.0f);
        __syncthreads();
    }
    int64_t r_ahead = rows.first;
    for (int d = 0; d < kDepth - 1; ++d) {
        if (r_ahead < a.rows) {
            rows.fetch(rows.base + d * rows.stage_bytes, 0, dy_ahead, a.dy, a.rows, a.dy_ld);
            rows.fetch(rows.base + d * rows.stage_bytes, 1, x_ahead, a.x, a.rows, a.x_ld);
        }
        copies_commit();
        x_ahead += x_step;
        dy_ahead += dy_step;
        r_ahead += rows.stride;
    }
    const float *mean_at = a.mean + rows.first, *rstd_at = a.rstd + rows.first;
    float mean = 0.0f, rstd = 0.0f;
    if (rows.first < a.rows) {
        mean = __ldg(mean_at);
        rstd = __ldg(rstd_at);
    }
    for (int64_t r = rows.first; rows.more(r, a.rows); r += rows.stride) {
        if (r_ahead < a.rows) {
            const uint32_t to = rows.before(slot);
            rows.fetch(to, 0, dy_ahead, a.dy, a.rows, a.dy_ld);
            rows.fetch(to, 1, x_ahead, a.x, a.rows, a.x_ld);
        }
        copies_commit();
        x_ahead += x_step;
        dy_ahead += dy_step;
        r_ahead += rows.stride;
        const f32x2 minus = both(-mean), by = both(rstd);
        const float scale = -rstd * n_inv;
        mean_at += rows.stride;
        rstd_at += rows.stride;
        if (r + rows.stride < a.rows) {
            mean = __ldg(mean_at);
            rstd = __ldg(rstd_at);
        }
        copies_wait<kDepth - 1>();
        const bool live = !kSolo || r < a.rows;
        // kAgain: 32 elements of a thread in fp32 twice, beside the sums of their columns, do not fit the registers: the second
        // pass reads and computes them again
        constexpr bool kAgain = kNum * kPairs > 8;
        f32x2 xhat[kNum][kPairs], d[kNum][kPairs], t0 = 0, t1 = 0;
        const uint32_t now = slot;
        auto load = [&](int k, f32x2 (&xh)[kPairs], f32x2 (&g)[kPairs]) {
            Few<T> raw_dy, raw_x;
            raw_dy.read(now + k * rows.step);
            raw_x.read(now + (kNum + k) * rows.step);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) {
                xh[i] = mul2(add2(raw_x.get(i), minus), by);
                g[i] = raw_dy.get(i);
            }
        };
        auto weigh = [&](int k, f32x2 (&g)[kPairs]) {
            if (weight && GG_IN_BOUNDS(rows.column(k) + rows.kVec - 1, a.cols)) {
                f32x2 w[kPairs];
                read_vector(weight + rows.column(k), w);
#pragma unroll
                for (int i = 0; i < kPairs; ++i) g[i] = mul2(g[i], w[i]);
            }
        };
        if (live)
#pragma unroll
            for (int k = 0; k < kNum; ++k)
                if (rows.has(k)) {
                    load(k, xhat[k], d[k]);
#pragma unroll
                    for (int i = 0; i < kPairs; ++i) {
                        dw[k][i] = fma2(d[k][i], xhat[k][i], dw[k][i]);
                        db[k][i] = add2(db[k][i], d[k][i]);
                    }
                    weigh(k, d[k]);
#pragma unroll
                    for (int i = 0; i < kPairs; ++i) {
                        t0 = add2(t0, d[k][i]);
                        t1 = fma2(d[k][i], xhat[k][i], t1);
                    }
                }
        slot = rows.after(slot);
        if (a.dx == nullptr) continue;
        const float2 f0 = halves(t0), f1 = halves(t1);
        const float2 c = row_sum2<kSolo>(f0.x + f0.y, f1.x + f1.y, sh, threads, half);
        if (live) {
            // rstd (d - c1 - xhat c2)
            const f32x2 c1 = both(c.x * scale), c2 = both(c.y * scale);
#pragma unroll
            for (int k = 0; k < kNum; ++k)
                if (rows.has(k)) {
                    if (kAgain) {
                        load(k, xhat[k], d[k]);
                        weigh(k, d[k]);
                    }
#pragma unroll
                    for (int i = 0; i < kPairs; ++i) d[k][i] = fma2(xhat[k][i], c2, fma2(d[k][i], by, c1));
                    if (GG_IN_MATRIX(dx + k * threads * rows.kVec, rows.kVec, a.dx, a.rows, a.cols, a.dx_ld)) Few<T>::store(dx + k * threads * rows.kVec, d[k]);
                }
        }
        dx += dx_step;
    }
    copies_wait<0>();
    if (part == nullptr) return;
    const int cols = rows.cols;
    float *out_w = part + (int64_t)blockIdx.x * cols, *out_b = out_w + (int64_t)gridDim.x * cols;
    if (kSolo) {
        // the rows of a warp, then the warps of the CTA in order, in shared memory (whose rows are done with): [2][cols]
        float *columns = reinterpret_cast<float *>(shared);
#pragma unroll
        for (int k = 0; k < kNum; ++k)
#pragma unroll
            for (int i = 0; i < kPairs; ++i)
                for (int o = threads; o < 32; o <<= 1) {
                    dw[k][i] = add2(dw[k][i], __shfl_xor_sync(0xFFFFFFFFu, dw[k][i], o));
                    db[k][i] = add2(db[k][i], __shfl_xor_sync(0xFFFFFFFFu, db[k][i], o));
                }
        __syncthreads();
        for (int turn = 0; turn < kSoloWarps; ++turn) {
            if ((int)(threadIdx.x >> 5) == turn && (threadIdx.x & 31) < threads)
#pragma unroll
                for (int k = 0; k < kNum; ++k)
                    if (rows.has(k))
#pragma unroll
                        for (int i = 0; i < kPairs; ++i) {
                            f32x2 *w = reinterpret_cast<f32x2 *>(columns + rows.column(k)) + i, *b = reinterpret_cast<f32x2 *>(columns + cols + rows.column(k)) + i;
                            *w = turn ? add2(*w, dw[k][i]) : dw[k][i];
                            *b = turn ? add2(*b, db[k][i]) : db[k][i];
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
    for (int k = 0; k < kNum; ++k)
        if (rows.has(k))
#pragma unroll
            for (int i = 0; i < kPairs; i += 2) {
                const f32x2 w[2] = {dw[k][i], dw[k][i + 1]}, b[2] = {db[k][i], db[k][i + 1]};
                if (!GG_IN_BOUNDS(blockIdx.x, row_ctas) || !GG_IN_BOUNDS(rows.column(k) + 2 * i + 3, cols)) continue;
                Few<float>::store(out_w + rows.column(k) + 2 * i, w);
                Few<float>::store(out_b + rows.column(k) + 2 * i, b);
            }
}

// ---- rows that are not made of 16-byte vectors, or do not start on their boundaries

// Room for the pieces of a row of n elements, wherever it starts.
template <typename T>
__host__ __device__ constexpr uint32_t piece_bytes(int n) { return ((uint32_t)n * (uint32_t)sizeof(T) + 15u + 15u) / 16u * 16u; }

// Room for `each` fp32 values a column.
__host__ __device__ constexpr uint32_t affine_bytes(int n, int each) { return ((uint32_t)n * (uint32_t)each * 4u + 15u) / 16u * 16u; }

template <int N>
struct Index {
    static constexpr int value = N;
    __device__ __forceinline__ constexpr operator int() const { return N; }
};

// The same plan with single elements.  Each warp computes 32 kNum consecutive elements, lane l those at l, l + 32, ...: all
// offsets within a row are then constants (with a stride of the row's threads they were most of 82 instructions an element,
// 260 against 103 us on bf16 [16384, 4095]).  The rows come in as the aligned 16-byte pieces that cover them.  A piece may
// hold elements of the rows beside, or of what lies between two rows; one that reaches out of the matrix at its very start
// or end is loaded element by element.  A row is fetched while the one before it is at work.
template <typename T, int kNum, int kOperands, bool kSolo>
struct Pieces {
    int threads, tid, cols;
    int column, left, whole;           // this thread's first element, how many the row has from there on, how many every lane has
    int64_t first, stride;
    uint32_t base, row_bytes, stage_bytes;
    // shared: the rows, behind `ahead` bytes of something else
    __device__ __forceinline__ Pieces(int t, int c, unsigned ctas, unsigned char *shared, uint32_t ahead) : threads(t), cols(c)
    {
        row_bytes = piece_bytes<T>(c);
        stage_bytes = kOperands * row_bytes;
        base = (uint32_t)__cvta_generic_to_shared(shared) + ahead;
        if (kSolo) {
            tid = threadIdx.x & 31;
            first = (int64_t)blockIdx.x * kSoloWarps + (threadIdx.x >> 5);
            stride = (int64_t)ctas * kSoloWarps;
            base += (threadIdx.x >> 5) * 2 * stage_bytes;
        } else {
            tid = threadIdx.x;
            first = blockIdx.x;
            stride = ctas;
        }
        column = (kSolo ? 0 : (int)(threadIdx.x >> 5) * 32 * kNum) + (int)(threadIdx.x & 31);
        left = c - column;
        whole = (c - column + (int)(threadIdx.x & 31)) / 32;
    }
    __device__ __forceinline__ void sync() const
    {
        if (kSolo) __syncwarp();
        else __syncthreads();
    }
    // [from, to): the matrix
    __device__ __forceinline__ void fetch(uint32_t slot, const T *row, uintptr_t from, uintptr_t to) const
    {
        const uintptr_t begin = reinterpret_cast<uintptr_t>(row), end = begin + (uint32_t)cols * (uint32_t)sizeof(T), origin = begin & ~(uintptr_t)15;
        const char *p = reinterpret_cast<const char *>(origin) + 16 * tid;
        const int pieces = (int)((uint32_t)(end - origin + 15u) / 16u);
        slot += 16u * tid;
        if (origin >= from && origin + 16u * (uint32_t)pieces <= to) {
            for (int i = tid; i < pieces; i += threads, p += 16 * threads, slot += 16u * threads)
                if (GG_IN_BOUNDS(reinterpret_cast<uintptr_t>(p) - from, to - from - 15)) copy16(slot, p);
            return;
        }
        for (int i = tid; i < pieces; i += threads, p += 16 * threads, slot += 16u * threads) {
            const uintptr_t at = reinterpret_cast<uintptr_t>(p);
            if (at >= from && at + 16 <= to) {
                copy16(slot, p);
            } else {
                for (uintptr_t q = at > begin ? at : begin; q < at + 16 && q < end; q += sizeof(T))
                    put(slot + (uint32_t)(q - at), *reinterpret_cast<const T *>(q));
            }
        }
    }
    static __device__ __forceinline__ void put(uint32_t at, float v) { asm volatile("st.shared.f32 [%0], %1;" ::"r"(at), "f"(v) : "memory"); }
    static __device__ __forceinline__ void put(uint32_t at, uint16_t v) { asm volatile("st.shared.u16 [%0], %1;" ::"r"(at), "h"(v) : "memory"); }
    // where this thread's first element is, for a row at this address
    __device__ __forceinline__ uint32_t place(uint32_t slot, const T *row) const
    {
        return slot + (uint32_t)(reinterpret_cast<uintptr_t>(row) & 15u) + (uint32_t)column * (uint32_t)sizeof(T);
    }
    template <int k>
    static __device__ __forceinline__ float get(uint32_t at)
    {
        if constexpr (sizeof(T) == 4) {
            float v;
            asm volatile("ld.shared.f32 %0, [%1 + %2];" : "=f"(v) : "r"(at), "n"(k * 32 * 4));
            return v;
        } else {
            uint16_t h;
            asm volatile("ld.shared.u16 %0, [%1 + %2];" : "=h"(h) : "r"(at), "n"(k * 32 * 2));
            return widen<uint16_t>(h);
        }
    }
    // The elements 2 j and 2 j + 1 of this thread, as many of them as the row has (all: two).
    template <int j>
    static __device__ __forceinline__ f32x2 get2(uint32_t at, int n)
    {
        const float lo = n > 0 ? get<2 * j>(at) : 0.0f, hi = n > 1 ? get<2 * j + 1>(at) : 0.0f;
        return pair(lo, hi);
    }
    // f(j, n) for the pairs of elements 32 (2 j), 32 (2 j + 1) of this thread (the number as a type, so that it can be an
    // offset), n of which the row has: two pairs at a time without a question, as long as all lanes have them.
    template <int j = 0, typename F>
    __device__ __forceinline__ void each(F f) const
    {
        if constexpr (2 * j < kNum) {
            if (2 * j + 4 <= whole) {
                f(Index<j>(), Index<2>());
                f(Index<j + 1>(), Index<2>());
            } else {
                f(Index<j>(), count(2 * j));
                f(Index<j + 1>(), count(2 * j + 2));
                if (whole < 2 * j) return;
            }
            each<j + 2>(f);
        }
    }
    __device__ __forceinline__ int count(int k) const { return 32 * k >= left ? 0 : 32 * (k + 1) >= left ? 1 : 2; }
};

// v where there is an element, else 0
__device__ __forceinline__ f32x2 only(f32x2 v, int n)
{
    const float2 f = halves(v);
    return pair(n > 0 ? f.x : 0.0f, n > 1 ? f.y : 0.0f);
}

// kStaged: weight and bias (1 and 0 where there is none) wait in shared memory as fp32, which saves the loads from L1 and their
// conversions (bf16 [16384, 4095]: 89 against 103 us), but takes a while to fill and room from other CTAs (fp32 [3000, 5001]:
// 45 against 37 us; bf16 [1000, 2001]: 12.4 against 8.4).
template <typename T, typename TW, int kNum, bool kSolo, bool kStaged>
__global__ void __launch_bounds__(kSolo ? kSoloWarps * 32 : 512, kSolo ? 6 : 1) layer_norm_pieces_kernel(const __grid_constant__ LayerNormArgs a, int threads)
{
    __shared__ __align__(16) float sh[2][32];
    extern __shared__ __align__(16) unsigned char shared[];
    const Pieces<T, kNum, 1, kSolo> rows(threads, (int)a.cols, gridDim.x, shared, kStaged ? affine_bytes((int)a.cols, 2) : 0u);
    const float n_inv = 1.0f / (float)rows.cols, eps = (float)a.eps;
    const T *x = static_cast<const T *>(a.x) + rows.first * a.x_ld;
    T *y = static_cast<T *>(a.y) + rows.first * a.y_ld + rows.column;
    const uintptr_t from = reinterpret_cast<uintptr_t>(a.x), to = reinterpret_cast<uintptr_t>(static_cast<const T *>(a.x) + (a.rows - 1) * a.x_ld + a.cols);
    const int64_t x_step = rows.stride * a.x_ld, y_step = rows.stride * a.y_ld;
    int half = 0;
    uint32_t slot = rows.base, other = rows.base + rows.stage_bytes;
    if (rows.first < a.rows) rows.fetch(slot, x, from, to);
    copies_commit();
    const TW *weight = static_cast<const TW *>(a.weight), *bias = static_cast<const TW *>(a.bias);
    auto from_l1 = [&](int c) { return make_float2(weight ? widen<TW>(__ldg(weight + c)) : 1.0f, bias ? widen<TW>(__ldg(bias + c)) : 0.0f); };
    float2 *affine = reinterpret_cast<float2 *>(shared);
    if (kStaged) {
        for (int c = threadIdx.x; c < rows.cols; c += blockDim.x) affine[c] = from_l1(c);
        affine += rows.column;
    } else {
        if (weight) weight += rows.column;
        if (bias) bias += rows.column;
    }
    if (!kSolo && threadIdx.x < 64) sh[threadIdx.x >> 5][threadIdx.x & 31] = 0.0f;
    __syncthreads();
    for (int64_t r = rows.first; r < a.rows; r += rows.stride) {
        copies_wait<0>();
        rows.sync();       // everyone's pieces of this row are here, and everyone is done with the row before
        if (r + rows.stride < a.rows) rows.fetch(other, x + x_step, from, to);
        copies_commit();
        const uint32_t at = rows.place(slot, x);
        f32x2 v[kNum / 2], t = 0;
        rows.each([&](auto j, auto n) {
            v[j] = rows.template get2<decltype(j)::value>(at, n);
            t = add2(t, v[j]);
        });
        float2 f = halves(t);
        const float mean = row_sum<kSolo>(f.x + f.y, sh, threads, half) * n_inv;
        const f32x2 minus = both(-mean);
        t = 0;
        rows.each([&](auto j, auto n) {
            v[j] = only(add2(v[j], minus), n);
            t = fma2(v[j], v[j], t);
        });
        f = halves(t);
        const float rstd = rsqrt_of(fmaf(row_sum<kSolo>(f.x + f.y, sh, threads, half), n_inv, eps));
        const f32x2 by = both(rstd);
        rows.each([&](auto j, auto n) {
            const float2 o = halves(mul2(v[j], by));
            if (n > 0) {
                const float2 w = kStaged ? affine[64 * j] : from_l1(64 * j);
                if (GG_IN_MATRIX(y + 64 * j, 1, a.y, a.rows, a.cols, a.y_ld)) y[64 * j] = narrow<T>(fmaf(o.x, w.x, w.y));
            }
            if (n > 1) {
                const float2 w = kStaged ? affine[64 * j + 32] : from_l1(64 * j + 32);
                if (GG_IN_MATRIX(y + 64 * j + 32, 1, a.y, a.rows, a.cols, a.y_ld)) y[64 * j + 32] = narrow<T>(fmaf(o.y, w.x, w.y));
            }
        });
        if (rows.tid == 0 && GG_IN_BOUNDS(r, a.rows)) {
            if (a.mean) a.mean[r] = mean;
            if (a.rstd) a.rstd[r] = rstd;
        }
        x += x_step;
        y += y_step;
        const uint32_t swap = slot;
        slot = other;
        other = swap;
    }
}

template <typename T, typename TW, int kNum, bool kSolo>
__global__ void __launch_bounds__(kSolo ? kSoloWarps * 32 : 512, kSolo ? 4 : 1) layer_norm_pieces_grad_kernel(const __grid_constant__ LayerNormGradArgs a, float *part, int strips, int threads)
{
    __shared__ __align__(16) float2 sh[2][32];
    extern __shared__ __align__(16) unsigned char shared[];
    const unsigned row_ctas = gridDim.x - (unsigned)strips;
    if (blockIdx.x >= row_ctas) {
        sum_strip<T>(a, (int)(blockIdx.x - row_ctas), reinterpret_cast<float *>(shared));
        return;
    }
    const Pieces<T, kNum, 2, kSolo> rows(threads, (int)a.cols, row_ctas, shared, affine_bytes((int)a.cols, 1));
    cudaTriggerProgrammaticLaunchCompletion();
    const float n_inv = 1.0f / (float)rows.cols;
    const T *x = static_cast<const T *>(a.x) + rows.first * a.x_ld, *dy = static_cast<const T *>(a.dy) + rows.first * a.dy_ld;
    T *dx = static_cast<T *>(a.dx) + rows.first * a.dx_ld + rows.column;
    const uintptr_t x_from = reinterpret_cast<uintptr_t>(a.x), x_to = reinterpret_cast<uintptr_t>(static_cast<const T *>(a.x) + (a.rows - 1) * a.x_ld + a.cols);
    const uintptr_t dy_from = reinterpret_cast<uintptr_t>(a.dy), dy_to = reinterpret_cast<uintptr_t>(static_cast<const T *>(a.dy) + (a.rows - 1) * a.dy_ld + a.cols);
    const int64_t x_step = rows.stride * a.x_ld, dy_step = rows.stride * a.dy_ld, dx_step = rows.stride * a.dx_ld;
    f32x2 dw[kNum / 2], db[kNum / 2];
#pragma unroll
    for (int j = 0; j < kNum / 2; ++j) dw[j] = db[j] = 0;
    int half = 0;
    uint32_t slot = rows.base, other = rows.base + rows.stage_bytes;
    float next_mean = 0.0f, next_rstd = 0.0f;
    if (rows.first < a.rows) {
        rows.fetch(slot, dy, dy_from, dy_to);
        rows.fetch(slot + rows.row_bytes, x, x_from, x_to);
        next_mean = __ldg(a.mean + rows.first);
        next_rstd = __ldg(a.rstd + rows.first);
    }
    copies_commit();
    float *weight = reinterpret_cast<float *>(shared);
    for (int c = threadIdx.x; c < rows.cols; c += blockDim.x) weight[c] = a.weight ? widen<TW>(__ldg(static_cast<const TW *>(a.weight) + c)) : 1.0f;
    weight += rows.column;
    if (!kSolo && threadIdx.x < 64) sh[threadIdx.x >> 5][threadIdx.x & 31] = make_float2(0.0f, 0.0f);
    __syncthreads();
    for (int64_t r = rows.first; r < a.rows; r += rows.stride) {
        copies_wait<0>();
        rows.sync();       // everyone's pieces of this row are here, and everyone is done with the row before
        const f32x2 minus = both(-next_mean), by = both(next_rstd);
        const float scale = -next_rstd * n_inv;
        if (r + rows.stride < a.rows) {
            rows.fetch(other, dy + dy_step, dy_from, dy_to);
            rows.fetch(other + rows.row_bytes, x + x_step, x_from, x_to);
            next_mean = __ldg(a.mean + r + rows.stride);
            next_rstd = __ldg(a.rstd + r + rows.stride);
        }
        copies_commit();
        const uint32_t dy_at = rows.place(slot, dy), x_at = rows.place(slot + rows.row_bytes, x);
        auto load = [&](auto j, auto n, f32x2 &g, f32x2 &xhat) {       // (an element that is not there counts nothing: its dy is 0)
            g = rows.template get2<decltype(j)::value>(dy_at, n);
            xhat = mul2(add2(rows.template get2<decltype(j)::value>(x_at, n), minus), by);
        };
        auto weigh = [&](auto j, auto n, f32x2 g) { return mul2(g, pair(n > 0 ? weight[64 * j] : 0.0f, n > 1 ? weight[64 * j + 32] : 0.0f)); };
        f32x2 t0 = 0, t1 = 0;
        rows.each([&](auto j, auto n) {
            f32x2 g, xhat;
            load(j, n, g, xhat);
            dw[j] = fma2(g, xhat, dw[j]);
            db[j] = add2(db[j], g);
            const f32x2 d = weigh(j, n, g);
            t0 = add2(t0, d);
            t1 = fma2(d, xhat, t1);
        });
        if (a.dx != nullptr) {
            const float2 f0 = halves(t0), f1 = halves(t1);
            const float2 s = row_sum2<kSolo>(f0.x + f0.y, f1.x + f1.y, sh, threads, half);
            const f32x2 c1 = both(s.x * scale), c2 = both(s.y * scale);
            rows.each([&](auto j, auto n) {       // rstd (d - c1 - xhat c2)
                f32x2 g, xhat;
                load(j, n, g, xhat);
                const float2 o = halves(fma2(xhat, c2, fma2(weigh(j, n, g), by, c1)));
                if (n > 0 && GG_IN_MATRIX(dx + 64 * j, 1, a.dx, a.rows, a.cols, a.dx_ld)) dx[64 * j] = narrow<T>(o.x);
                if (n > 1 && GG_IN_MATRIX(dx + 64 * j + 32, 1, a.dx, a.rows, a.cols, a.dx_ld)) dx[64 * j + 32] = narrow<T>(o.y);
            });
        }
        x += x_step;
        dy += dy_step;
        dx += dx_step;
        const uint32_t swap = slot;
        slot = other;
        other = swap;
    }
    if (part == nullptr) return;
    const int cols = rows.cols;
    float *out_w = part + (int64_t)blockIdx.x * cols, *out_b = out_w + (int64_t)gridDim.x * cols;
    auto add = [&](float *at, f32x2 v, auto n, bool onto) {
        const float2 f = halves(v);
        if (n > 0) at[0] = onto ? at[0] + f.x : f.x;
        if (n > 1) at[32] = onto ? at[32] + f.y : f.y;
    };
    if (kSolo) {       // the warps of the CTA in order, where their rows were
        float *columns = reinterpret_cast<float *>(shared);
        __syncthreads();
        for (int turn = 0; turn < kSoloWarps; ++turn) {
            if ((int)(threadIdx.x >> 5) == turn)
                rows.each([&](auto j, auto n) {
                    add(columns + rows.column + 64 * j, dw[j], n, turn > 0);
                    add(columns + cols + rows.column + 64 * j, db[j], n, turn > 0);
                });
            __syncthreads();
        }
        for (int c = threadIdx.x; c < cols; c += kSoloWarps * 32) {
            out_w[c] = columns[c];
            out_b[c] = columns[cols + c];
        }
        return;
    }
    rows.each([&](auto j, auto n) {
        if (n > 0 && (!GG_IN_BOUNDS(blockIdx.x, row_ctas) || !GG_IN_BOUNDS(rows.column + 64 * j + (n > 1 ? 32 : 0), cols))) return;
        add(out_w + rows.column + 64 * j, dw[j], n, false);
        add(out_b + rows.column + 64 * j, db[j], n, false);
    });
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

// Adds the slices of a column: 32 columns a CTA, a warp for every 32nd slice, the warps in order.
constexpr int kFinishWarps = 32;
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
#pragma unroll 16
        for (int i = warp; i < slices; i += kFinishWarps) s += p[(int64_t)i * cols];
    sh[warp][lane] = s;
    __syncthreads();
    if (warp != 0 || c >= cols) return;
    double t = accumulate ? (double)out[c] : 0.0;
    for (int w = 0; w < kFinishWarps; ++w) t += (double)sh[w][lane];
    out[c] = (float)t;
}

inline unsigned row_grid(int64_t rows) { return (unsigned)(rows < (1 << 20) ? rows : (1 << 20)); }

// How the rows of a matrix are laid over threads: vectors a thread, threads a row; num == 0: not at all.
struct RowShape {
    int num = 0, threads = 0;
    bool pieces = false;
    unsigned block() const { return (unsigned)(threads <= 32 ? kSoloWarps * 32 : threads); }
    int64_t rows_a_cta() const { return threads <= 32 ? kSoloWarps * (32 / threads) : 1; }
};

// Few rows are spread over as many threads as they can use (one vector each); many over as few as give a thread `wanted`
// vectors, or more where a CTA of 512 would not hold them otherwise.
constexpr int kMostNum = 4;
// Dynamic shared memory of any launch: every size is tested against it, and every kernel that wants more than 40 KB is allowed it.
// (An SM has 227 KB for a CTA, of which these kernels' own variables take up to 512 bytes.  With 192 KB fp32 [4096, 12288] forward, then
// not staged, takes 118 against 91 us; the gradient of fp32 [4096, 11000], then by the kernels for any row length, 295 against 125.)
constexpr int64_t kMostShared = 224 * 1024;
static_assert(kDepth * 2 * kMostNum * 512 * 16 <= kMostShared, "the vector form has no test of its own");
RowShape row_shape(int64_t rows, int64_t cols, int vec, int wanted, int sm_count)
{
    RowShape s;
    const int64_t vecs = cols / vec;
    if (rows < 4 * (int64_t)sm_count) wanted = 1;
    while (wanted > 1 && vecs <= 8 * wanted) wanted /= 2;      // (short rows: not fewer than 16 lanes for one)
    for (int num = wanted; num <= kMostNum && s.num == 0; num *= 2) {
        int64_t threads = (vecs + num - 1) / num;
        if (threads <= 32) {
            int p = 1;
            while (p < threads) p *= 2;
            threads = p;
        } else {
            threads = (threads + 31) / 32 * 32;
        }
        if (threads > (num == 1 ? 1024 : 512)) continue;
        s.num = num;
        s.threads = (int)threads;
    }
    return s;
}

// Single elements: `wanted` a thread for many rows, eight for few.  (Forward 32: the fewer threads, the less the sums of a row
// cost.  Backward 16, and eight below eight million elements, where a wave of wide threads has only a row or two for each:
// fp32 [4099, 1023] takes 35, 25 and 23 us with 32, 16 and 8, bf16 [16384, 1023] 56, 54 and 56.)  Wider rows, or rows of
// which two stages (`bytes`, with the affine part) do not fit shared memory, have no shape.
RowShape piece_shape(int64_t rows, int64_t cols, int64_t bytes, int wanted, int sm_count)
{
    RowShape s;
    s.pieces = true;
    int num = rows < 4 * (int64_t)sm_count || cols <= 256 ? 8 : cols <= 512 ? 16 : wanted;
    if (cols > 512 * num) num = 32;
    const int64_t threads = (cols + 32 * num - 1) / (32 * num) * 32;
    if (threads > 512 || (threads > 32 && bytes > kMostShared)) return s;
    s.num = num;
    s.threads = (int)threads;
    return s;
}

// A launch of a kernel over rows: one wave of CTAs, or less if there are fewer rows.
struct RowLaunch {
    const void *kernel = nullptr;
    RowShape shape;
    size_t shared = 0;
    // The CTAs of a launch over so many rows.
    cudaError_t grid(int64_t rows, int sm_count, int64_t *grid_ctas) const
    {
        // (asking takes microseconds: the answers are kept, for each device, whose kernels have limits of their own)
        struct Known { const void *kernel; unsigned block; size_t shared; int device, ctas; };
        static thread_local Known known[32];
        static thread_local int n_known = 0, next = 0;
        int ctas = 0, device = -1;
        cudaError_t e = cudaGetDevice(&device);
        if (e != cudaSuccess) return e;
        for (int i = 0; i < n_known && ctas == 0; ++i)
            if (known[i].device == device && known[i].kernel == kernel && known[i].block == shape.block() && known[i].shared == shared) ctas = known[i].ctas;
        if (ctas == 0) {
            if (shared > 40 * 1024) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMostShared);
            if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&ctas, kernel, (int)shape.block(), shared);
            if (e == cudaSuccess && ctas < 1) e = cudaErrorLaunchOutOfResources;
            if (e != cudaSuccess) return e;
            known[next] = Known{kernel, shape.block(), shared, device, ctas};
            next = (next + 1) % 32;
            if (n_known < 32) ++n_known;
        }
        const int64_t each = shape.rows_a_cta(), want = (rows + each - 1) / each, wave = (int64_t)sm_count * ctas;
        *grid_ctas = want < wave ? want : wave;
        return cudaSuccess;
    }
};

bool on_16_bytes(const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// Does every row of the matrix start on a 16-byte boundary?
bool rows_on_16_bytes(const void *p, int64_t rows, int64_t ld, int dtype)
{
    return on_16_bytes(p) && (rows <= 1 || ld * (dtype == GG_F32 ? 4 : 2) % 16 == 0);
}

template <typename T, typename TW, int kNum>
const void *forward_kernel(const RowShape &s, int64_t cols, bool affine)
{
    if (s.num == kNum) {
        const bool full = cols * (int64_t)sizeof(T) == (int64_t)s.num * s.threads * 16;
        if (s.threads <= 32)
            return full ? reinterpret_cast<const void *>(layer_norm_rows_kernel<T, TW, kNum, kFull, true>)
                        : reinterpret_cast<const void *>(layer_norm_rows_kernel<T, TW, kNum, kRagged, true>);
        if constexpr (sizeof(T) == sizeof(TW))
            if (full && affine) return reinterpret_cast<const void *>(layer_norm_rows_kernel<T, TW, kNum, kKept, false>);
        return full ? reinterpret_cast<const void *>(layer_norm_rows_kernel<T, TW, kNum, kFull, false>)
                    : reinterpret_cast<const void *>(layer_norm_rows_kernel<T, TW, kNum, kRagged, false>);
    }
    if constexpr (kNum > 1) return forward_kernel<T, TW, kNum / 2>(s, cols, affine);
    return nullptr;
}

template <typename T, typename TW, int kNum>
const void *backward_kernel(const RowShape &s, int64_t cols)
{
    if (s.num == kNum) {
        const bool full = cols * (int64_t)sizeof(T) == (int64_t)s.num * s.threads * 16;
        if (s.threads <= 32)
            return full ? reinterpret_cast<const void *>(layer_norm_rows_grad_kernel<T, TW, kNum, kFull, true>)
                        : reinterpret_cast<const void *>(layer_norm_rows_grad_kernel<T, TW, kNum, kRagged, true>);
        return full ? reinterpret_cast<const void *>(layer_norm_rows_grad_kernel<T, TW, kNum, kFull, false>)
                    : reinterpret_cast<const void *>(layer_norm_rows_grad_kernel<T, TW, kNum, kRagged, false>);
    }
    if constexpr (kNum > 1) return backward_kernel<T, TW, kNum / 2>(s, cols);
    return nullptr;
}

template <typename T, typename TW, int kNum>
const void *forward_pieces(const RowShape &s, bool staged)
{
    if (s.num == kNum) {
        if (s.threads <= 32) return reinterpret_cast<const void *>(layer_norm_pieces_kernel<T, TW, kNum, true, true>);
        return staged ? reinterpret_cast<const void *>(layer_norm_pieces_kernel<T, TW, kNum, false, true>)
                      : reinterpret_cast<const void *>(layer_norm_pieces_kernel<T, TW, kNum, false, false>);
    }
    if constexpr (kNum > 8) return forward_pieces<T, TW, kNum / 2>(s, staged);
    return nullptr;
}

template <typename T, typename TW, int kNum>
const void *backward_pieces(const RowShape &s)
{
    if (s.num == kNum)
        return s.threads <= 32 ? reinterpret_cast<const void *>(layer_norm_pieces_grad_kernel<T, TW, kNum, true>)
                               : reinterpret_cast<const void *>(layer_norm_pieces_grad_kernel<T, TW, kNum, false>);
    if constexpr (kNum > 8) return backward_pieces<T, TW, kNum / 2>(s);
    return nullptr;
}

template <typename T, typename TW>
cudaError_t forward(const LayerNormArgs &a, int sm_count, cudaStream_t st)
{
    constexpr int kVec = 16 / sizeof(T);
    const bool vectors = a.cols % kVec == 0 && rows_on_16_bytes(a.x, a.rows, a.x_ld, a.dtype) && rows_on_16_bytes(a.y, a.rows, a.y_ld, a.dtype) &&
                         on_16_bytes(a.weight) && on_16_bytes(a.bias);
    RowLaunch l;
    if (vectors) l.shape = row_shape(a.rows, a.cols, kVec, 4, sm_count);
    if (l.shape.num == 0 && a.cols <= 1 << 16) l.shape = piece_shape(a.rows, a.cols, 2 * (int64_t)piece_bytes<T>((int)a.cols), 32, sm_count);
    if (l.shape.num == 0) {
        layer_norm_kernel<T, TW><<<row_grid(a.rows), kThreads, 0, st>>>(a);
        return cudaGetLastError();
    }
    if (l.shape.pieces) {
        const size_t ring = (size_t)2 * piece_bytes<T>((int)a.cols) * (l.shape.threads <= 32 ? kSoloWarps : 1), affine = affine_bytes((int)a.cols, 2);
        // (staged where the registers, about 112 a thread, allow no more CTAs than then fit shared memory)
        const size_t by_registers = 65536 / (112 * (size_t)l.shape.threads);
        const bool staged = l.shape.threads <= 32 || (a.rows >= 16 * (int64_t)sm_count && by_registers * (ring + affine) <= (size_t)kMostShared);
        l.kernel = forward_pieces<T, TW, 32>(l.shape, staged);
        l.shared = ring + (staged ? affine : 0);
    } else {
        l.kernel = forward_kernel<T, TW, kMostNum>(l.shape, a.cols, a.weight && a.bias);
        l.shared = (size_t)kDepth * l.shape.num * l.shape.block() * 16;
    }
    int64_t ctas = 0;
    const cudaError_t e = l.grid(a.rows, sm_count, &ctas);
    if (e != cudaSuccess) return e;
    void *args[] = {const_cast<LayerNormArgs *>(&a), &l.shape.threads};
    return cudaLaunchKernel(l.kernel, dim3((unsigned)ctas), dim3(l.shape.block()), args, l.shared, st);
}

template <typename T, typename TW>
RowLaunch backward_launch(const LayerNormGradArgs &a, int sm_count)
{
    constexpr int kVec = 16 / sizeof(T);
    const bool vectors = a.cols % kVec == 0 && rows_on_16_bytes(a.x, a.rows, a.x_ld, a.dtype) && rows_on_16_bytes(a.dy, a.rows, a.dy_ld, a.dtype) &&
                         rows_on_16_bytes(a.dx, a.rows, a.dx_ld, a.dtype) && on_16_bytes(a.weight);
    RowLaunch l;
    if (vectors && a.rows > 0) l.shape = row_shape(a.rows, a.cols, kVec, 2, sm_count);
    if (l.shape.num == 0 && a.rows > 0 && a.cols <= 1 << 16) l.shape = piece_shape(a.rows, a.cols, 4 * (int64_t)piece_bytes<T>((int)a.cols) + affine_bytes((int)a.cols, 1),
                                                                                       a.rows * a.cols < (8 << 20) ? 8 : 16, sm_count);
    if (l.shape.num == 0) return l;
    if (l.shape.pieces) {      // (also room for the sums of the columns, 8 bytes each)
        l.kernel = backward_pieces<T, TW, 32>(l.shape);
        l.shared = affine_bytes((int)a.cols, 1) + (size_t)4 * piece_bytes<T>((int)a.cols) * (l.shape.threads <= 32 ? kSoloWarps : 1);
    } else {                   // (the same: 32 lanes' columns)
        l.kernel = backward_kernel<T, TW, kMostNum>(l.shape, a.cols);
        l.shared = (size_t)kDepth * 2 * l.shape.num * l.shape.block() * 16;
    }
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

// So few rows for each warp of a CTA are summed by strips (33 rows of 896, four warps: 3.1 us on the GPU and 4.3 a call, against
// 4.0 and 6.1 with slices; 64 rows 4.3, but 128 rows 7.1 against 5.4.  128 rows of 4096, sixteen warps: 3.8 against 6.8).
constexpr int64_t kFewRows = 16;
static bool by_strips(const LayerNormGradArgs &a, const RowLaunch &l)
{
    return l.kernel != nullptr && (a.dweight != nullptr || a.dbias != nullptr) && a.rows <= kFewRows * (int64_t)(l.shape.block() / 32);
}

cudaError_t layer_norm_grad_slices(const LayerNormGradArgs &a, int sm_count, int *slices)
{
    const RowLaunch l = backward_launch(a, sm_count);
    *slices = 0;
    if (by_strips(a, l)) return cudaSuccess;
    if (l.kernel != nullptr) {
        int64_t n = 0;
        const cudaError_t e = l.grid(a.rows, sm_count, &n);
        if (e != cudaSuccess) return e;
        // four rows or more for each thread of the vector form, where a wave would have less: what the CTAs gain by sharing
        // the rows the sum over their slices takes back (bf16 [2048, 896]: 10.5 against 13.1 us; larger ones do not change)
        const int64_t each = l.shape.rows_a_cta() * (l.shape.pieces ? 1 : 4), most = (a.rows + each - 1) / each;
        *slices = (int)(n < most ? n : most);
        return cudaSuccess;
    }
    const int64_t strips = (a.cols + 31) / 32, most = (a.rows + 63) / 64;
    int64_t n = (4 * (int64_t)sm_count + strips - 1) / strips;
    n = n < most ? n : most;
    *slices = (int)(n < 1 ? 1 : n);
    return cudaSuccess;
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
        auto launch = [&](unsigned ctas, float *slices_of, int strips) {
            int threads = l.shape.threads;
            void *args[] = {const_cast<LayerNormGradArgs *>(&a), &slices_of, &strips, &threads};
            *launches += 1;
            const size_t shared = strips > 0 && l.shared < 8192 ? 8192 : l.shared;
            return cudaLaunchKernel(l.kernel, dim3(ctas + (unsigned)strips), dim3(l.shape.block()), args, shared, st);
        };
        if (by_strips(a, l)) {
            const int strips = (int)((a.cols + 31) / 32);
            const bool over = a.dx == a.x || a.dx == a.dy;       // (then the strips have to be done before dx is written)
            int64_t ctas = 0;
            e = l.grid(a.rows, sm_count, &ctas);
            if (e == cudaSuccess) e = launch(a.dx && !over ? (unsigned)ctas : 0u, nullptr, strips);
            return e == cudaSuccess && a.dx && over ? launch((unsigned)ctas, nullptr, 0) : e;
        }
        e = launch((unsigned)slices, part, 0);
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
