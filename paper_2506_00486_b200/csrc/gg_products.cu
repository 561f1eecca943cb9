// Matrix products of the training operators on the tensor cores: the gated block, the vocabulary loss, their gradients.
//
// One kernel, C = A B^T in bf16 with fp32 sums, and four ends for its tiles (ProductEnd): the operators differ in what becomes
// of a tile while it is still in tensor memory, so neither the logits nor the two projections need a pass of their own.
// A persistent CTA (or pair of CTAs, each with half of A's and half of B's rows of a shared 256 x 256 tile) takes tiles in turn.
// One warp copies the operands into a ring of stages of 64 summed elements by TMA, which also fills what lies beyond a matrix
// with zeros, so no size is special; one feeds the tensor cores; eight end the tile before, which lies in the other half of
// tensor memory.
//
// What bounds it.  Large products: the tensor cores, then the power limit.  The logits of 8192 positions, width 4096, vocabulary 16384, with their
// loss, keep the tensor pipe busy 94 % of the time (657 us, 1673 TFLOP/s); in a loop of seconds the clock falls to 1.25 - 1.45 GHz and
// 16384 x 4096 x 32000 takes 2.97 ms = 1445 TFLOP/s, where a library product that only writes the logits takes 2.95 - 3.07.  A few rows: one pass over
// B (5.1 - 5.7 TB/s).  What made most of it: pairs of CTAs on 256 x 256 tiles (3.74 -> 3.36 ms for that loss), loops that a whole warp
// walks, so that addresses stay in uniform registers (-> 2.94 ms), barriers that do not wait for stores (below).
#include <cuda.h>
#include <math.h>

#include <atomic>
#include <type_traits>

#include "gg.h"
#include "gg_after.cuh"
#include "gg_element.cuh"
#include "gg_products.cuh"
#include "gg_tensor.cuh"

namespace gg {
namespace {

constexpr int kBlockK = 64;             // summed elements of a stage: 128 bytes, a row of the swizzle
// Warps that end tiles: eight, with 192 KB for the ring of stages; or sixteen, which need 32 KB of that for what they send out.
__host__ __device__ constexpr int ring_bytes(int end_warps) { return (end_warps == 16 ? 160 : 192) * 1024; }
constexpr int kMostStages = 16;
constexpr int kOutBytes = 4096;         // 32 rows of 64 bf16 on their way out, for each warp of the end
constexpr int kShared = 1024 + ring_bytes(8) + 8 * kOutBytes;      // (either way)
constexpr int kAccColumns = 256;        // of tensor memory for one accumulator; there are two
constexpr int kLseRun = 8;              // stages after which the sums of a logit are taken out of the tensor cores
constexpr int kLseOfOne = kStore + 1;       // kLse where the sum is one such run
constexpr float kLog2e = 1.4426950408889634f;

struct Output {
    uint16_t *p;
    int64_t ld;
    int whole;           // every row starts on a 16-byte boundary
};

// n / d for 0 <= n < 2^31 without a division (five of them stand in the path of each tile otherwise), as Granlund and Montgomery
// divide by invariant integers (1994): mul is
// 2^(32 + shift) / d rounded up, and the error of that stays below 1 / d as 2^(31 + ceil(log2 d)) / d has 32 bits.
struct Divider {
    uint32_t d, mul, shift;
    __device__ __forceinline__ int of(int n) const { return d == 1 ? n : (int)(__umulhi((uint32_t)n, mul) >> shift); }
};

struct Params {
    CUtensorMap a[2], b[2];
    Output out[3];                      // kGated: h, gate, up
    int64_t m, n;
    int tile_n;                         // rows of B in a tile (kGated: half of them gate's, half up's)
    int cols;                           // columns of C in a tile
    int tiles_m, tiles_n, band, total, kblocks, all_k, splits;      // (up to two batches of so many splits)
    int each_k, more_k;                 // stages of a split, and how many splits have one more
    Divider by_outer, by_band, by_height, by_last;      // tiles of a batch or split, of a band; its height, the last band's
    int stages, bytes_a, bytes_b;       // of the ring: A's part has only as many rows as A
    int act;
    float2 *part;
    float *target_logit;
    const int64_t *target;
    int64_t vocab, first;
    const float *lse, *dloss;
    int64_t positions;
    float *scale;
    float *f32;
    int64_t f32_ld;
    int mode;
    uint32_t polls, extra_bytes;        // after so many a wait gives up; test hook: bytes that are expected and never come
    uint32_t *gave_up;
};

// 2^x in one instruction (2 units off at most; what would be subnormal is 0).
__device__ __forceinline__ float power2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// ------------------------------------------------------------------ activations
// Two at a time: the ends of a narrow product are bound by them (gelu at width 896: 97 us a call with erfcf, 75 one by one, 67 so; silu 52 to 65).
__device__ __forceinline__ float reciprocal(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ f32x2 power2(f32x2 x)
{
    const float2 f = halves(x);
    return pair(power2(f.x), power2(f.y));
}
__device__ __forceinline__ f32x2 reciprocal(f32x2 x)
{
    const float2 f = halves(x);
    return pair(reciprocal(f.x), reciprocal(f.y));
}
// 1 / (1 + e^-a): an e^-a that overflows gives 0.
__device__ __forceinline__ f32x2 sigmoid(f32x2 a) { return reciprocal(add2(power2(mul2(a, both(-kLog2e))), both(1.0f))); }
// The normal distribution function of a and e = exp(-a^2 / 2).  Its tail at -z is e R(z), R falling slowly from 1/2; R is a polynomial in
// t = 1 / (1 + 0.3 z) without a constant term, fitted for least relative error over [0, 20] (6.5e-7 in fp32).  (1 + erf is no good for negative a.)
__device__ __forceinline__ f32x2 normal(f32x2 a, f32x2 &e)
{
    const f32x2 z = a & 0x7FFFFFFF7FFFFFFFull, t = reciprocal(fma2(z, both(0.3f), both(1.0f)));
    f32x2 r = both(0.0330343359f);
    r = fma2(r, t, both(-0.1463946f));
    r = fma2(r, t, both(0.188128167f));
    r = fma2(r, t, both(-0.0373476765f));
    r = fma2(r, t, both(0.120195597f));
    r = fma2(r, t, both(0.102349824f));
    r = fma2(r, t, both(0.120381962f));
    r = fma2(r, t, both(0.119652203f));
    e = power2(mul2(mul2(z, z), both(-0.5f * kLog2e)));
    const float2 tail = halves(mul2(e, mul2(r, t))), x = halves(a);
    return pair(x.x > 0.0f ? 1.0f - tail.x : tail.x, x.y > 0.0f ? 1.0f - tail.y : tail.y);
}
// The sigmoid of 2 sqrt(2 / pi) (a + 0.044715 a^3), which is (1 + tanh) / 2, and the derivative of that argument.  Beyond 30 it is 0 or 1.
__device__ __forceinline__ f32x2 cubic_sigmoid(f32x2 a, f32x2 &inner)
{
    const float2 f = halves(a);
    const f32x2 b = pair(fminf(fmaxf(f.x, -30.0f), 30.0f), fminf(fmaxf(f.y, -30.0f), 30.0f)), q = mul2(b, b);
    inner = fma2(q, both(1.5957691216057308f * 0.134145f), both(1.5957691216057308f));
    return sigmoid(mul2(b, fma2(q, both(1.5957691216057308f * 0.044715f), both(1.5957691216057308f))));
}
// max(a, 0), NaN for NaN
__device__ __forceinline__ float positive(float a)
{
    float y;
    asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(y) : "f"(a));
    return y;
}
template <int kAct>
__device__ __forceinline__ f32x2 activation(f32x2 a)
{
    f32x2 more;
    if constexpr (kAct == GG_ACT_SILU) return mul2(a, sigmoid(a));
    if constexpr (kAct == GG_ACT_GELU) return mul2(a, normal(a, more));
    if constexpr (kAct == GG_ACT_GELU_TANH) return mul2(a, cubic_sigmoid(a, more));
    const float2 f = halves(a);
    return pair(positive(f.x), positive(f.y));
}
// act(a) and its derivative
template <int kAct>
__device__ __forceinline__ void slope(f32x2 a, f32x2 &value, f32x2 &d)
{
    f32x2 more;
    if constexpr (kAct == GG_ACT_SILU) {
        const f32x2 s = sigmoid(a);
        value = mul2(a, s);
        d = fma2(value, fma2(s, both(-1.0f), both(1.0f)), s);
    } else if constexpr (kAct == GG_ACT_GELU) {
        const f32x2 c = normal(a, more);
        value = mul2(a, c);
        d = fma2(mul2(a, both(0.3989422804014327f)), more, c);
    } else if constexpr (kAct == GG_ACT_GELU_TANH) {
        const f32x2 s = cubic_sigmoid(a, more);
        value = mul2(a, s);
        d = fma2(mul2(value, fma2(s, both(-1.0f), both(1.0f))), more, s);
    } else {
        const float2 f = halves(a);
        value = activation<GG_ACT_RELU>(a);
        d = pair(f.x > 0.0f ? 1.0f : f.x != f.x ? f.x : 0.0f, f.y > 0.0f ? 1.0f : f.y != f.y ? f.y : 0.0f);
    }
}
template <typename F>
__device__ __forceinline__ void by_activation(int act, F f)
{
    if (act == GG_ACT_SILU) f(std::integral_constant<int, GG_ACT_SILU>());
    else if (act == GG_ACT_GELU) f(std::integral_constant<int, GG_ACT_GELU>());
    else if (act == GG_ACT_GELU_TANH) f(std::integral_constant<int, GG_ACT_GELU_TANH>());
    else f(std::integral_constant<int, GG_ACT_RELU>());
}

// ------------------------------------------------------------------ the ends of a tile
struct Tile {
    int64_t row0, row;   // first row of the warp, row of this thread
    int64_t col;         // first column of the tile
    int width;           // its columns that C has
    int batch, sums, n_tile;      // sums: which of the fp32 matrices (kStore)
    uint32_t acc;        // its sums: tensor memory of the warp's lanes
    // of this thread's row (both ends of the loss, kDlogits)
    int64_t of;          // its target
    float lse, weight;
    __device__ __forceinline__ int target(int64_t first) const      // where in the tile that is, or -1
    {
        const int64_t at = of - first - col;
        return of >= 0 && at >= 0 && at < width ? (int)at : -1;
    }
};

// Takes 32 rows of up to 64 bf16 out through shared memory, so that a store instruction writes whole 128-byte pieces of rows and
// not 16 bytes of each.  (The gradient of a 151936 x 896 matrix from 33 positions, which is nearly all stores: 114 us by tensor copies of
// 32 x 32, 95 so.)  A lane has a row; its 16-byte pieces are exchanged by row, so that eight lanes reach all banks either way.
struct Way {
    uint32_t at, mine;   // the warp's place; the lane's row in it, its first piece where the exchange puts it
    int lane;
    __device__ __forceinline__ Way(uint32_t place, int lane_) : at(place), mine(place + lane_ * 128 + ((lane_ & 7) << 4)), lane(lane_) {}
    __device__ __forceinline__ void put(int part, const uint32_t (&w)[16]) const       // 32 columns, part 0 or 1
    {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(mine ^ (uint32_t)((4 * part + j) << 4)), "r"(w[4 * j]), "r"(w[4 * j + 1]),
                         "r"(w[4 * j + 2]), "r"(w[4 * j + 3]) : "memory");
    }
    // The rows from column c of the tile on; kPieces 16-byte pieces of each: 8, or 4 for part 0 alone.
    template <int kPieces>
    __device__ __forceinline__ void send(const Params &p, const Output &o, const Tile &t, int c) const
    {
        constexpr int kRows = 32 / kPieces;
        __syncwarp();
        const int piece = lane % kPieces, first = lane / kPieces, rows = p.m - t.row0 < 32 ? (int)(p.m - t.row0) : 32;
        uint16_t *q = o.p + (t.row0 + first) * o.ld + t.col + c + piece * 8;
        if (o.whole && rows == 32 && t.width - c >= kPieces * 8) {
            // (rows `first`, first + kRows, ...: the exchange has two turns, or one)
            const uint32_t from = at + first * 128 + ((piece ^ first) << 4), turned = kPieces == 8 ? from ^ 64u : from;
            uint32_t w[kPieces][4];
#pragma unroll
            for (int i = 0; i < kPieces; ++i)
                asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[i][0]), "=r"(w[i][1]), "=r"(w[i][2]), "=r"(w[i][3])
                             : "r"((i & 1 ? turned : from) + i * kRows * 128) : "memory");
            const int64_t down = kRows * o.ld;
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                *reinterpret_cast<uint4 *>(q) = make_uint4(w[i][0], w[i][1], w[i][2], w[i][3]);
                q += down;
            }
        } else {
            send_some<kPieces>(o, t, c, q, piece, first, rows);
        }
        __syncwarp();
    }
    template <int kPieces>
    __device__ __forceinline__ void send_some(const Output &o, const Tile &t, int c, uint16_t *q, int piece, int first, int rows) const
    {
        constexpr int kRows = 32 / kPieces;
        const int left = t.width - c - piece * 8;
        if (!o.whole) {
            // element by element: a lane takes columns lane and lane + 32 of every row (pairs from the first even element on measured
            // twice as long)
            const bool one = c + lane < t.width, two = kPieces == 8 && c + 32 + lane < t.width;
            const uint32_t from = at + ((uint32_t)lane >> 3 << 4) + (lane & 7) * 2;
            uint16_t *e = o.p + t.row0 * o.ld + t.col + c + lane;
#pragma unroll 8
            for (int r = 0; r < 32; ++r) {
                uint16_t v = 0, w = 0;
                asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"((from ^ (r & 7) << 4) + r * 128) : "memory");
                if constexpr (kPieces == 8) asm volatile("ld.shared.u16 %0, [%1];" : "=h"(w) : "r"((from ^ ((r & 7) << 4 ^ 64)) + r * 128) : "memory");
                if (one && r < rows) e[0] = v;
                if (two && r < rows) e[32] = w;
                e += o.ld;
            }
        } else if (left >= 8) {
            for (int r = first; r < rows; r += kRows) {
                uint32_t w[4];
                asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
                             : "r"(at + r * 128 + ((piece ^ (r & 7)) << 4)) : "memory");
                *reinterpret_cast<uint4 *>(q + (r - first) * o.ld) = make_uint4(w[0], w[1], w[2], w[3]);
            }
        } else {
            // the last columns of rows that are no multiple of eight long
            for (int r = first; r < rows; r += kRows)
                for (int e = 0; e < left; ++e) q[(r - first) * o.ld + e] = element(r, piece * 8 + e);
        }
    }
    __device__ __forceinline__ uint16_t element(int r, int e) const
    {
        uint16_t v;
        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(at + r * 128 + ((e >> 3 ^ (r & 7)) << 4) + (e & 7) * 2) : "memory");
        return v;
    }
};

// The weights of the positions are mostly one number, 1 / their count, and d = weight * (p - 1) is then mostly that number too: rounded
// to bf16 it may be off by 2^-8 in all of them alike (the gradient of 33 positions: 0.4 % off as a whole).  So d is kept relative to the
// mantissa, 1 .. 2, of the first weight that is not 0, and the sums are multiplied by it: p - 1 itself is rounded (0.2 %, and
// no longer alike).  Every warp of the end looks at the first 256 rows; a batch that begins without any (padding) is searched by all of them together,
// 256 rows each at once and four times that between barriers.  The products that sum d, and later pieces of the vocabulary, are told.  A search of 2^19 rows
// takes 0.45 ms; by each warp for itself it took 6.5.
__device__ __forceinline__ float first_weight(const float *dloss, const int64_t *target, int64_t from, int64_t rows)      // of 256 rows, or 0
{
    const int lane = threadIdx.x & 31;
    float g[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int64_t at = from + 32 * j + lane;
        g[j] = at < rows && target[at] >= 0 ? fabsf(dloss[at]) : 0.0f;
    }
    float first = 0.0f;
#pragma unroll
    for (int j = 7; j >= 0; --j) {
        const uint32_t some = __ballot_sync(~0u, g[j] > 1e-30f && g[j] < 1e30f);
        const float v = __shfl_sync(~0u, g[j], some != 0 ? __ffs(some) - 1 : 0);
        if (some != 0) first = v;
    }
    return first;
}
template <int kWarps>
__device__ __forceinline__ float weight_mantissa(const float *dloss, const int64_t *target, int64_t rows, int warp)
{
    constexpr int kEach = 4;                       // blocks of 256 rows
    __shared__ float found[2][kWarps * kEach];
    float first = first_weight(dloss, target, 0, rows);
    int turn = 0;
    for (int64_t from = 256; first == 0.0f && from < rows; from += 256 * kWarps * kEach, turn ^= 1) {
#pragma unroll 1
        for (int i = 0; i < kEach; ++i) {
            const float v = first_weight(dloss, target, from + 256 * (i * kWarps + warp), rows);
            if ((threadIdx.x & 31) == 0) found[turn][i * kWarps + warp] = v;
        }
        // (of these warps alone.  What is written in this turn is read before the next but one, behind the next's barrier)
        asm volatile("bar.sync 1, %0;" ::"n"(32 * kWarps) : "memory");
        for (int i = 0; i < kWarps * kEach && first == 0.0f; ++i) first = found[turn][i];
    }
    return first == 0.0f ? 1.0f : __uint_as_float((__float_as_uint(first) & 0x7FFFFFu) | 0x3F800000u);
}

// 32 columns as pairs.
__device__ __forceinline__ void read_pairs(uint32_t at, f32x2 (&v)[16])
{
    float x[32];
    tmem_read(at, x);
    tmem_read_wait();
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = pair(x[2 * i], x[2 * i + 1]);
}

// A tile's columns go to the warps of a lane quarter in turn, 32 or 64 at a time.
__device__ __forceinline__ void end_gated(const Params &p, const Tile &t, int share, const Way &way)
{
#pragma unroll 1
    for (int c = share * 32; c < t.width; c += 64) {
        f32x2 g[16], u[16];
        {
            float x[32], y[32];
            tmem_read(t.acc + c, x);
            tmem_read(t.acc + p.cols + c, y);
            tmem_read_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                g[i] = pair(x[2 * i], x[2 * i + 1]);
                u[i] = pair(y[2 * i], y[2 * i + 1]);
            }
        }
        uint32_t w[16];
        if (p.out[1].p != nullptr) {
#pragma unroll
            for (int i = 0; i < 16; ++i) w[i] = narrow2(g[i]);
            way.put(0, w);
            way.send<4>(p, p.out[1], t, c);
        }
        if (p.out[2].p != nullptr) {
#pragma unroll
            for (int i = 0; i < 16; ++i) w[i] = narrow2(u[i]);
            way.put(0, w);
            way.send<4>(p, p.out[2], t, c);
        }
        by_activation(p.act, [&](auto act) {
#pragma unroll
            for (int i = 0; i < 16; ++i) w[i] = narrow2(mul2(activation<decltype(act)::value>(g[i]), u[i]));
        });
        way.put(0, w);
        way.send<4>(p, p.out[0], t, c);
    }
}

// The logits of a warp's share of the tile, 32 columns of every 32 * kShare.  The tensor cores do not round their sums to nearest: a long one
// comes out too small.  So after every kLseRun stages what they have is added here, rounded, and they begin anew, in the other
// accumulator.  The loss of 16384 positions of width 4096: 2.5e-6 off without that, 6e-7 with runs of 16 stages, 2.8e-7 with 8, all at one speed; 1.4e-7
// with 4, which takes 15 % longer.
template <int kShare>
struct Logits {
    static constexpr int kRuns = 16 / kShare;            // of 16 columns
    f32x2 v[kRuns][8];
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < kRuns; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = both(0.0f);
    }
    static __device__ __forceinline__ int column(int share, int i) { return share * 32 + (i >> 1) * 32 * kShare + (i & 1) * 16; }
    __device__ __forceinline__ void take(const Tile &t, int share)
    {
#pragma unroll
        for (int i = 0; i < kRuns; ++i)
            if (column(share, i) < t.width) {
                float x[16];
                tmem_read(t.acc + column(share, i), x);
                tmem_read_wait();
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i][j] = add2(v[i][j], pair(x[2 * j], x[2 * j + 1]));
            }
    }
};

// The sum is taken relative to the largest.  A NaN, which no maximum shows, reaches the sum by its own term.
template <int kShare>
__device__ __forceinline__ void end_lse(const Params &p, const Tile &t, int share, Logits<kShare> &l)
{
    const int target = t.target(p.first);
    float most = -INFINITY;
#pragma unroll
    for (int i = 0; i < Logits<kShare>::kRuns; ++i) {
        const int c = Logits<kShare>::column(share, i), left = t.width - c;
        if (left < 16) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float2 x = halves(l.v[i][j]);
                l.v[i][j] = pair(2 * j < left ? x.x : -INFINITY, 2 * j + 1 < left ? x.y : -INFINITY);
            }
        }
        if ((unsigned)(target - c) < 16u) {
            float x = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float2 y = halves(l.v[i][j]);
                x = target - c == 2 * j ? y.x : target - c == 2 * j + 1 ? y.y : x;
            }
            p.target_logit[t.row] = x;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float2 x = halves(l.v[i][j]);
            most = fmaxf(most, fmaxf(x.x, x.y));
        }
    }
    const f32x2 base = both(most == -INFINITY ? 0.0f : -most);
    f32x2 sum[2] = {both(0.0f), both(0.0f)};
#pragma unroll
    for (int i = 0; i < Logits<kShare>::kRuns; ++i)
        if (Logits<kShare>::column(share, i) < t.width) {
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j & 1] = add2(sum[j & 1], power2(mul2(add2(l.v[i][j], base), both(kLog2e))));
        }
    const float2 s = halves(add2(sum[0], sum[1]));
    if (t.row < p.m) p.part[(int64_t)(kShare * t.n_tile + share) * p.m + t.row] = make_float2(most, s.x + s.y);
}

// The same for sums of one run: 32 columns at a time from tensor memory, a sum rescaled where the largest grows.  A tile of so few stages is
// all end, and the end above, unrolled around its registers and run once a tile, is bound by the fetching of its instructions: in a build that read
// the clock around it, 6909 x 64 x 50688 took 4560 clocks for a tile of 64 columns and 5600 for one of 256, this 2070 and 4250; with sixteen warps
// 4770 and 3750 for 256 (the exponentials alone 2050).  The loss of 6909 x 64 x 50688 176 and 143 us, of 526 x 128 x 34071 22.7 and 19.3.
template <int kShare>
__device__ __forceinline__ void end_lse_of_one(const Params &p, const Tile &t, int share)
{
    const int target = t.target(p.first);
    float most = -INFINITY, sum = 0.0f;
#pragma unroll 1
    for (int c = share * 32; c < t.width; c += 32 * kShare) {
        f32x2 v[16];
        read_pairs(t.acc + c, v);
        const int left = t.width - c, at = target - c;
        if (left < 32) {
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const float2 x = halves(v[j]);
                v[j] = pair(2 * j < left ? x.x : -INFINITY, 2 * j + 1 < left ? x.y : -INFINITY);
            }
        }
        if ((unsigned)at < 32u) {
            float x = 0.0f;
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const float2 y = halves(v[j]);
                x = at == 2 * j ? y.x : at == 2 * j + 1 ? y.y : x;
            }
            p.target_logit[t.row] = x;
        }
        __syncwarp();
        float top[4] = {most, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const float2 x = halves(v[j]);
            top[j & 3] = fmaxf(top[j & 3], fmaxf(x.x, x.y));
        }
        const float grown = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])), from = grown == -INFINITY ? 0.0f : grown;
        const f32x2 base = both(-from);
        f32x2 part[2] = {both(0.0f), both(0.0f)};
#pragma unroll
        for (int j = 0; j < 16; ++j) part[j & 1] = add2(part[j & 1], power2(mul2(add2(v[j], base), both(kLog2e))));
        const float2 s = halves(add2(part[0], part[1]));
        sum = sum * power2((most - from) * kLog2e) + (s.x + s.y);
        most = grown;
    }
    if (t.row < p.m) p.part[(int64_t)(kShare * t.n_tile + share) * p.m + t.row] = make_float2(most, sum);
}

template <int kShare>
__device__ __forceinline__ void end_dlogits(const Params &p, const Tile &t, int share, const Way &way, float scale)
{
    const int64_t of = t.of;
    const int target = t.target(p.first);
    const float g = of < 0 ? 0.0f : of >= p.vocab ? NAN : t.weight / scale;
    const f32x2 lse = both(-t.lse);
#pragma unroll 1
    for (int c = share * 64; c < t.width; c += 64 * kShare) {
#pragma unroll
        for (int part = 0; part < 2; ++part) {
            f32x2 v[16];
            read_pairs(t.acc + c + 32 * part, v);
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = mul2(both(g), power2(mul2(add2(v[i], lse), both(kLog2e))));
            const int at = target - c - 32 * part;
            if ((unsigned)at < 32u) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float2 x = halves(v[i]);
                    v[i] = pair(at == 2 * i ? x.x - g : x.x, at == 2 * i + 1 ? x.y - g : x.y);
                }
            }
            uint32_t w[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) w[i] = of < 0 ? 0u : narrow2(v[i]);       // (no position: 0, whatever its logits are)
            way.put(part, w);
            __syncwarp();
        }
        way.send<8>(p, p.out[0], t, c);
    }
}

__device__ __forceinline__ void add_old(const Output &o, const Tile &t, int c, f32x2 (&v)[16])
{
    const uint16_t *q = o.p + t.row * o.ld + t.col + c;
    const int left = t.width - c;
    if (left >= 32 && o.whole) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint4 x = reinterpret_cast<const uint4 *>(q)[i];
            v[4 * i] = add2(v[4 * i], widen2(x.x));
            v[4 * i + 1] = add2(v[4 * i + 1], widen2(x.y));
            v[4 * i + 2] = add2(v[4 * i + 2], widen2(x.z));
            v[4 * i + 3] = add2(v[4 * i + 3], widen2(x.w));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            v[i] = add2(v[i], pair(2 * i < left ? widen<uint16_t>(q[2 * i]) : 0.0f, 2 * i + 1 < left ? widen<uint16_t>(q[2 * i + 1]) : 0.0f));
    }
}

// fp32 sums: into memory, added to what is there, or what is there added to them.
__device__ __forceinline__ void fp32_sums(const Params &p, const Tile &t, int c, f32x2 (&v)[16])
{
    float4 *f = reinterpret_cast<float4 *>(p.f32 + ((int64_t)t.sums * p.m + t.row) * p.f32_ld + t.col + c);
    if (p.mode != kStoreF32) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float4 o = f[i];
            v[2 * i] = add2(v[2 * i], pair(o.x, o.y));
            v[2 * i + 1] = add2(v[2 * i + 1], pair(o.z, o.w));
        }
    }
    if (p.mode != kStoreBf16OfSum) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 x = halves(v[2 * i]), y = halves(v[2 * i + 1]);
            f[i] = make_float4(x.x, x.y, y.x, y.y);
        }
    }
}

template <int kShare>
__device__ __forceinline__ void end_store(const Params &p, const Tile &t, int share, const Way &way, float scale)
{
    const bool there = t.row < p.m;
    const f32x2 scales = both(scale);
#pragma unroll 1
    for (int c = share * 64; c < t.width; c += 64 * kShare) {
#pragma unroll
        for (int part = 0; part < 2; ++part) {
            f32x2 v[16];
            read_pairs(t.acc + c + 32 * part, v);
            if (p.mode != kStoreBf16 && p.mode != kAddBf16) {
                if (there && c + 32 * part < t.width) fp32_sums(p, t, c + 32 * part, v);
                __syncwarp();
                if (p.mode != kStoreBf16OfSum) continue;
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = mul2(v[i], scales);
            if (p.mode == kAddBf16) {
                if (there && c + 32 * part < t.width) add_old(p.out[t.batch], t, c + 32 * part, v);
                __syncwarp();
            }
            uint32_t w[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) w[i] = narrow2(v[i]);
            way.put(part, w);
        }
        if (p.mode != kStoreF32 && p.mode != kAddF32) way.send<8>(p, p.out[t.batch], t, c);
    }
}

// ------------------------------------------------------------------ the kernel
struct Work { int m_tile, n_tile, outer; };
__device__ __forceinline__ Work work_of(const Params &p, int w)
{
    Work r;
    r.outer = p.by_outer.of(w);
    w -= r.outer * (int)p.by_outer.d;
    const int band = p.by_band.of(w), first = band * p.band;
    w -= band * (int)p.by_band.d;
    const bool last = p.tiles_m - first < p.band;
    r.n_tile = last ? p.by_last.of(w) : p.by_height.of(w);
    r.m_tile = first + (w - r.n_tile * (int)(last ? p.by_last.d : p.by_height.d));
    return r;
}
__device__ __forceinline__ int split_start(const Params &p, int split) { return split * p.each_k + (split < p.more_k ? split : p.more_k); }

// What was started on its way to a CTA's shared memory, as the warps that started it leave it there for both CTAs of a pair.
struct Started {
    uint32_t failed;        // a wait ran out, in either CTA
    uint32_t copied[2];     // stages that each CTA's copies were issued for (read in the first)
    uint32_t used;          // stages that the products hand back
    uint32_t ended[2];      // times that an accumulator was handed over
};
// A CTA may end only when nothing is under way to its shared memory any more.  Where every wait was met that is so: the copies
// have been multiplied, the ends have waited for the accumulators and the copying warp for its stages.  Where one ran out, this waits for the copies, the
// products and the arrivals that had been started, by the first two warps of each CTA; the second may have copied for more stages than the first.
constexpr uint32_t kLeastPolls = 1 << 14;       // (8 ms or so, whatever the cap on waits is: a copy takes microseconds)
template <int kCtas>
__device__ __forceinline__ void settle(volatile const Started &was, int warp, uint32_t rank, uint32_t stages, uint32_t full, uint32_t empty, uint32_t done, uint32_t drained,
                                       uint32_t polls)
{
    uint32_t left = polls / 16 > kLeastPolls ? polls / 16 : kLeastPolls;      // (for all of them together: they all started long ago)
    auto wait = [&](uint32_t bar, uint32_t parity) {
        while (left > 0 && !barrier_test(bar, parity)) --left;
    };
    auto last_of = [&](uint32_t bars, uint32_t n) {
        for (uint32_t i = n > stages ? n - stages : 0; i < n; ++i) wait(bars + 8 * (i % stages), (i / stages) & 1);
    };
    if (warp == 0) {
        if (rank == 0) last_of(full, was.copied[0] > was.copied[1] ? was.copied[0] : was.copied[1]);
        last_of(empty, was.used);
    } else if (warp == 1) {
        if (rank == 0 && elect_lane()) product_commit<kCtas>(drained);      // (the lane that issued the products)
        __syncwarp();
        wait(drained, 0);
        for (uint32_t i = 0; i < 2; ++i)
            if (was.ended[i] > 0) wait(done + 8 * i, (was.ended[i] - 1) & 1);
    }
    __syncwarp();
}

// kHalves 2: a pair's tile has 512 rows, as two halves of 256 with an accumulator each.  Otherwise the two accumulators take turns.
template <int kCtas, int kHalves, bool kAT, bool kBT, int kEnd, int kEndWarps>
__global__ void __launch_bounds__(32 * (4 + kEndWarps), 1) product_kernel(const __grid_constant__ Params p)
{
    constexpr int kShare = kEndWarps / 4;
    extern __shared__ uint8_t shared_bytes[];
    __shared__ uint64_t bars[2 * kMostStages + 5];
    __shared__ uint32_t tmem_at;
    __shared__ Started started;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = kCtas == 2 ? cluster_rank() : 0;
    const uint32_t ring = (shared_address(shared_bytes) + 1023) & ~1023u, half_a = p.bytes_a, bytes_a = kHalves * half_a, bytes = bytes_a + p.bytes_b, stages = p.stages;
    const uint32_t full = shared_address(bars), empty = full + 8 * kMostStages, done = empty + 8 * kMostStages, free_at = done + 16, drained = done + 32;

    if (warp == 0 && lane == 0) {
        for (uint32_t i = 0; i < stages; ++i) {
            barrier_init(full + 8 * i, 1);
            barrier_init(empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            barrier_init(done + 8 * i, 1);
            barrier_init(free_at + 8 * i, kEndWarps * kCtas);
        }
        barrier_init(drained, 1);
        started = Started{};
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        prefetch_map(&p.a[0]);
        prefetch_map(&p.b[0]);
    }
    if (warp == 2) tmem_alloc<kCtas>(shared_address(&tmem_at), 2 * kAccColumns);
    tmem_before_sync();
    if constexpr (kCtas == 2) cluster_sync();
    else __syncthreads();
    tmem_after_sync();
    const uint32_t tmem = tmem_at;
    wait_for_the_one_before();

    const int first = blockIdx.x / kCtas, step = gridDim.x / kCtas;
    bool failed = false;
    auto leave = [&](const uint32_t &field, uint32_t value, uint32_t cta) { cluster_store(peer_address(shared_address(&field), cta), value); };
    // (a warp walks its loop as one, and one lane issues: so addresses and coordinates stay in uniform registers)
    if (warp == 0) {
        // ---- copies
        const bool leader = elect_lane();
        const int rows_b = p.tile_n / kCtas;
        uint32_t stage = 0, phase = 0, issued = 0;
        for (int w = first; w < p.total && !failed; w += step) {
            const Work t = work_of(p, w);
            const int batch = t.outer >= p.splits, split = t.outer - batch * p.splits;
            const int m0 = t.m_tile * 128 * kCtas * kHalves + (int)rank * 128;
            const int n0 = t.n_tile * p.cols + (kEnd == kGated ? 0 : (int)rank * rows_b);
            const int end = split_start(p, split + 1);
            for (int kb = split_start(p, split); kb < end; ++kb) {
                if (!barrier_wait(empty + 8 * stage, phase ^ 1, p.polls)) { failed = true; break; }
                if (leader) {
                    if (rank == 0) barrier_expect(full + 8 * stage, bytes * kCtas + p.extra_bytes);
                    const int segment = kb >= p.kblocks, k0 = (kb - segment * p.kblocks) * kBlockK, which = segment | batch;
                    const uint32_t to_a = ring + stage * bytes, to_b = to_a + bytes_a;
                    const uint32_t signal = kCtas == 2 ? peer_address(full + 8 * stage, 0) : full + 8 * stage;
#pragma unroll
                    for (int h = 0; h < kHalves; ++h) {
                        if constexpr (kAT) {
                            tensor_copy<kCtas>(to_a + half_a * h, &p.a[which], m0 + 256 * h, k0, signal);
                            tensor_copy<kCtas>(to_a + half_a * h + 8192, &p.a[which], m0 + 256 * h + 64, k0, signal);
                        } else {
                            tensor_copy<kCtas>(to_a + half_a * h, &p.a[which], k0, m0 + 256 * h, signal);
                        }
                    }
                    if constexpr (kBT) {
                        for (int i = 0; i < rows_b; i += 64) tensor_copy<kCtas>(to_b + 128 * i, &p.b[which], n0 + i, k0, signal);
                    } else if constexpr (kEnd == kGated && kCtas == 1) {
                        tensor_copy<kCtas>(to_b, &p.b[0], k0, n0, signal);
                        tensor_copy<kCtas>(to_b + p.cols * 128, &p.b[1], k0, n0, signal);
                    } else if constexpr (kEnd == kGated) {
                        tensor_copy<kCtas>(to_b, &p.b[rank], k0, n0, signal);
                    } else {
                        tensor_copy<kCtas>(to_b, &p.b[which], k0, n0, signal);
                    }
                }
                ++issued;
                if (++stage == stages) { stage = 0; phase ^= 1; }
            }
        }
        if (leader) leave(started.copied[rank], issued, 0);
        // the products hand every stage back, to both CTAs of a pair
        for (uint32_t i = 0; i < stages && !failed; ++i) {
            failed = !barrier_wait(empty + 8 * stage, phase ^ 1, p.polls);
            if (++stage == stages) { stage = 0; phase ^= 1; }
        }
    } else if (warp == 1 && rank == 0) {
        // ---- products
        const bool leader = elect_lane();
        const uint32_t shape = product_shape<128 * kCtas, kAT, kBT>(p.tile_n);
        uint32_t stage = 0, phase = 0, units = 0, used = 0, ended_first = 0, ended_second = 0;
        auto issue = [&](uint32_t at, uint32_t acc, bool fresh) {
            const uint64_t a = tile_descriptor<kAT>(ring + at * bytes + (kHalves == 2 ? acc * half_a : 0)), b = tile_descriptor<kBT>(ring + at * bytes + bytes_a);
            if (leader) {
#pragma unroll
                for (int i = 0; i < kBlockK / 16; ++i)
                    product_issue<kCtas>(tmem + acc * kAccColumns, a + i * tile_step<kAT>(), b + i * tile_step<kBT>(), shape, !fresh || i > 0);
            }
        };
        auto commit = [&](uint32_t bar) {
            if (leader) product_commit<kCtas>(bar);
        };
        for (int w = first; w < p.total && !failed; w += step) {
            const int outer = work_of(p, w).outer, split = outer - (outer >= p.splits ? p.splits : 0);
            const int begin = split_start(p, split), end = split_start(p, split + 1);
            if constexpr (kHalves == 1) {
                const int run = kEnd == kLse ? kLseRun : end - begin;
                for (int from = begin; from < end && !failed; from += run, ++units) {
                    const uint32_t acc = units & 1;
                    if (!barrier_wait(free_at + 8 * acc, (units >> 1 & 1) ^ 1, p.polls)) { failed = true; break; }
                    tmem_after_sync();
                    const int to = from + run < end ? from + run : end;
                    for (int kb = from; kb < to; ++kb) {
                        if (!barrier_wait(full + 8 * stage, phase, p.polls)) { failed = true; break; }
                        tmem_after_sync();
                        issue(stage, acc, kb == from);
                        commit(empty + 8 * stage);
                        ++used;
                        if (++stage == stages) { stage = 0; phase ^= 1; }
                    }
                    if (failed) break;
                    commit(done + 8 * acc);
                    ended_first += acc ^ 1;
                    ended_second += acc;
                }
            } else {
                // Both accumulators belong to this tile.  At its start and its end a ring's worth of stages is taken for the first
                // half and then again for the second, so that the first half's end runs while the second is still summed, and
                // the second's while the next tile's first has begun.
                const uint32_t acc_phase = units & 1;
                for (int kb = begin; kb < end && !failed;) {
                    const bool head = kb == begin;
                    const int left = end - kb, many = (int)stages;
                    const int run = head || left <= many ? (left < many ? left : many) : 1;
                    const bool last = left == run;
                    if (head && !barrier_wait(free_at, acc_phase ^ 1, p.polls)) { failed = true; break; }
                    uint32_t at = stage, at_phase = phase;
                    for (int i = 0; i < run; ++i) {
                        if (!barrier_wait(full + 8 * at, at_phase, p.polls)) { failed = true; break; }
                        tmem_after_sync();
                        issue(at, 0, head && i == 0);
                        if (++at == stages) { at = 0; at_phase ^= 1; }
                    }
                    if (failed) break;
                    if (last) {
                        commit(done);
                        ++ended_first;
                    }
                    if (head && !barrier_wait(free_at + 8, acc_phase ^ 1, p.polls)) { failed = true; break; }
                    tmem_after_sync();
                    for (int i = 0; i < run; ++i) {
                        issue(stage, 1, head && i == 0);
                        commit(empty + 8 * stage);
                        ++used;
                        if (++stage == stages) { stage = 0; phase ^= 1; }
                    }
                    if (last) {
                        commit(done + 8);
                        ++ended_second;
                    }
                    kb += run;
                }
                ++units;
            }
        }
        if (leader) {
#pragma unroll
            for (int cta = 0; cta < kCtas; ++cta) {
                leave(started.used, used, cta);
                leave(started.ended[0], ended_first, cta);
                leave(started.ended[1], ended_second, cta);
            }
        }
    } else if (warp >= 4) {
        // ---- ends (a lane quarter's warps share a tile's columns)
        const int share = (warp - 4) >> 2, quarter = warp & 3;
        const Way way(ring + ring_bytes(kEndWarps) + (uint32_t)(warp - 4) * kOutBytes, lane);      // (kLse and kLseOfOne send nothing)
        float scale = 1.0f;
        if constexpr (kEnd == kDlogits)
            if (p.positions > 0) {
                scale = weight_mantissa<kEndWarps>(p.dloss, p.target, p.positions, warp - 4);
                if (blockIdx.x == 0 && warp == 4 && lane == 0) *p.scale = scale;
            }
        if ((kEnd == kDlogits && p.positions == 0) || (kEnd == kStore && p.scale != nullptr)) scale = *p.scale;
        uint32_t units = 0;
        for (int w = first; w < p.total && !failed; w += step) {
            const Work t = work_of(p, w);
            Tile tile;
            tile.col = (int64_t)t.n_tile * p.cols;
            tile.width = p.n - tile.col < p.cols ? (int)(p.n - tile.col) : p.cols;
            tile.batch = t.outer >= p.splits;
            tile.sums = t.outer;
            tile.n_tile = t.n_tile;
            if constexpr (kEnd == kLse || kEnd == kLseOfOne || kEnd == kDlogits) {      // (read while the tile is being summed)
                const int64_t row = (int64_t)t.m_tile * 128 * kCtas + rank * 128 + quarter * 32 + lane;
                tile.of = row < p.m ? p.target[row] : -1;
                if constexpr (kEnd == kDlogits) {
                    tile.lse = row < p.m ? p.lse[row] : 0.0f;
                    tile.weight = row < p.m ? p.dloss[row] : 0.0f;
                }
            }
            const int runs = kEnd == kLse ? (p.kblocks + kLseRun - 1) / kLseRun : kHalves;
            Logits<kShare> logits;
            if constexpr (kEnd == kLse) logits.clear();
#pragma unroll 1
            for (int h = 0; h < runs; ++h, ++units) {
                const uint32_t acc = units & 1;
                // (tensor memory is read by whole warps: if one lane gave up, all do)
                if (!__all_sync(~0u, barrier_wait(done + 8 * acc, units >> 1 & 1, p.polls))) { failed = true; break; }
                __syncwarp();
                tmem_after_sync();
                tile.row0 = (int64_t)t.m_tile * 128 * kCtas * kHalves + (kHalves == 2 ? 256 * h : 0) + rank * 128 + quarter * 32;
                tile.row = tile.row0 + lane;
                tile.acc = tmem + acc * kAccColumns + ((uint32_t)quarter << 21);      // (lane 32 * quarter, in the upper half of the word)
                if constexpr (kEnd == kGated) end_gated(p, tile, share, way);
                if constexpr (kEnd == kLse) logits.take(tile, share);
                if constexpr (kEnd == kLseOfOne) end_lse_of_one<kShare>(p, tile, share);
                if constexpr (kEnd == kDlogits) end_dlogits<kShare>(p, tile, share, way, scale);
                if constexpr (kEnd == kStore) end_store<kShare>(p, tile, share, way, scale);
                __syncwarp();
                tmem_before_sync();
                if (lane == 0) barrier_arrive(peer_address(free_at + 8 * acc, 0));
            }
            if constexpr (kEnd == kLse)
                if (!failed) end_lse<kShare>(p, tile, share, logits);
        }
    }
    if (failed) {
        for (int cta = 0; cta < kCtas; ++cta) leave(started.failed, 1, cta);
        if (p.gave_up != nullptr) *reinterpret_cast<volatile uint32_t *>(p.gave_up) = 1;
    }
    auto meet = [&]() {
        __syncwarp();
        tmem_before_sync();
        if constexpr (kCtas == 2) cluster_sync();
        else __syncthreads();
        tmem_after_sync();
    };
    meet();
    if (*reinterpret_cast<volatile uint32_t *>(&started.failed) != 0) {
        settle<kCtas>(started, warp, rank, stages, full, empty, done, drained, p.polls);
        meet();
    }
    if (warp == 2) tmem_free<kCtas>(tmem, 2 * kAccColumns);
}

// ------------------------------------------------------------------ around the products
// Copies of up to three matrices, a thread for eight columns of a row: by words of two elements, shifted where the row starts on an odd
// one; single elements at a row's ends.
__device__ __forceinline__ uint4 eight_anywhere(const uint16_t *p, int64_t col, int64_t cols)
{
    uint32_t w[5];
    const int odd = (int)(reinterpret_cast<uintptr_t>(p) >> 1 & 1);
    if (col >= odd && col + 8 + odd <= cols) {
        const uint32_t *q = reinterpret_cast<const uint32_t *>(p - odd);
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = q[j];
        if (odd) {
            w[4] = q[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = __funnelshift_r(w[j], w[j + 1], 16);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t lo = col + 2 * j < cols ? p[2 * j] : 0, hi = col + 2 * j + 1 < cols ? p[2 * j + 1] : 0;
            w[j] = lo | hi << 16;
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__global__ void __launch_bounds__(256) realign_kernel(const Copies c)
{
    wait_for_the_one_before();
    for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < c.end[2]; i += gridDim.x * 256ll) {
        const int which = (i >= c.end[0]) + (i >= c.end[1]);
        const int64_t at = i - (which == 0 ? 0 : c.end[which - 1]), groups = (c.from[which].cols + 7) / 8;
        const int64_t row = at <= 0x7FFFFFFF ? (int64_t)((uint32_t)at / (uint32_t)groups) : at / groups, col = (at - row * groups) * 8;
        const Bf16Matrix &m = c.from[which];
        *reinterpret_cast<uint4 *>(c.to[which] + row * c.ld[which] + col) = eight_anywhere(m.p + row * m.ld + col, col, m.cols);
    }
}

// dgate and dup are rounded to bf16, because the products that follow multiply bf16: the gradients are 0.23 % off in the 2-norm where fp32 operands would
// leave the rounding of the result, 0.17 %, at two or three times the products.
// Eight columns a thread, two of them under way, where every row starts on a 16-byte boundary ...
template <int kAct>
__global__ void __launch_bounds__(256) gated_slopes_kernel(const Bf16Matrix dh, const Bf16Matrix gate, const Bf16Matrix up, uint16_t *dgate, uint16_t *dup,
                                                           int64_t ld, uint32_t groups, int64_t total)
{
    wait_for_the_one_before();
    const int64_t step = gridDim.x * 256ll;
    for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < total; i += 2 * step) {
        uint4 d[2], g[2], u[2];
        int64_t row[2];
        int col[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int64_t at = i + k * step;
            row[k] = total <= 0x7FFFFFFF ? (int64_t)((uint32_t)at / groups) : at / groups;
            col[k] = (int)(at - row[k] * groups) * 8;
            if (at < total) {
                d[k] = *reinterpret_cast<const uint4 *>(dh.p + row[k] * dh.ld + col[k]);
                g[k] = *reinterpret_cast<const uint4 *>(gate.p + row[k] * gate.ld + col[k]);
                u[k] = *reinterpret_cast<const uint4 *>(up.p + row[k] * up.ld + col[k]);
            }
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (i + k * step >= total) break;
            const uint32_t dw[4] = {d[k].x, d[k].y, d[k].z, d[k].w}, gw[4] = {g[k].x, g[k].y, g[k].z, g[k].w}, uw[4] = {u[k].x, u[k].y, u[k].z, u[k].w};
            uint32_t wg[4], wu[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const f32x2 d2 = widen2(dw[j]);
                f32x2 value, s;
                slope<kAct>(widen2(gw[j]), value, s);
                wg[j] = narrow2(mul2(mul2(d2, widen2(uw[j])), s));
                wu[j] = narrow2(mul2(d2, value));
            }
            *reinterpret_cast<uint4 *>(dgate + row[k] * ld + col[k]) = make_uint4(wg[0], wg[1], wg[2], wg[3]);
            *reinterpret_cast<uint4 *>(dup + row[k] * ld + col[k]) = make_uint4(wu[0], wu[1], wu[2], wu[3]);
        }
    }
}
// ... else single columns, a warp's side by side, eight runs of them under way.
template <int kAct>
__global__ void __launch_bounds__(128) gated_slopes_any_kernel(const Bf16Matrix dh, const Bf16Matrix gate, const Bf16Matrix up, uint16_t *dgate, uint16_t *dup,
                                                               int64_t ld)
{
    wait_for_the_one_before();
    for (int64_t row = blockIdx.y; row < dh.rows; row += gridDim.y)
        for (int64_t first = blockIdx.x * 1024ll + threadIdx.x; first < dh.cols; first += gridDim.x * 1024ll) {
            const int left = dh.cols - first < 1024 ? (int)(dh.cols - first) : 1024;
            const uint16_t *dp = dh.p + row * dh.ld + first, *gp = gate.p + row * gate.ld + first, *up_ = up.p + row * up.ld + first;
            uint16_t d[8], g[8], u[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                d[k] = g[k] = u[k] = 0;
                if (128 * k < left) {
                    d[k] = dp[128 * k];
                    g[k] = gp[128 * k];
                    u[k] = up_[128 * k];
                }
            }
            uint16_t *dg = dgate + row * ld + first, *du = dup + row * ld + first;
#pragma unroll
            for (int k = 0; k < 8; k += 2) {
                f32x2 value, s;
                slope<kAct>(pair(widen<uint16_t>(g[k]), widen<uint16_t>(g[k + 1])), value, s);
                const f32x2 d2 = pair(widen<uint16_t>(d[k]), widen<uint16_t>(d[k + 1]));
                const uint32_t wg = narrow2(mul2(mul2(d2, pair(widen<uint16_t>(u[k]), widen<uint16_t>(u[k + 1]))), s)), wu = narrow2(mul2(d2, value));
                if (128 * k < left) {
                    dg[128 * k] = (uint16_t)wg;
                    du[128 * k] = (uint16_t)wu;
                }
                if (128 * k + 128 < left) {
                    dg[128 * k + 128] = (uint16_t)(wg >> 16);
                    du[128 * k + 128] = (uint16_t)(wu >> 16);
                }
            }
        }
}

// The largest logit and the sum of exp(l - that) of two parts of a row.
__device__ __forceinline__ float2 join(float2 a, float2 b)
{
    const float top = fmaxf(a.x, b.x), base = top == -INFINITY ? 0.0f : top;
    return make_float2(top, a.y * power2((a.x - base) * kLog2e) + b.y * power2((b.x - base) * kLog2e));
}
__device__ __forceinline__ void finish_row(float2 v, int64_t row, float target_logit, const int64_t *target, int64_t vocab, float *lse, float *loss)
{
    const float l = v.x + logf(v.y);
    if (lse != nullptr) lse[row] = l;
    if (loss != nullptr) {
        const int64_t t = target[row];
        loss[row] = t < 0 ? 0.0f : t >= vocab ? NAN : l - target_logit;
    }
}

// `rows_a_cta` (a power of two up to 32) rows a CTA, 1024 / that threads for each: joined in a fixed order.
__global__ void __launch_bounds__(1024) lse_finish_kernel(const float2 *part, int n_part, int64_t rows, int rows_a_cta, const float *target_logit,
                                                          const int64_t *target, int64_t vocab, float *lse, float *loss)
{
    __shared__ float2 of[1024];
    wait_for_the_one_before();
    const int mine = threadIdx.x & (rows_a_cta - 1), lanes = 1024 / rows_a_cta, of_row = threadIdx.x / rows_a_cta;
    const int64_t row = (int64_t)blockIdx.x * rows_a_cta + mine;
    float2 v = make_float2(-INFINITY, 0.0f);
    if (row < rows)
        for (int i = of_row; i < n_part; i += lanes) v = join(v, part[(int64_t)i * rows + row]);
    of[threadIdx.x] = v;
    for (int n = lanes / 2; n >= 1; n /= 2) {
        __syncthreads();
        if (of_row < n) of[threadIdx.x] = v = join(v, of[threadIdx.x + n * rows_a_cta]);
    }
    if (of_row == 0 && row < rows) finish_row(v, row, target_logit[row], target, vocab, lse, loss);
}

// A thread for four columns; or, where there are many splits, kParts of them, which take every kParts-th split and are added in order.
template <int kParts>
__global__ void __launch_bounds__(256) sum_splits_kernel(const float *f32, int splits, int64_t rows, int64_t cols, int64_t f32_ld, uint16_t *out, int64_t out_ld,
                                                         const float *scale_of, int add)
{
    constexpr int kRuns = 256 / kParts;
    __shared__ float4 of[kParts][kRuns];
    const int64_t groups = (cols + 3) / 4;
    const int lane = threadIdx.x % kRuns, part = threadIdx.x / kRuns;
    wait_for_the_one_before();
    const float scale = scale_of != nullptr ? *scale_of : 1.0f;
    for (int64_t first = blockIdx.x * (int64_t)kRuns; first < groups * rows; first += gridDim.x * (int64_t)kRuns) {
        const int64_t i = first + lane, row = i / groups, col = (i - row * groups) * 4;
        float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (row < rows) {
#pragma unroll 4
            for (int j = part; j < splits; j += kParts) {
                const float4 v = *reinterpret_cast<const float4 *>(f32 + (j * rows + row) * f32_ld + col);
                s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
            }
        }
        if constexpr (kParts > 1) {
            of[part][lane] = s;
            __syncthreads();
            if (part == 0) {
#pragma unroll
                for (int j = 1; j < kParts; ++j) {
                    const float4 v = of[j][lane];
                    s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
                }
            }
        }
        if (part == 0 && row < rows) {
            uint16_t *o = out + row * out_ld + col;
            float v[4] = {s.x * scale, s.y * scale, s.z * scale, s.w * scale};
            if (add) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (col + j < cols) v[j] += widen<uint16_t>(o[j]);
            }
            const uint32_t w[2] = {narrow2(pair(v[0], v[1])), narrow2(pair(v[2], v[3]))};
            if (col + 4 <= cols && reinterpret_cast<uintptr_t>(o) % 8 == 0) {
                *reinterpret_cast<uint2 *>(o) = make_uint2(w[0], w[1]);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (col + j < cols) o[j] = (uint16_t)(w[j / 2] >> 16 * (j & 1));
            }
        }
        if constexpr (kParts > 1) __syncthreads();
    }
}

// ------------------------------------------------------------------ one row
// One row of A: a pass over both weights with nothing to fill a tile.  A warp takes two rows of gate and the same two of up, its
// lanes side by side in pieces of 16 bytes, the next 512 columns on their way while these are added; A lies in shared memory.
// Less to start and to drain than the tensor cores' kernel: 1 x 896 against 2 x 4864 rows 6.2 and 7.1 us a call, 256 against 2 x 512 3.4 and 4.2,
// 4096 against 2 x 11008 32.0 and 33.1 (2048 against 2 x 8192 12.2 and 11.3); with two rows there is nothing left of that.
struct RowArgs {
    const uint16_t *x, *w[2];
    int64_t w_ld[2], n;
    int k;
    uint16_t *h, *gate, *up;
    int act;
};
constexpr int kRowWarps = 8;

// 512 columns of four rows: two pieces of eight for each lane.  Beyond column k they are 0, as A is there.
struct RowPiece {
    uint4 w[4][2];
    __device__ __forceinline__ void read(const uint16_t *const (&row)[4], int c, int lane, int k)
    {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int col = c + 256 * h + lane * 8;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                w[r][h] = make_uint4(0, 0, 0, 0);
                if (col + 8 <= k) w[r][h] = __ldcs(reinterpret_cast<const uint4 *>(row[r] + col));
                else if (col < k) w[r][h] = some(row[r] + col, k - col);
            }
        }
    }
    static __device__ __noinline__ uint4 some(const uint16_t *p, int n)
    {
        uint32_t h[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = e < n ? p[e] : 0;
        return make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
    }
    __device__ __forceinline__ void add(uint32_t x_at, int c, f32x2 (&sum)[4]) const
    {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t x[4];
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(x_at + (uint32_t)(c + 256 * h) * 2u));
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const uint4 &q = w[r][h];
                    sum[r] = fma2(widen2(j == 0 ? q.x : j == 1 ? q.y : j == 2 ? q.z : q.w), widen2(x[j]), sum[r]);
                }
        }
    }
};

// Where a warp is: four rows and a run of 512 columns.
struct RowPlace {
    int64_t unit;
    int c;
    const uint16_t *row[4];
    __device__ __forceinline__ void go(const RowArgs &a, int64_t to)
    {
        unit = to;
        c = 0;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int64_t of = 2 * unit + (r >> 1), there = of < a.n ? of : a.n - 1;
            row[r] = a.w[r & 1] + there * a.w_ld[r & 1];
        }
    }
    __device__ __forceinline__ void next(const RowArgs &a, int64_t step)
    {
        c += 512;
        if (c >= a.k) go(a, unit + step);
    }
};

__global__ void __launch_bounds__(kRowWarps * 32, 2) gated_row_kernel(const RowArgs a)
{
    extern __shared__ uint4 row_shared[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, padded = (a.k + 511) / 512 * 512;
    const int64_t units = (a.n + 1) / 2, step = (int64_t)gridDim.x * kRowWarps;
    wait_for_the_one_before();
    RowPlace now, then;
    RowPiece piece[2];
    now.go(a, blockIdx.x * (int64_t)kRowWarps + warp);
    if (now.unit < units) piece[0].read(now.row, now.c, lane, a.k);
    for (int c = threadIdx.x * 8; c < padded; c += kRowWarps * 256) {
        uint4 q = make_uint4(0, 0, 0, 0);
        if (c < a.k) q = c + 8 <= a.k ? *reinterpret_cast<const uint4 *>(a.x + c) : RowPiece::some(a.x + c, a.k - c);
        row_shared[c / 8] = q;
    }
    __syncthreads();
    const uint32_t at = shared_address(row_shared) + lane * 16;
    f32x2 sum[4] = {both(0.0f), both(0.0f), both(0.0f), both(0.0f)};
    while (now.unit < units) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            then = now;
            then.next(a, step);
            if (then.unit < units) piece[i ^ 1].read(then.row, then.c, lane, a.k);
            piece[i].add(at, now.c, sum);
            if (then.unit != now.unit) {
                float v[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float2 f = halves(sum[r]);
                    v[r] = f.x + f.y;
                    sum[r] = both(0.0f);
#pragma unroll
                    for (int d = 16; d > 0; d >>= 1) v[r] += __shfl_xor_sync(~0u, v[r], d);
                }
                const float gate = lane == 0 ? v[0] : v[2], up = lane == 0 ? v[1] : v[3];
                const int64_t of = 2 * now.unit + lane;
                if (lane < 2 && of < a.n) {
                    by_activation(a.act, [&](auto act) { a.h[of] = narrow<uint16_t>(halves(activation<decltype(act)::value>(both(gate))).x * up); });
                    if (a.gate != nullptr) a.gate[of] = narrow<uint16_t>(gate);
                    if (a.up != nullptr) a.up[of] = narrow<uint16_t>(up);
                }
                __syncwarp();
            }
            now = then;
            if (now.unit >= units) break;
        }
    }
}

// ------------------------------------------------------------------ launches
using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                 const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled encoder()
{
    static std::atomic<void *> found{nullptr};
    void *f = found.load(std::memory_order_relaxed);
    if (f == nullptr) {
        cudaDriverEntryPointQueryResult how;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &how) != cudaSuccess || how != cudaDriverEntryPointSuccess) return nullptr;
        found.store(f, std::memory_order_relaxed);
    }
    return reinterpret_cast<EncodeTiled>(f);
}

// Boxes of 64 columns (128 bytes, the width of the swizzle) and so many rows.
cudaError_t encode(CUtensorMap *map, const Bf16Matrix &m, int box_rows)
{
    const EncodeTiled f = encoder();
    if (f == nullptr) return cudaErrorNotSupported;
    const cuuint64_t dims[2] = {(cuuint64_t)m.cols, (cuuint64_t)m.rows}, strides[1] = {(cuuint64_t)m.ld * 2};
    const cuuint32_t box[2] = {(cuuint32_t)kBlockK, (cuuint32_t)box_rows}, each[2] = {1, 1};
    const CUresult r = f(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<uint16_t *>(m.p), dims, strides, box, each, CU_TENSOR_MAP_INTERLEAVE_NONE,
                         CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

int grid_of(int64_t threads) { const int64_t n = (threads + 255) / 256; return (int)(n < 148 * 16 ? (n > 0 ? n : 1) : 148 * 16); }

Divider divider(int d)
{
    Divider r{(uint32_t)d, 0, 0};
    if (d > 1) {
        uint32_t up = 0;
        while ((1u << up) < (uint32_t)d) ++up;
        r.mul = (uint32_t)(((1ull << (31 + up)) + (uint32_t)d - 1) / (uint32_t)d);
        r.shift = up - 1;
    }
    return r;
}

}  // namespace

// How C is cut into tiles.  All units (CTAs, or pairs of them) take tiles in turn, so the time is that of the unit with the
// most, and a width is chosen that leaves the last round full: 517 rows against 32003 are 6 rounds of 3 x 126 tiles of 256 x 256, and 6 of
// 3 x 143 of 224 columns, which are shorter (53.3 and 52.2 us; 128 columns 68.8).  Clocks of a stage of 64 summed elements for 128 rows, from a product of
// 16384 x 4096 x 32000: 512 for 256 columns, 457 for 224, 421 for 192, 405 for 128, 302 for 64, 272 for 32; a single CTA, which brings in more bytes
// for its products, takes 25 % longer (517 rows: 77 and 52 us), two halves of 256 rows, which bring in fewer, 7 % less.  The other figures (the end of
// a tile, its turn, what a pair, sixteen warps and a split add) are those under which the choices lose the least against the fastest tiling of 248 products of
// up to 2.5e11 multiplications: 1.4 % on average.  Where they are large: 247 x 80 x 25292 13.5 us with 176 columns of a single CTA, 24 with 64 of a pair;
// dx of 700 x 640 x 1600 15.7 with 128 columns and four splits, 20.3 with 32 columns and none; a loss of 526 x 128 x 34071 19 with 256 columns, with 128 a third more.
Tiling product_tiling(ProductEnd end, bool bt, int64_t m, int64_t n, int64_t k, int segments, int batches, bool may_split, int sm_count)
{
    const int64_t stages = (k + kBlockK - 1) / kBlockK * segments;
    Tiling best;
    double least = 0.0;
    // (halves only where the end is short: that of the loss is not hidden behind them, 3.00 against 2.86 ms)
    for (int form = m > 256 && end == kStore ? 2 : m > 128 ? 1 : 0; form >= 0; --form) {
        const int ctas = form > 0 ? 2 : 1, halves = form == 2 ? 2 : 1, rows = 128 * ctas * halves;
        const double factor = form == 2 ? 0.93 : form == 1 ? 1.0 : 1.25;
        const int64_t tiles_m = (m + rows - 1) / rows, units = sm_count / ctas;
        // columns of C: the tensor cores take multiples of 16, of a pair of 32; kGated halves them
        const int step = ctas == 1 && end != kDlogits && end != kStore ? 16 : 32, widest = end == kGated ? 128 : 256;
        for (int cols = widest; cols >= step; cols -= step) {
            const int width = end == kGated ? 2 * cols : cols;
            const int64_t tiles_n = (n + cols - 1) / cols, tiles = tiles_m * tiles_n * batches;
            int64_t splits = 1, each = stages;
            if (may_split && tiles < units && stages >= 16) {
                splits = units / tiles < stages / 8 ? units / tiles : stages / 8;
                each = (stages + splits - 1) / splits;
            }
            const int64_t rounds = (tiles * splits + units - 1) / units;
            for (int end_warps = 8; end_warps <= 16; end_warps += 8) {
                if (end_warps == 16 && (end == kGated || halves == 2 || each > 8 || m <= 128)) continue;
                const double stage = (2.0 * width > 240.0 + width ? 2.0 * width : 240.0 + width) * factor, main = each * stage;
                const double store = 6.5 * (cols % 64 == 0 ? 1.0 : 1.5) * (end_warps == 16 ? 0.75 : 1.0) * width + 450.0;
                double cost = rounds * ((main > store ? main : store) + 200.0) * halves + store + (ctas == 2 ? 1500.0 : 0.0) + (end_warps == 16 ? 350.0 : 0.0);
                if (splits > 1) cost += 600.0 + (double)splits * batches * m * n * 8.0 / 2500.0;       // the sums of the splits, written and read
                if (least == 0.0 || cost < least) {
                    least = cost;
                    best = Tiling{ctas, halves, width, cols, (int)splits, end_warps, tiles_m, tiles_n};
                }
            }
        }
    }
    return best;
}
namespace {

template <int kCtas, int kHalves, bool kAT, bool kBT, int kEnd, int kEndWarps>
cudaError_t launch_product(const ProductArgs &a, int sm_count, cudaStream_t st)
{
    Params p{};
    const Tiling &t = a.tiling;
    const int maps_a = a.segments > 1 || a.batches > 1 ? 2 : 1, maps_b = kEnd == kGated || maps_a == 2 ? 2 : 1;
    const int rows_a = kAT || a.m > 128 ? 128 : (int)((a.m + 7) / 8 * 8);
    cudaError_t e = cudaSuccess;
    for (int i = 0; i < maps_a && e == cudaSuccess; ++i) e = encode(&p.a[i], a.a[i], kAT ? 64 : rows_a);
    for (int i = 0; i < maps_b && e == cudaSuccess; ++i) e = encode(&p.b[i], a.b[i], kBT ? 64 : kEnd == kGated ? t.cols : t.tile_n / kCtas);
    const int outs = kEnd == kGated ? 3 : kEnd == kDlogits ? 1 : kEnd == kStore ? a.batches : 0;
    for (int i = 0; i < outs; ++i) p.out[i] = Output{a.out[i], a.out_ld[i], tma_reads(Bf16Matrix{a.out[i], a.m, a.n, a.out_ld[i]})};
    if (e != cudaSuccess) return e;
    p.m = a.m; p.n = a.n;
    p.tile_n = t.tile_n; p.cols = t.cols;
    p.tiles_m = (int)t.tiles_m; p.tiles_n = (int)t.tiles_n;
    p.kblocks = (int)((a.k + kBlockK - 1) / kBlockK);
    p.all_k = p.kblocks * a.segments; p.splits = t.splits;
    p.each_k = p.all_k / t.splits; p.more_k = p.all_k % t.splits;
    const int64_t total = t.tiles_m * t.tiles_n * a.batches * t.splits;
    if (total > 0x3FFFFFFF || (t.tiles_m + 16) * t.tiles_n > 0x3FFFFFFF) return cudaErrorInvalidValue;
    p.total = (int)total;
    p.band = 16 / kHalves;
    const int last = p.tiles_m % p.band;
    p.by_outer = divider(p.tiles_m * p.tiles_n);
    p.by_band = divider(p.band * p.tiles_n);
    p.by_height = divider(p.band);
    p.by_last = divider(last == 0 ? p.band : last);
    // (a product reads 128 rows of A from the ring, also where A has fewer and other bytes follow: rows of C that nobody stores)
    p.bytes_a = rows_a * 128;
    p.bytes_b = (kBT ? (t.tile_n / kCtas + 63) / 64 * 64 : t.tile_n / kCtas) * 128;
    p.stages = (ring_bytes(kEndWarps) - (16384 - p.bytes_a)) / (kHalves * p.bytes_a + p.bytes_b);
    if (p.stages > kMostStages) p.stages = kMostStages;
    p.act = a.act;
    p.part = a.part; p.target_logit = a.target_logit; p.target = a.target; p.vocab = a.vocab; p.first = a.first;
    p.lse = a.lse; p.dloss = a.dloss; p.positions = a.positions; p.scale = a.scale;
    p.f32 = a.f32; p.f32_ld = a.f32_ld; p.mode = a.mode; p.gave_up = a.gave_up;
    // (the longest wait, for the sums of a tile, grows with the stages: about 0.3 us each)
    const int64_t polls = (int64_t)(1 << 22) + 8 * (int64_t)p.all_k;
    p.polls = a.polls != 0 ? a.polls : polls < 0xFFFFFFFF ? (uint32_t)polls : 0xFFFFFFFF;
    p.extra_bytes = a.extra_bytes;
    auto kernel = product_kernel<kCtas, kHalves, kAT, kBT, kEnd, kEndWarps>;
    static std::atomic<uint64_t> known{0};      // devices on which the kernel has its shared memory
    int device = 0;
    e = cudaGetDevice(&device);
    if (e == cudaSuccess && (device > 63 || !(known.load(std::memory_order_relaxed) >> device & 1))) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kShared);
        if (e == cudaSuccess && device <= 63) known.fetch_or(1ull << device, std::memory_order_relaxed);
    }
    if (e != cudaSuccess) return e;
    const int most = sm_count / kCtas, groups = p.total < most ? p.total : most;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(groups * kCtas));
    cfg.blockDim = dim3(32 * (4 + kEndWarps));
    cfg.dynamicSmemBytes = kShared;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = kCtas; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, p);
}

template <bool kAT, bool kBT, int kEnd>
cudaError_t launch_tiles(const ProductArgs &a, int sm_count, cudaStream_t st)
{
    if constexpr (kEnd == kStore)
        if (a.tiling.halves == 2) return launch_product<2, 2, kAT, kBT, kEnd, 8>(a, sm_count, st);
    // (kLse has more than eight stages a tile)
    if constexpr (kEnd != kGated && kEnd != kLse)
        if (a.tiling.end_warps == 16)
            return a.tiling.ctas == 2 ? launch_product<2, 1, kAT, kBT, kEnd, 16>(a, sm_count, st) : launch_product<1, 1, kAT, kBT, kEnd, 16>(a, sm_count, st);
    return a.tiling.ctas == 2 ? launch_product<2, 1, kAT, kBT, kEnd, 8>(a, sm_count, st) : launch_product<1, 1, kAT, kBT, kEnd, 8>(a, sm_count, st);
}

int64_t row_shared_bytes(int64_t k) { return (k + 511) / 512 * 512 * 2; }

}  // namespace

cudaError_t launch_product_rows(ProductEnd end, const ProductArgs &a, int sm_count, cudaStream_t st)
{
    if (end == kGated) return launch_tiles<false, false, kGated>(a, sm_count, st);
    if (end == kLse)
        return a.k <= kLseRun * kBlockK ? launch_tiles<false, false, kLseOfOne>(a, sm_count, st) : launch_tiles<false, false, kLse>(a, sm_count, st);
    if (end == kDlogits) return launch_tiles<false, false, kDlogits>(a, sm_count, st);
    return cudaErrorInvalidValue;
}
cudaError_t launch_product_drows(const ProductArgs &a, int sm_count, cudaStream_t st) { return launch_tiles<false, true, kStore>(a, sm_count, st); }
cudaError_t launch_product_dweight(const ProductArgs &a, int sm_count, cudaStream_t st) { return launch_tiles<true, true, kStore>(a, sm_count, st); }

bool tma_reads(const Bf16Matrix &m)
{
    return reinterpret_cast<uintptr_t>(m.p) % 16 == 0 && m.ld % 8 == 0;
}

cudaError_t launch_realign(Copies c, cudaStream_t st)
{
    int64_t n = 0;
    for (int i = 0; i < 3; ++i) {
        n += (c.from[i].cols + 7) / 8 * c.from[i].rows;
        c.end[i] = n;
    }
    return n == 0 ? cudaSuccess : launch_after(st, dim3(grid_of(n)), 256, 0, realign_kernel, c);
}

cudaError_t launch_lse_finish(const float2 *part, int n_part, int64_t rows, const float *target_logit, const int64_t *target, int64_t vocab, float *lse,
                              float *loss, cudaStream_t st)
{
    int each = 1;
    while (each < 32 && rows > 256 * each) each *= 2;
    return launch_after(st, dim3((unsigned)((rows + each - 1) / each)), 1024, 0, lse_finish_kernel, part, n_part, rows, each, target_logit, target, vocab, lse, loss);
}

cudaError_t launch_sum_splits(const float *f32, int splits, int64_t rows, int64_t cols, int64_t f32_ld, uint16_t *out, int64_t out_ld, const float *scale,
                              bool add, cudaStream_t st)
{
    const int64_t threads = (cols + 3) / 4 * rows;
    if (splits < 8) return launch_after(st, dim3(grid_of(threads)), 256, 0, sum_splits_kernel<1>, f32, splits, rows, cols, f32_ld, out, out_ld, scale, (int)add);
    return launch_after(st, dim3(grid_of(threads * 8)), 256, 0, sum_splits_kernel<8>, f32, splits, rows, cols, f32_ld, out, out_ld, scale, (int)add);
}

cudaError_t launch_gated_slopes(const Bf16Matrix &dh, const Bf16Matrix &gate, const Bf16Matrix &up, int act, uint16_t *dgate, uint16_t *dup, int64_t ld,
                                cudaStream_t st)
{
    auto go = [&](auto kernel, auto any) {
        if (dh.cols % 8 == 0 && tma_reads(dh) && tma_reads(gate) && tma_reads(up)) {
            const int64_t groups = dh.cols / 8, total = groups * dh.rows, want = (total + 511) / 512;
            return launch_after(st, dim3((unsigned)(want < 0x7FFFFFFF ? want : 0x7FFFFFFF)), 256, 0, kernel, dh, gate, up, dgate, dup, ld, (uint32_t)groups, total);
        }
        return launch_after(st, dim3((unsigned)((dh.cols + 1023) / 1024), (unsigned)(dh.rows < 65535 ? dh.rows : 65535)), 128, 0, any, dh, gate, up, dgate, dup, ld);
    };
    if (act == GG_ACT_SILU) return go(gated_slopes_kernel<GG_ACT_SILU>, gated_slopes_any_kernel<GG_ACT_SILU>);
    if (act == GG_ACT_GELU) return go(gated_slopes_kernel<GG_ACT_GELU>, gated_slopes_any_kernel<GG_ACT_GELU>);
    if (act == GG_ACT_GELU_TANH) return go(gated_slopes_kernel<GG_ACT_GELU_TANH>, gated_slopes_any_kernel<GG_ACT_GELU_TANH>);
    return go(gated_slopes_kernel<GG_ACT_RELU>, gated_slopes_any_kernel<GG_ACT_RELU>);
}

bool gated_row(int64_t m, int64_t k) { return m == 1 && row_shared_bytes(k) <= 48 * 1024; }

cudaError_t launch_gated_row(const ProductArgs &a, int sm_count, cudaStream_t st)
{
    RowArgs r{};
    r.x = a.a[0].p;
    for (int i = 0; i < 2; ++i) {
        r.w[i] = a.b[i].p;
        r.w_ld[i] = a.b[i].ld;
    }
    r.n = a.n; r.k = (int)a.k;
    r.h = a.out[0]; r.gate = a.out[1]; r.up = a.out[2];
    r.act = a.act;
    // two CTAs an SM, or a unit of work for each warp
    const int64_t want = (a.n + 2 * kRowWarps - 1) / (2 * kRowWarps), most = 2 * (int64_t)sm_count;
    return launch_after(st, dim3((unsigned)(want < most ? want : most)), kRowWarps * 32, (size_t)row_shared_bytes(a.k), gated_row_kernel, r);
}

}  // namespace gg
