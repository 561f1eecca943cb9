// Matrix products of the training operators on the tensor cores: the gated block, the vocabulary loss, their gradients.
//
// One kernel, C = A B^T in bf16 with fp32 sums, and four ends for its tiles (ProductEnd): the operators differ in what becomes
// of a tile while it is still in tensor memory, so neither the logits nor the two projections need a pass of their own.
// A persistent CTA (or pair of CTAs, each with half of A's and half of B's rows of a shared 256 x 256 tile) takes tiles in turn.
// One thread copies the operands into a ring of stages of 64 summed elements by TMA, which also fills what lies beyond a matrix
// with zeros, so no size is special; one thread feeds the tensor cores; eight warps end the tile before the last, which
// lies in the other half of tensor memory.
#include <cuda.h>
#include <math.h>

#include <atomic>
#include <type_traits>

#include "gg.h"
#include "gg_element.cuh"
#include "gg_products.cuh"
#include "gg_tensor.cuh"

namespace gg {
namespace {

constexpr int kBlockK = 64;             // summed elements of a stage: 128 bytes, a row of the swizzle
constexpr int kEndWarps = 8, kThreads = 32 * (4 + kEndWarps);
constexpr int kRing = 192 * 1024;       // bytes of the ring of stages
constexpr int kBand = 8;                // tiles of C that are taken in bands of so many rows, so that B's stay in L2
constexpr float kLog2e = 1.4426950408889634f;

struct Params {
    CUtensorMap a[2], b[2];
    int64_t m, n;
    int tiles_m, tiles_n, total, kblocks, segments, batches, splits;
    uint16_t *h, *gate, *up;
    int64_t h_ld, gate_ld, up_ld;
    int act, h_align, gate_align, up_align;
    float2 *part;
    float *target_logit;
    const int64_t *target;
    int64_t vocab, first;
    const float *lse, *dloss;
    uint16_t *out[2];
    int64_t out_ld[2];
    int out_align;
    float *f32;
    int64_t f32_ld;
    int mode;
    uint32_t *gave_up;
};

// ------------------------------------------------------------------ activations
// a / (1 + e^-a): an e^-a that overflows gives 0, as the product does.
__device__ __forceinline__ float sigmoid(float a) { return __fdividef(1.0f, 1.0f + __expf(-a)); }
template <int kAct>
__device__ __forceinline__ float activation(float a)
{
    if constexpr (kAct == GG_ACT_SILU) return a * sigmoid(a);
    if constexpr (kAct == GG_ACT_GELU) return 0.5f * a * erfcf(-0.70710678118654752f * a);      // (erfc: 1 + erf cancels)
    if constexpr (kAct == GG_ACT_GELU_TANH) {           // (1 + tanh z) / 2 = sigmoid(2 z), which is 0 or 1 beyond 30
        const float b = fminf(fmaxf(a, -30.0f), 30.0f);
        return a * sigmoid(1.5957691216057308f * (b + 0.044715f * b * b * b));
    }
    return a > 0.0f ? a : (a != a ? a : 0.0f);
}
// act(a) and its derivative
template <int kAct>
__device__ __forceinline__ void slope(float a, float &value, float &d)
{
    if constexpr (kAct == GG_ACT_SILU) {
        const float s = sigmoid(a);
        value = a * s;
        d = s + value * (1.0f - s);
    } else if constexpr (kAct == GG_ACT_GELU) {
        const float c = 0.5f * erfcf(-0.70710678118654752f * a);
        value = a * c;
        d = c + a * 0.3989422804014327f * __expf(-0.5f * a * a);
    } else if constexpr (kAct == GG_ACT_GELU_TANH) {
        const float b = fminf(fmaxf(a, -30.0f), 30.0f), s = sigmoid(1.5957691216057308f * (b + 0.044715f * b * b * b));
        value = a * s;
        d = s + value * (1.0f - s) * 1.5957691216057308f * (1.0f + 0.134145f * b * b);
    } else {
        value = activation<GG_ACT_RELU>(a);
        d = a > 0.0f ? 1.0f : (a != a ? a : 0.0f);
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

// ------------------------------------------------------------------ rows of 32 columns
__device__ __forceinline__ uint32_t narrow_pair(float lo, float hi) { return narrow2(pair(lo, hi)); }

// The first n of 32 bf16 values to p, which is on a boundary of `align` bytes.
__device__ __forceinline__ void store_row(uint16_t *p, const uint32_t (&w)[16], int64_t n, int align)
{
    if (n >= 32 && align >= 32) {
#pragma unroll
        for (int i = 0; i < 16; i += 8)
            asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p + 2 * i), "r"(w[i]), "r"(w[i + 1]), "r"(w[i + 2]), "r"(w[i + 3]),
                         "r"(w[i + 4]), "r"(w[i + 5]), "r"(w[i + 6]), "r"(w[i + 7]) : "memory");
    } else if (n >= 32 && align >= 16) {
#pragma unroll
        for (int i = 0; i < 16; i += 4) *reinterpret_cast<uint4 *>(p + 2 * i) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
    } else {
#pragma unroll
        for (int i = 0; i < 32; ++i)
            if (i < n) p[i] = (uint16_t)(w[i / 2] >> 16 * (i & 1));
    }
}
__device__ __forceinline__ void narrow_row(const float (&v)[32], uint32_t (&w)[16])
{
#pragma unroll
    for (int i = 0; i < 16; ++i) w[i] = narrow_pair(v[2 * i], v[2 * i + 1]);
}

// ------------------------------------------------------------------ the ends of a tile
struct Tile {
    int64_t row;         // of this thread
    int64_t col;         // first column of the tile
    int batch, split, n_tile;
};

// kN columns of the tile, of which a warp has the half that `half` says; `at` is the accumulator of the warp's lanes.
template <int kN>
__device__ __forceinline__ void end_gated(const Params &p, const Tile &t, uint32_t at, int half)
{
    constexpr int kMine = kN / 4;        // columns of h for a warp
    const bool there = t.row < p.m;
#pragma unroll 1
    for (int c = half * kMine; c < (half + 1) * kMine; c += 32) {
        float g[32], u[32];
        tmem_read(at + c, g);
        tmem_read(at + kN / 2 + c, u);
        tmem_read_wait();
        const int64_t col = t.col + c, left = there ? p.n - col : 0;
        if (left > 0) {
            uint32_t w[16];
            if (p.gate != nullptr) {
                narrow_row(g, w);
                store_row(p.gate + t.row * p.gate_ld + col, w, left, p.gate_align);
            }
            if (p.up != nullptr) {
                narrow_row(u, w);
                store_row(p.up + t.row * p.up_ld + col, w, left, p.up_align);
            }
            by_activation(p.act, [&](auto act) {
#pragma unroll
                for (int i = 0; i < 32; ++i) g[i] = activation<decltype(act)::value>(g[i]) * u[i];
            });
            narrow_row(g, w);
            store_row(p.h + t.row * p.h_ld + col, w, left, p.h_align);
        }
        __syncwarp();
    }
}

// The sum is taken relative to the running maximum.  A NaN, which no maximum shows, reaches the sum by its own term.
template <int kN>
__device__ __forceinline__ void end_lse(const Params &p, const Tile &t, uint32_t at, int half)
{
    constexpr int kMine = kN / 2;
    const bool there = t.row < p.m;
    const int64_t target = there ? p.target[t.row] - p.first : -1;
    float most = -INFINITY, sum = 0.0f;
#pragma unroll 1
    for (int c = half * kMine; c < (half + 1) * kMine; c += 32) {
        float v[32];
        tmem_read(at + c, v);
        tmem_read_wait();
        const int64_t col = t.col + c, left = p.n - col;
        if (target >= col && target < col + 32 && target < p.n) {
            const int j = (int)(target - col);
            float l = 0.0f;
#pragma unroll
            for (int i = 0; i < 32; ++i) l = i == j ? v[i] : l;
            p.target_logit[t.row] = l;
        }
        if (left < 32) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = i < left ? v[i] : -INFINITY;
        }
        float top = most;
#pragma unroll
        for (int i = 0; i < 32; ++i) top = fmaxf(top, v[i]);
        const float base = top == -INFINITY ? 0.0f : top;
        float s0 = sum * exp2f((most - base) * kLog2e), s1 = 0.0f;
#pragma unroll
        for (int i = 0; i < 32; i += 2) {
            s0 += exp2f((v[i] - base) * kLog2e);
            s1 += exp2f((v[i + 1] - base) * kLog2e);
        }
        sum = s0 + s1;
        most = top;
        __syncwarp();
    }
    if (there) p.part[(int64_t)(2 * t.n_tile + half) * p.m + t.row] = make_float2(most, sum);
}

template <int kN>
__device__ __forceinline__ void end_dlogits(const Params &p, const Tile &t, uint32_t at, int half)
{
    constexpr int kMine = kN / 2;
    const bool there = t.row < p.m;
    const int64_t of = there ? p.target[t.row] : -1, target = of - p.first;
    const float lse = there ? p.lse[t.row] : 0.0f, g = of < 0 ? 0.0f : of >= p.vocab ? NAN : p.dloss[t.row];
#pragma unroll 1
    for (int c = half * kMine; c < (half + 1) * kMine; c += 32) {
        float v[32];
        tmem_read(at + c, v);
        tmem_read_wait();
        const int64_t col = t.col + c;
        if (there && col < p.n) {
            uint32_t w[16];
            if (of < 0) {              // no position, whatever its logits are
#pragma unroll
                for (int i = 0; i < 16; ++i) w[i] = 0;
            } else {
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] = g * exp2f((v[i] - lse) * kLog2e);
                if (target >= col && target < col + 32) {
                    const int j = (int)(target - col);
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] = i == j ? v[i] - g : v[i];
                }
                narrow_row(v, w);
            }
            store_row(p.out[0] + t.row * p.out_ld[0] + col, w, 32, 32);      // (a row has room for whole runs of 32)
        }
        __syncwarp();
    }
}

__device__ __forceinline__ void store_part(const Params &p, const Tile &t, float (&v)[32], int64_t col, int64_t left)
{
    if (p.mode != kStoreBf16 && p.mode != kAddBf16) {
        float4 *f = reinterpret_cast<float4 *>(p.f32 + ((int64_t)t.split * p.m + t.row) * p.f32_ld + col);
        if (p.mode != kStoreF32) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float4 o = f[i];
                v[4 * i] += o.x; v[4 * i + 1] += o.y; v[4 * i + 2] += o.z; v[4 * i + 3] += o.w;
            }
        }
        if (p.mode != kStoreBf16OfSum) {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
            return;
        }
    }
    uint16_t *o = p.out[t.batch] + t.row * p.out_ld[t.batch] + col;
    if (p.mode == kAddBf16) {
        if (left >= 32 && p.out_align >= 16) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint4 q = reinterpret_cast<const uint4 *>(o)[i];
                const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 f = halves(widen2(w[j]));
                    v[8 * i + 2 * j] += f.x;
                    v[8 * i + 2 * j + 1] += f.y;
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (i < left) v[i] += widen<uint16_t>(o[i]);
        }
    }
    uint32_t w[16];
    narrow_row(v, w);
    store_row(o, w, left, p.out_align);
}

template <int kN>
__device__ __forceinline__ void end_store(const Params &p, const Tile &t, uint32_t at, int half)
{
    constexpr int kMine = kN / 2;
    const bool there = t.row < p.m;
#pragma unroll 1
    for (int c = half * kMine; c < (half + 1) * kMine; c += 32) {
        float v[32];
        tmem_read(at + c, v);
        tmem_read_wait();
        const int64_t col = t.col + c, left = there ? p.n - col : 0;
        if (left > 0) store_part(p, t, v, col, left);
        __syncwarp();
    }
}

// ------------------------------------------------------------------ the kernel
struct Work { int m_tile, n_tile, outer; };
__device__ __forceinline__ Work work_of(const Params &p, int w)
{
    const int each = p.tiles_m * p.tiles_n;
    Work r;
    r.outer = w / each;
    w -= r.outer * each;
    const int band = w / (kBand * p.tiles_n), first = band * kBand;
    const int height = p.tiles_m - first < kBand ? p.tiles_m - first : kBand;
    w -= first * p.tiles_n;
    r.n_tile = w / height;
    r.m_tile = first + (w - r.n_tile * height);
    return r;
}

template <int kCtas, int kN, bool kAT, bool kBT, int kEnd>
__global__ void __launch_bounds__(kThreads, 1) product_kernel(const __grid_constant__ Params p)
{
    constexpr int kRowsB = kN / kCtas;                    // rows of B that a CTA brings in
    constexpr uint32_t kBytesA = 128 * kBlockK * 2, kBytes = kBytesA + kRowsB * kBlockK * 2;
    constexpr int kStages = kRing / kBytes;
    constexpr uint32_t kColumns = 2 * kN;                 // of tensor memory: two accumulators
    extern __shared__ uint8_t ring_bytes[];
    __shared__ uint64_t bars[2 * kStages + 5];
    __shared__ uint32_t tmem_at;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = kCtas == 2 ? cluster_rank() : 0;
    const uint32_t ring = (shared_address(ring_bytes) + 1023) & ~1023u;
    const uint32_t bar = shared_address(bars);
    const uint32_t full = bar, empty = bar + 8 * kStages, done = bar + 16 * kStages, free_at = done + 16, drained = done + 32;

    if (warp == 0 && lane == 0) {
        for (int i = 0; i < kStages; ++i) {
            barrier_init(full + 8 * i, 1);
            barrier_init(empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            barrier_init(done + 8 * i, 1);
            barrier_init(free_at + 8 * i, kEndWarps * kCtas);
        }
        barrier_init(drained, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        prefetch_map(&p.a[0]);
        prefetch_map(&p.b[0]);
    }
    if (warp == 2) tmem_alloc<kCtas>(shared_address(&tmem_at), kColumns);
    tmem_before_sync();
    if constexpr (kCtas == 2) cluster_sync();
    else __syncthreads();
    tmem_after_sync();
    const uint32_t tmem = tmem_at;

    const int first = blockIdx.x / kCtas, step = gridDim.x / kCtas, all_k = p.kblocks * p.segments;
    bool failed = false;
    if (warp == 0 && lane == 0) {
        // ---- copies
        uint32_t stage = 0, phase = 0, issued = 0;
        for (int w = first; w < p.total && !failed; w += step) {
            const Work t = work_of(p, w);
            const int batch = p.batches > 1 ? t.outer : 0, split = p.batches > 1 ? 0 : t.outer;
            const int m0 = t.m_tile * 128 * kCtas + (int)rank * 128;
            const int n0 = kEnd == kGated ? t.n_tile * (kN / 2) : t.n_tile * kN + (int)rank * kRowsB;
            const int end = (int)((int64_t)all_k * (split + 1) / p.splits);
            for (int kb = (int)((int64_t)all_k * split / p.splits); kb < end; ++kb) {
                if (!barrier_wait(empty + 8 * stage, phase ^ 1)) { failed = true; break; }
                if (rank == 0) barrier_expect(full + 8 * stage, kBytes * kCtas);
                const int segment = kb >= p.kblocks, k0 = (kb - segment * p.kblocks) * kBlockK, which = segment | batch;
                const uint32_t to_a = ring + stage * kBytes, to_b = to_a + kBytesA;
                const uint32_t signal = kCtas == 2 ? peer_address(full + 8 * stage, 0) : full + 8 * stage;
                if constexpr (kAT) {
                    tensor_copy<kCtas>(to_a, &p.a[which], m0, k0, signal);
                    tensor_copy<kCtas>(to_a + 8192, &p.a[which], m0 + 64, k0, signal);
                } else {
                    tensor_copy<kCtas>(to_a, &p.a[which], k0, m0, signal);
                }
                if constexpr (kBT) {
#pragma unroll
                    for (int i = 0; i < kRowsB / 64; ++i) tensor_copy<kCtas>(to_b + 8192 * i, &p.b[which], n0 + 64 * i, k0, signal);
                } else if constexpr (kEnd == kGated && kCtas == 1) {
                    tensor_copy<kCtas>(to_b, &p.b[0], k0, n0, signal);
                    tensor_copy<kCtas>(to_b + kRowsB / 2 * kBlockK * 2, &p.b[1], k0, n0, signal);
                } else if constexpr (kEnd == kGated) {
                    tensor_copy<kCtas>(to_b, &p.b[rank], k0, n0, signal);
                } else {
                    tensor_copy<kCtas>(to_b, &p.b[which], k0, n0, signal);
                }
                ++issued;
                if (++stage == kStages) { stage = 0; phase ^= 1; }
            }
        }
        // what is still under way when a wait gave up has to land before the CTA may end
        if (failed && rank == 0)
            for (uint32_t i = 0; i < kStages && i < issued; ++i) {
                stage = stage == 0 ? kStages - 1 : stage - 1;
                if (stage == kStages - 1) phase ^= 1;
                barrier_wait(full + 8 * stage, phase);
            }
    } else if (warp == 1 && lane == 0 && rank == 0) {
        // ---- products
        constexpr uint32_t shape = product_shape<128 * kCtas, kN, kAT, kBT>();
        uint32_t stage = 0, phase = 0, acc = 0, acc_phase = 0;
        for (int w = first; w < p.total && !failed; w += step) {
            const int split = p.batches > 1 ? 0 : work_of(p, w).outer;
            if (!barrier_wait(free_at + 8 * acc, acc_phase ^ 1)) { failed = true; break; }
            tmem_after_sync();
            const int begin = (int)((int64_t)all_k * split / p.splits), end = (int)((int64_t)all_k * (split + 1) / p.splits);
            for (int kb = begin; kb < end; ++kb) {
                if (!barrier_wait(full + 8 * stage, phase)) { failed = true; break; }
                tmem_after_sync();
                const uint64_t a = tile_descriptor<kAT>(ring + stage * kBytes), b = tile_descriptor<kBT>(ring + stage * kBytes + kBytesA);
#pragma unroll
                for (int i = 0; i < kBlockK / 16; ++i)
                    product_issue<kCtas>(tmem + acc * kN, a + i * tile_step<kAT>(), b + i * tile_step<kBT>(), shape, kb > begin || i > 0);
                product_commit<kCtas>(empty + 8 * stage);
                if (++stage == kStages) { stage = 0; phase ^= 1; }
            }
            if (failed) break;
            product_commit<kCtas>(done + 8 * acc);
            acc ^= 1;
            acc_phase ^= acc == 0;
        }
        if (failed) {
            product_commit<kCtas>(drained);
            barrier_wait(drained, 0);
        }
    } else if (warp >= 4) {
        // ---- ends
        const int half = (warp - 4) >> 2, quarter = warp & 3;
        uint32_t acc = 0, acc_phase = 0;
        for (int w = first; w < p.total; w += step) {
            const Work t = work_of(p, w);
            if (!barrier_wait(done + 8 * acc, acc_phase)) { failed = true; break; }
            tmem_after_sync();
            Tile tile;
            tile.row = (int64_t)t.m_tile * 128 * kCtas + rank * 128 + quarter * 32 + lane;
            tile.col = (int64_t)t.n_tile * (kEnd == kGated ? kN / 2 : kN);
            tile.batch = p.batches > 1 ? t.outer : 0;
            tile.split = p.batches > 1 ? 0 : t.outer;
            tile.n_tile = t.n_tile;
            const uint32_t at = tmem + acc * kN + ((uint32_t)quarter << 21);      // (lane 32 * quarter, in the upper half of the word)
            if constexpr (kEnd == kGated) end_gated<kN>(p, tile, at, half);
            if constexpr (kEnd == kLse) end_lse<kN>(p, tile, at, half);
            if constexpr (kEnd == kDlogits) end_dlogits<kN>(p, tile, at, half);
            if constexpr (kEnd == kStore) end_store<kN>(p, tile, at, half);
            __syncwarp();
            tmem_before_sync();
            if (lane == 0) barrier_arrive(peer_address(free_at + 8 * acc, 0));
            acc ^= 1;
            acc_phase ^= acc == 0;
        }
    }
    if (failed && p.gave_up != nullptr) *reinterpret_cast<volatile uint32_t *>(p.gave_up) = 1;
    __syncwarp();
    tmem_before_sync();
    if constexpr (kCtas == 2) cluster_sync();
    else __syncthreads();
    tmem_after_sync();
    if (warp == 2) tmem_free<kCtas>(tmem, kColumns);
}

// ------------------------------------------------------------------ around the products
// One thread for eight columns of a row.
__global__ void __launch_bounds__(256) realign_kernel(const Bf16Matrix from, uint16_t *to, int64_t ld, int64_t groups)
{
    for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < groups * from.rows; i += gridDim.x * 256ll) {
        const int64_t row = i / groups, col = (i - row * groups) * 8;
        const uint16_t *f = from.p + row * from.ld + col;
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t lo = col + 2 * j < from.cols ? f[2 * j] : 0, hi = col + 2 * j + 1 < from.cols ? f[2 * j + 1] : 0;
            w[j] = lo | hi << 16;
        }
        *reinterpret_cast<uint4 *>(to + row * ld + col) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

__device__ __forceinline__ void eight_of(const Bf16Matrix &m, int64_t row, int64_t col, bool vector, float (&v)[8])
{
    const uint16_t *p = m.p + row * m.ld + col;
    if (vector) {
        const uint4 q = *reinterpret_cast<const uint4 *>(p);
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = halves(widen2(w[i]));
            v[2 * i] = f.x;
            v[2 * i + 1] = f.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = col + i < m.cols ? widen<uint16_t>(p[i]) : 0.0f;
    }
}

template <int kAct>
__global__ void __launch_bounds__(256) gated_slopes_kernel(const Bf16Matrix dh, const Bf16Matrix gate, const Bf16Matrix up, uint16_t *dgate, uint16_t *dup,
                                                           int64_t ld, int64_t groups, int vector)
{
    for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < groups * dh.rows; i += gridDim.x * 256ll) {
        const int64_t row = i / groups, col = (i - row * groups) * 8;
        const bool whole = vector && col + 8 <= dh.cols;
        float d[8], g[8], u[8];
        eight_of(dh, row, col, whole, d);
        eight_of(gate, row, col, whole, g);
        eight_of(up, row, col, whole, u);
        uint32_t wg[4], wu[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float v0, v1, s0, s1;
            slope<kAct>(g[2 * j], v0, s0);
            slope<kAct>(g[2 * j + 1], v1, s1);
            wg[j] = narrow_pair(d[2 * j] * u[2 * j] * s0, d[2 * j + 1] * u[2 * j + 1] * s1);
            wu[j] = narrow_pair(d[2 * j] * v0, d[2 * j + 1] * v1);
        }
        *reinterpret_cast<uint4 *>(dgate + row * ld + col) = make_uint4(wg[0], wg[1], wg[2], wg[3]);
        *reinterpret_cast<uint4 *>(dup + row * ld + col) = make_uint4(wu[0], wu[1], wu[2], wu[3]);
    }
}

// 32 rows a CTA, a warp for every 32nd partial of each; the warps' results are joined in their order.
__global__ void __launch_bounds__(1024) lse_finish_kernel(const float2 *part, int n_part, int64_t rows, const float *target_logit, const int64_t *target,
                                                          int64_t vocab, float *lse, float *loss)
{
    __shared__ float2 of[32][33];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t row = blockIdx.x * 32ll + lane;
    auto join = [](float2 a, float2 b) {
        const float top = fmaxf(a.x, b.x), base = top == -INFINITY ? 0.0f : top;
        return make_float2(top, a.y * exp2f((a.x - base) * kLog2e) + b.y * exp2f((b.x - base) * kLog2e));
    };
    float2 v = make_float2(-INFINITY, 0.0f);
    if (row < rows)
        for (int i = warp; i < n_part; i += 32) v = join(v, part[(int64_t)i * rows + row]);
    of[warp][lane] = v;
    __syncthreads();
    // (a warp has a row now, its lanes the 32 parts)
    v = of[lane][warp];
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const float2 o = make_float2(__shfl_xor_sync(~0u, v.x, d), __shfl_xor_sync(~0u, v.y, d));
        v = lane & d ? join(o, v) : join(v, o);
    }
    const int64_t r = blockIdx.x * 32ll + warp;
    if (lane == 0 && r < rows) {
        const float l = v.x + logf(v.y);
        if (lse != nullptr) lse[r] = l;
        if (loss != nullptr) {
            const int64_t t = target[r];
            loss[r] = t < 0 ? 0.0f : t >= vocab ? NAN : l - target_logit[r];
        }
    }
}

__global__ void __launch_bounds__(256) sum_splits_kernel(const float *f32, int splits, int64_t rows, int64_t cols, int64_t f32_ld, uint16_t *out, int64_t out_ld)
{
    const int64_t groups = (cols + 3) / 4;
    for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < groups * rows; i += gridDim.x * 256ll) {
        const int64_t row = i / groups, col = (i - row * groups) * 4;
        float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int j = 0; j < splits; ++j) {
            const float4 v = *reinterpret_cast<const float4 *>(f32 + (j * rows + row) * f32_ld + col);
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
        const float v[4] = {s.x, s.y, s.z, s.w};
        uint16_t *o = out + row * out_ld + col;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (col + j < cols) o[j] = narrow<uint16_t>(v[j]);
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

// Bytes of which both the address and every row's start are multiples, as far as stores care.
int row_align(const void *p, int64_t ld, int esize)
{
    const uint64_t both = reinterpret_cast<uintptr_t>(p) | (uint64_t)(ld * esize);
    return both % 32 == 0 ? 32 : both % 16 == 0 ? 16 : esize;
}

int grid_of(int64_t threads) { const int64_t n = (threads + 255) / 256; return (int)(n < 148 * 16 ? (n > 0 ? n : 1) : 148 * 16); }

template <int kCtas, int kN, bool kAT, bool kBT, int kEnd>
cudaError_t launch_product(const ProductArgs &a, int sm_count, cudaStream_t st)
{
    Params p{};
    constexpr int kColumns = kEnd == kGated ? kN / 2 : kN;
    const int maps_a = a.segments > 1 || a.batches > 1 ? 2 : 1, maps_b = kEnd == kGated || maps_a == 2 ? 2 : 1;
    cudaError_t e = cudaSuccess;
    for (int i = 0; i < maps_a && e == cudaSuccess; ++i) e = encode(&p.a[i], a.a[i], kAT ? 64 : 128);
    for (int i = 0; i < maps_b && e == cudaSuccess; ++i) e = encode(&p.b[i], a.b[i], kBT ? 64 : kEnd == kGated && kCtas == 1 ? kN / 2 : kN / kCtas);
    if (e != cudaSuccess) return e;
    p.m = a.m; p.n = a.n;
    p.tiles_m = (int)((a.m + 128 * kCtas - 1) / (128 * kCtas));
    p.tiles_n = (int)((a.n + kColumns - 1) / kColumns);
    p.kblocks = (int)((a.k + kBlockK - 1) / kBlockK);
    p.segments = a.segments; p.batches = a.batches; p.splits = a.splits;
    const int64_t total = (int64_t)p.tiles_m * p.tiles_n * a.batches * a.splits;
    if (total > 0x3FFFFFFF) return cudaErrorInvalidValue;
    p.total = (int)total;
    p.h = a.h; p.gate = a.gate; p.up = a.up;
    p.h_ld = a.h_ld; p.gate_ld = a.gate_ld; p.up_ld = a.up_ld;
    p.act = a.act;
    p.h_align = row_align(a.h, a.h_ld, 2); p.gate_align = row_align(a.gate, a.gate_ld, 2); p.up_align = row_align(a.up, a.up_ld, 2);
    p.part = a.part; p.target_logit = a.target_logit; p.target = a.target; p.vocab = a.vocab; p.first = a.first;
    p.lse = a.lse; p.dloss = a.dloss;
    p.out_align = 32;
    for (int i = 0; i < a.batches; ++i) {
        p.out[i] = a.out[i]; p.out_ld[i] = a.out_ld[i];
        const int align = row_align(a.out[i], a.out_ld[i], 2);
        p.out_align = align < p.out_align ? align : p.out_align;
    }
    p.f32 = a.f32; p.f32_ld = a.f32_ld; p.mode = a.mode; p.gave_up = a.gave_up;
    auto kernel = product_kernel<kCtas, kN, kAT, kBT, kEnd>;
    constexpr int kShared = kRing + 1024;
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
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kShared;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = kCtas; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, p);
}

constexpr int kTileN = 256;      // columns of C in a tile
// Two CTAs for a tile of 256 rows, where there are more than one CTA's.
int ctas_of(int64_t m) { return m > 128 ? 2 : 1; }

template <bool kAT, bool kBT, int kEnd>
cudaError_t launch_tiles(const ProductArgs &a, int sm_count, cudaStream_t st)
{
    return ctas_of(a.m) == 2 ? launch_product<2, kTileN, kAT, kBT, kEnd>(a, sm_count, st) : launch_product<1, kTileN, kAT, kBT, kEnd>(a, sm_count, st);
}

}  // namespace

cudaError_t launch_product_rows(ProductEnd end, const ProductArgs &a, int sm_count, cudaStream_t st)
{
    if (end == kGated) return launch_tiles<false, false, kGated>(a, sm_count, st);
    if (end == kLse) return launch_tiles<false, false, kLse>(a, sm_count, st);
    if (end == kDlogits) return launch_tiles<false, false, kDlogits>(a, sm_count, st);
    return cudaErrorInvalidValue;
}
cudaError_t launch_product_drows(const ProductArgs &a, int sm_count, cudaStream_t st) { return launch_tiles<false, true, kStore>(a, sm_count, st); }
cudaError_t launch_product_dweight(const ProductArgs &a, int sm_count, cudaStream_t st) { return launch_tiles<true, true, kStore>(a, sm_count, st); }

int product_partials(int64_t, int64_t n) { return (int)(2 * ((n + kTileN - 1) / kTileN)); }

int product_splits(int64_t m, int64_t n, int64_t k, int segments, int sm_count)
{
    // as many as give every SM a tile, but at least 16 stages for each
    const int64_t ctas = ctas_of(m), tiles = ((m + 128 * ctas - 1) / (128 * ctas)) * ((n + kTileN - 1) / kTileN);
    const int64_t most = (k + kBlockK - 1) / kBlockK * segments / 16, want = sm_count / ctas / (tiles > 0 ? tiles : 1);
    const int64_t s = want < most ? want : most;
    return (int)(s < 1 ? 1 : s);
}

bool tma_reads(const Bf16Matrix &m)
{
    return reinterpret_cast<uintptr_t>(m.p) % 16 == 0 && m.ld % 8 == 0;
}

cudaError_t launch_realign(const Bf16Matrix &from, uint16_t *to, int64_t ld, cudaStream_t st)
{
    const int64_t groups = (from.cols + 7) / 8;
    realign_kernel<<<grid_of(groups * from.rows), 256, 0, st>>>(from, to, ld, groups);
    return cudaGetLastError();
}

cudaError_t launch_lse_finish(const float2 *part, int n_part, int64_t rows, const float *target_logit, const int64_t *target, int64_t vocab, float *lse,
                              float *loss, cudaStream_t st)
{
    lse_finish_kernel<<<(unsigned)((rows + 31) / 32), 1024, 0, st>>>(part, n_part, rows, target_logit, target, vocab, lse, loss);
    return cudaGetLastError();
}

cudaError_t launch_sum_splits(const float *f32, int splits, int64_t rows, int64_t cols, int64_t f32_ld, uint16_t *out, int64_t out_ld, cudaStream_t st)
{
    sum_splits_kernel<<<grid_of((cols + 3) / 4 * rows), 256, 0, st>>>(f32, splits, rows, cols, f32_ld, out, out_ld);
    return cudaGetLastError();
}

cudaError_t launch_gated_slopes(const Bf16Matrix &dh, const Bf16Matrix &gate, const Bf16Matrix &up, int act, uint16_t *dgate, uint16_t *dup, int64_t ld,
                                cudaStream_t st)
{
    const int64_t groups = (dh.cols + 7) / 8;
    const int grid = grid_of(groups * dh.rows), vector = tma_reads(dh) && tma_reads(gate) && tma_reads(up);
    auto go = [&](auto kernel) { kernel<<<grid, 256, 0, st>>>(dh, gate, up, dgate, dup, ld, groups, vector); };
    if (act == GG_ACT_SILU) go(gated_slopes_kernel<GG_ACT_SILU>);
    else if (act == GG_ACT_GELU) go(gated_slopes_kernel<GG_ACT_GELU>);
    else if (act == GG_ACT_GELU_TANH) go(gated_slopes_kernel<GG_ACT_GELU_TANH>);
    else go(gated_slopes_kernel<GG_ACT_RELU>);
    return cudaGetLastError();
}

}  // namespace gg
