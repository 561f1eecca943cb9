// Tables and constants that the host side of the AdamW step passes to its kernel (not installed).
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "gg.h"

namespace gg {

constexpr int kBlock = GG_ADAMW_BLOCK;      // elements that share one scale of an 8-bit state
constexpr int kStepWarps = 4;               // warps of a CTA
constexpr int kTableSmall = 64, kTableLarge = 512;      // (multiples of 64)

// The tensors of one launch, passed by value: kernel parameters may take 32,764 bytes, which holds 512 tensors.  A
// step so needs no device memory of its own, no upload and no cache, whatever addresses the tensors have this time.
// Two sizes: a launch with up to 4 KB of parameters costs the host 2.7 us, one with 30 KB 5.5 us (and 4 us more until
// the kernel has ended), so up to 64 tensors take the small table.
struct StepEntry {
    void *w;
    const void *g;
    void *m, *v, *copy;
    int64_t len;
    int32_t block0;            // first scale of the tensor (8-bit states)
    int32_t id;                // its place in the caller's list; bit 31: every array starts where Eight wants it
};
template <int N>
struct StepTable {
    int32_t tile0[N];          // first tile of each tensor; beyond the last, INT32_MAX
    StepEntry entry[N];
    int32_t n, tiles;
    int32_t per_warp;          // (at most 32) blocks of a tensor that one warp steps, one after the other; a tile is kStepWarps times that
};
constexpr int32_t kAligned = (int32_t)0x80000000;
static_assert(sizeof(StepTable<512>) <= 32 * 1024 - 512 && sizeof(StepTable<64>) <= 4096 - 224, "the table and the scalars have to fit the kernel parameters");

struct StepScalars {
    const float *grad_scale;       // device, or null
    const float *decay;            // device [n_seg], or null: decay_all
    float *m_scale, *v_scale;      // device, 8-bit states
    // each twice, as the two halves of a pair
    float2 b1, one_b1, b2, one_b2;
    float2 step;                   // -lr / (1 - b1^t)
    float2 root;                   // 1 / sqrt(1 - b2^t)
    float2 eps;
    float lr, decay_all;
    uint32_t t;
    uint32_t key[20];              // the key of each round of Philox: seed mod 2^32 + r * W0, seed div 2^32 + r * W1
};

cudaError_t launch_adamw(const StepTable<kTableSmall> &tab, const StepScalars &c, int w_dtype, int g_dtype, bool narrow_states, cudaStream_t st);
cudaError_t launch_adamw(const StepTable<kTableLarge> &tab, const StepScalars &c, int w_dtype, int g_dtype, bool narrow_states, cudaStream_t st);
cudaError_t launch_grad_norm(const double *s2, const uint32_t *bad, int32_t n_tiles, double max_norm, double *norm, float *scale, cudaStream_t st);

}  // namespace gg
