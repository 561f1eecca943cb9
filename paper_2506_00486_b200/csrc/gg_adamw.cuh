// Tables and constants that the host side of the AdamW step passes to its kernel (not installed).
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "gg.h"

namespace gg {

constexpr int kBlock = GG_ADAMW_BLOCK;      // elements that share one scale of an 8-bit state
constexpr int kTileBlocks = 16;             // blocks of a CTA: 4096 elements
constexpr int kTableSmall = 16, kTableLarge = 512;

// The tensors of one launch, passed by value: kernel parameters may take 32,764 bytes, which holds 512 tensors.  A
// step so needs no device memory of its own, no upload and no cache, whatever addresses the tensors have this time.
template <int N>
struct StepTable {
    void *w[N];
    const void *g[N];
    void *m[N], *v[N], *copy[N];
    int64_t len[N];
    int32_t tile0[N + 1];      // first tile of each tensor; [n]: the number of tiles
    int32_t block0[N];         // first scale of each tensor (8-bit states)
    int32_t id[N];             // its place in the caller's list; bit 31: every array starts where Eight wants it
    int32_t n;
};
constexpr int32_t kAligned = (int32_t)0x80000000;
static_assert(sizeof(StepTable<512>) <= 32 * 1024 - 256, "the table and the scalars have to fit the kernel parameters");

struct StepScalars {
    const float *grad_scale;       // device, or null
    const float *decay;            // device [n_seg], or null: decay_all
    float *m_scale, *v_scale;      // device, 8-bit states
    float b1, one_b1, b2, one_b2, lr, decay_all;
    float step;                    // lr / (1 - b1^t)
    float root;                    // 1 / sqrt(1 - b2^t)
    float eps;
    uint32_t t, seed_lo, seed_hi;
};

cudaError_t launch_adamw(const StepTable<kTableSmall> &tab, const StepScalars &c, int w_dtype, int g_dtype, bool narrow_states, cudaStream_t st);
cudaError_t launch_adamw(const StepTable<kTableLarge> &tab, const StepScalars &c, int w_dtype, int g_dtype, bool narrow_states, cudaStream_t st);
cudaError_t launch_grad_norm(const double *s2, const uint32_t *bad, int32_t n_tiles, double max_norm, double *norm, float *scale, cudaStream_t st);

}  // namespace gg
