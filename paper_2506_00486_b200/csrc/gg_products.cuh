// Matrix products of the training operators on the tensor cores (gg_products.cu), as the host side calls them (not installed).
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace gg {

// A row-major bf16 matrix: `ld` elements from row to row.
struct Bf16Matrix {
    const uint16_t *p;
    int64_t rows, cols, ld;
};

// What becomes of a tile of the product C = A B^T, fp32 in tensor memory.
enum ProductEnd : int {
    kGated,       // columns of two products side by side: h = act(gate) * up, and both of them if they are wanted
    kLse,         // the largest logit of a row in half a tile of the vocabulary and the sum of exp(l - that)
    kDlogits,     // g * (exp(l - lse) - [v is the target]) in bf16
    kStore,       // C itself
};
// kStore: bf16, bf16 added to what is there, fp32 (one matrix for each split of the long axis), fp32 added to what is
// there, bf16 of the sum with the fp32 that is there.
enum StoreMode : int { kStoreBf16, kAddBf16, kStoreF32, kAddF32, kStoreBf16OfSum };

// How C is cut into tiles (product_tiling): CTAs of a tile, its halves, rows of B and columns of C in it, splits of the long axis,
// warps that end it.
struct Tiling {
    int ctas, halves, tile_n, cols, splits, end_warps;
    int64_t parts() const { return end_warps / 4 * tiles_n; }      // of a row, that kLse leaves
    int64_t tiles_m, tiles_n;
};

struct ProductArgs {
    // C[m, n] = sum over the segments of A B^T.  K-major operands are [m or n, k] matrices, the others [k, m or n].
    Bf16Matrix a[2], b[2];      // of a segment, or of a batch (one of the two); kGated: b[0] gate, b[1] up
    int64_t m, n, k;            // kGated: n counts the columns of h
    int segments, batches;
    Tiling tiling;
    int act;                    // kGated
    // kLse: [end_warps / 4 * tiles_n][m] partials; target[m], the logits of the targets.  kDlogits: target, lse, dloss, out.
    float2 *part;
    float *target_logit;
    const int64_t *target;
    int64_t vocab;              // targets count from 0 to vocab - 1 ...
    int64_t first;              // ... and this call's columns begin there
    const float *lse, *dloss;
    int64_t positions;          // entries of target and dloss to look for `scale` in (0: it is there)
    float *scale;               // what kDlogits' numbers are relative to: it leaves it here, kStore multiplies its sums by it (null: 1)
    // kGated: h, gate, up (each of the last two may be null); kDlogits: out[0]; kStore: of a batch
    uint16_t *out[3];
    int64_t out_ld[3];
    float *f32;                 // kStore: [batches][splits][m][f32_ld], f32_ld a multiple of 32
    int64_t f32_ld;
    int mode;
    uint32_t *gave_up;          // host-visible word: set if a wait inside the kernel ran out
    uint32_t polls;             // after which one does (0: the default)
    uint32_t extra_bytes;       // test hook: bytes a stage expects beyond what is copied (the waits then run out)
};

// C = A B^T with both operands K-major ...
cudaError_t launch_product_rows(ProductEnd end, const ProductArgs &a, int sm_count, cudaStream_t st);
// ... with A K-major and B [k, n] (the gradient of the rows), and with A [k, m] and B [k, n] (that of a weight); kStore
cudaError_t launch_product_drows(const ProductArgs &a, int sm_count, cudaStream_t st);
cudaError_t launch_product_dweight(const ProductArgs &a, int sm_count, cudaStream_t st);
// The cut that leaves least to wait for; bt: B is [k, n].  With may_split the long axis may be cut too (kStoreF32 then).
Tiling product_tiling(ProductEnd end, bool bt, int64_t m, int64_t n, int64_t k, int segments, int batches, bool may_split, int sm_count);
// kGated for a single row, without the tensor cores
bool gated_row(int64_t m, int64_t k);
cudaError_t launch_gated_row(const ProductArgs &a, int sm_count, cudaStream_t st);

// Can TMA read the matrix where it is?  If not, launch_realign copies it (up to three in one launch) to rows of `ld` elements, a multiple
// of 8; what a row has beyond the matrix becomes 0.
bool tma_reads(const Bf16Matrix &m);
struct Copies {
    Bf16Matrix from[3];         // (rows 0: none)
    uint16_t *to[3];
    int64_t ld[3];
    int64_t end[3];             // (set by launch_realign)
};
cudaError_t launch_realign(Copies c, cudaStream_t st);

// lse and loss of a row from its partials; a negative target has loss 0, one beyond the vocabulary NaN
cudaError_t launch_lse_finish(const float2 *part, int n_part, int64_t rows, const float *target_logit, const int64_t *target, int64_t vocab, float *lse,
                              float *loss, cudaStream_t st);
// out = bf16 of the sum of `splits` fp32 matrices (scale as in ProductArgs), and of what is there with `add`
cudaError_t launch_sum_splits(const float *f32, int splits, int64_t rows, int64_t cols, int64_t f32_ld, uint16_t *out, int64_t out_ld, const float *scale,
                              bool add, cudaStream_t st);
// dgate = dh * up * act'(gate), dup = dh * act(gate)
cudaError_t launch_gated_slopes(const Bf16Matrix &dh, const Bf16Matrix &gate, const Bf16Matrix &up, int act, uint16_t *dgate, uint16_t *dup, int64_t ld,
                                cudaStream_t st);

}  // namespace gg
