// bdlm_dense.h -- internal interface between the entry points of the dense operators
// (bdlm_dense_api.cpp: projections, the vocabulary loss, token selection) and their HIP kernels
// (bdlm_tile.hip, bdlm_skinny.hip, bdlm_dense.hip).  Plain C++; no HIP types.
//
// All products are of bf16 terms accumulated in fp32 on the matrix cores.  An fp32 operand is
// three bf16 terms (v = hi + mid + lo, 24 bits; split_terms in bdlm_dense_device.h), stored as
// three planes, and a product of two such operands is the six plane products of weight 2^-16 or
// more: what is left out is about 2^-25 of |a||b|, below fp32's own rounding.  The fp32 matrix
// rate is a sixteenth of the bf16 one, so six bf16 products are 2.7 times faster than one in fp32.
#pragma once

#include <stdint.h>

#include "bdlm.h"

namespace bdlm {

// A matrix of bf16 terms: element (row, col) of term p at p * plane + row * ld + col.
struct Mat {
    const uint16_t *p;
    int64_t ld, plane;
};

// What becomes of a tile of products acc[row][col].
enum TileOut {
    kTileStore = 0,    // v = act(acc + bias) + residual -> out
    kTilePartial = 1,  // fp32 partial sums, one slice per split (added onto what is there, if asked)
    kTileBest = 2,     // per row: the tile's largest value, its column, the others' sum of exps
    kTileProb = 3      // gradient of the loss by the logits, in bf16 terms
};

// Store: the epilogue of a projection (also applied by the join of partial sums).
struct StoreArgs {
    void *out;
    const float *bias;         // [ncol] or null
    const void *residual;      // like out, or null
    void *pre;                 // acc + bias, or null
    int64_t ld_out, ld_res, ld_pre;
    int32_t out_bf16, pre_bf16;
    int32_t act;
    const int32_t *row_of;     // row r goes to row row_of[r] of out (null: r)
};

// One record per (row, column tile): largest value, sum over the others of exp(v - largest).
struct BestArgs {
    float *top, *others;       // [nrow][ntile]
    int32_t *at;               // [nrow][ntile] column of the largest (lowest of equals)
    float *label_logit;        // [nrow]: written where label[row] is met (null: no labels)
    const int32_t *label;      // [nrow]
    int32_t ntile, exclude;
};

// Of one bf16 term, a row of the logits' gradients is divided by its label's entry: that one, which
// outweighs the others, is 1 and loses nothing.  The divisor (RowsArgs' scale) multiplies dx's row in
// fp32, and x's row, rounded to bf16 element by element, in dw's product.  (Rounded as it
// was, the label's entry put one error on a whole row of dx: 0.0028 over a few rows with
// large weights, where the rounding of dx itself is 0.0017.)
struct ProbArgs {
    uint16_t *p;               // [terms][nrow][ld]
    int64_t ld, plane;
    int32_t terms;             // 1, 2 or 3
    const float *lse, *loss, *weight;   // [nrow]
    const int32_t *label;      // [nrow], counted from column 0 of the vocabulary
    int32_t exclude, col0;     // col0: the vocabulary column of the call's column 0
    int32_t width;             // columns of p to be written (zeros past ncol)
};

// acc[row][col] = sum over k of row(row, k) * col(col, k), over `npair` pairs of planes.
// The operand of `row` is [nrow][k] (or [k][nrow] if row_t), of `col` [ncol][k] ([k][ncol] if
// col_t).  Operands are read in 16-byte pieces, 64 contraction indices at a time: ld a multiple of
// 8, bases 16-byte aligned, rows readable up to a multiple of 8 columns; an operand whose
// contraction index is contiguous holds zeros from k to the next multiple of 64, and if both
// operands' is the slow one, `row` holds rows of zeros up to a multiple of 64.
struct TileArgs {
    Mat row, col;
    int32_t nrow, ncol, k;
    const int32_t *nrow_dev, *k_dev;   // the count in device memory, at most nrow / k (null: nrow / k)
    int32_t npair;                     // pairs of planes: 1, 2 (two terms of row) or 6 (three of each)
    int32_t row_t, col_t;
    int32_t skip;                      // a contraction index at which col is not read, below k - 1 (col_t;
                                       // row holds zeros there), or -1
    int32_t big;                       // 1: 256 x 256 tiles, 0: 128 x 128
    int32_t splits;                    // > 1: kTilePartial only; 0: as many as fill the chip with
                                       // the rows that count (split_count)
    int32_t add;                       // kTilePartial: add onto the slices
    float *part;                       // [splits][nrow][ncol]; splits 0: [split_count][nrow counted][ncol]
    int32_t out;                       // TileOut
    StoreArgs store;
    BestArgs best;
    ProbArgs prob;
};
int launch_tile(const TileArgs &a, void *stream);
constexpr int32_t kChip = 256;   // workgroups of large tiles that run at once
constexpr int32_t kMostSplits = 16;
// Splits of a product whose row count is known on the device alone, by its tiles.
#ifdef __HIPCC__
__host__ __device__
#endif
inline int32_t split_count(int64_t tiles) {
    const int64_t s = tiles > 0 ? kChip / tiles : 1;
    return static_cast<int32_t>(s < 1 ? 1 : s > kMostSplits ? kMostSplits : s);
}
constexpr int32_t kTileThreads = 512;   // of a workgroup, whatever its tile
// Columns of a tile (what kTileBest's ntile counts).
inline int32_t tile_edge(bool big) { return big ? 256 : 128; }

// out = epilogue(sum of the partial slices); splits 0: as many as a tiled product of these sizes
// made (big: its tiles)
// scale: a factor of every row, or null
int launch_join(const float *part, int32_t splits, int32_t big, int32_t nrow, int32_t ncol, const int32_t *nrow_dev,
                const float *scale, const StoreArgs &s, void *stream);

// Few rows (skinny_rows): the weights stream through once.  x [nrow][k], w [ncol][k], both bf16
// or both fp32, any stride; out kTileStore or kTileBest (one record per skinny_cols columns).
struct SkinnyArgs {
    const void *x, *w;
    int64_t ldx, ldw;
    int32_t nrow, ncol, k;
    const int32_t *nrow_dev, *row_of;  // the rows that count: how many, and row r's row of x (null: all)
    int32_t bf16;
    int32_t out;
    StoreArgs store;
    BestArgs best;
};
// Above that many rows the tiles are faster: over 50,257 columns of 1,024 in bf16, 32 rows take 34
// us here and 29 there, 64 rows 54 and 34, but over 4,384 of them 32 rows take 9 and 11; in fp32,
// where the tiles lay the weights out anew, 64 rows take 110 and 215.  One limit for every width: it costs the widest
// calls of nearly 32 bf16 rows a sixth and saves the narrow ones as much.
inline int32_t skinny_rows(bool bf16) { return bf16 ? 32 : 64; }
// Columns of a workgroup: fewer where there are not two workgroups for every CU.
inline int32_t skinny_cols(int64_t ncol) { return ncol >= 32 * 512 ? 32 : 16; }
int launch_skinny(const SkinnyArgs &a, void *stream);

// Copies an operand to bf16 terms: dst[p][r][0 .. ld_dst) from row r of src (row_of: row row_of[r]),
// zeros past its columns, and rows of zeros up to a multiple of 64.
struct PackArgs {
    const void *src;
    int64_t ld;
    int32_t rows, cols, src_bf16;
    const int32_t *rows_dev, *row_of;
    const float *scale;        // factors of the rows laid out (a bf16 copy of one term), or null
    uint16_t *dst;
    int64_t ld_dst, plane;
    int32_t terms;
    // gradient of a projection's activation: src is dy, dst = dy * act'(pre)
    int32_t act;
    const void *pre;
    int64_t ld_pre;
    int32_t pre_bf16;
    float *colsum;             // [pack_row_blocks(rows)][cols] partial column sums of dst, or null
};
int launch_pack(const PackArgs &a, void *stream);
constexpr int32_t kPackRows = 16;   // rows per workgroup
#ifdef __HIPCC__
__host__ __device__
#endif
inline int32_t pack_row_blocks(int32_t rows) { return (rows + 63) / 64 * (64 / kPackRows); }
// out[c] = sum over the blocks of part[b][c]
int launch_colsum(const float *part, int32_t blocks, int32_t cols, float *out, void *stream);

// The rows that count: row_of[0 .. *count) the rows whose label is a token of the vocabulary
// other than `exclude`, in order; label[i] that token, and (if given) weight, loss, lse by row.
struct RowsArgs {
    const int64_t *labels;
    int32_t rows, vocab;
    int64_t exclude;
    int32_t *count, *row_of, *label;
    const float *dloss, *loss, *lse;     // null in the forward call
    float *weight_c, *loss_c, *lse_c, *scale_c;   // scale: the gradient by the label's logit
};
int launch_rows(const RowsArgs &a, void *stream);

// Merges the tiles' records.  Loss: loss and lse of the rows that count (row_of), zeros for
// the others; select: token and log-probability.
struct FinishArgs {
    const float *top, *others;
    const int32_t *at;
    int32_t ntile, rows, vocab, exclude;
    const int32_t *count, *row_of;
    const int64_t *labels;               // loss
    const float *label_logit;
    float *loss, *lse;
    int64_t *token;                      // select
    float *logprob;
};
int launch_finish(const FinishArgs &a, void *stream);

// Zeros the rows of dx (bytes per row a multiple of the element) whose label does not count.
int launch_zero_rows(const int64_t *labels, int64_t exclude, int32_t vocab, int32_t rows, void *dx,
                     int64_t ld, int32_t cols, int32_t bf16, void *stream);

}  // namespace bdlm
