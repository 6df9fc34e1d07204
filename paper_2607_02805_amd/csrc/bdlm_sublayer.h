// bdlm_sublayer.h -- internal interface between the entry points at a sublayer's entry
// (bdlm_sublayer_api.cpp) and their HIP kernels (bdlm_addnorm.hip).  Plain C++; no HIP types.
#pragma once

#include <stdint.h>

#include "bdlm.h"

namespace bdlm {

constexpr int32_t kScaleBlock = 128;   // columns of an 8-bit output that share a scale, unless a row does

// y = w s / sqrt(mean s^2 + eps), s = x + residual.
struct AddNormArgs {
    const void *x, *residual;      // residual may be null
    void *sum, *out;               // sum may be null
    const float *w;
    float *scale;                  // of 8 bits: [rows][1, or blocks of kScaleBlock columns]
    int64_t ldx, ldr, lds, ldo;
    int32_t rows, width;
    int32_t x_bf16, res_bf16;      // (sum as residual)
    int32_t out_dtype;             // enum bdlm_dtype
    int32_t blocks;                // scales of a row: 1, or one for each kScaleBlock columns
    int32_t by_block;
    float eps;
};
int launch_add_norm(const AddNormArgs &a, void *stream);

// ds = rstd (w dy - n mean(n w dy)) + dsum, n = s rstd; dw = sum over the rows of dy n.
struct AddNormGradArgs {
    const void *dy, *s, *dsum;     // dsum may be null
    void *ds;                      // may be null
    const float *w;
    float *part;                   // [add_norm_grad_blocks][width], or null: dw is not wanted
    int64_t ldy, lds, ldt, ldd;    // of dy, s, dsum, ds
    int32_t rows, width;
    int32_t dy_bf16, s_bf16, ds_bf16;   // (dsum as ds)
    float eps;
};
int launch_add_norm_grad(const AddNormGradArgs &a, void *stream);
// Workgroups of the gradient with dw, each with a row of partial sums of it.
int32_t add_norm_grad_blocks(int64_t rows, int64_t width);

}  // namespace bdlm
