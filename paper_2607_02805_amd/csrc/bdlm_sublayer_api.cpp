// bdlm_sublayer_api.cpp -- the C ABI of the operators of a sublayer (include/bdlm.h): the norm at its entry, with
// the residual's addition, and its gradient.  Argument checks, workspaces and launches.
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "bdlm.h"
#include "bdlm_dense.h"
#include "bdlm_dense_plan.h"
#include "bdlm_sublayer.h"

namespace {

int64_t size_of(int32_t dt) { return dt == BDLM_DTYPE_F32 ? 4 : dt == BDLM_DTYPE_BF16 ? 2 : 1; }

int check_norm(int64_t rows, int64_t width, const float *norm_w, float eps) {
    if (rows < 0 || width <= 0 || rows > kMaxSize || width > kMaxSize) return BDLM_E_SHAPE;
    if (!(eps >= 0.f) || !std::isfinite(eps)) return BDLM_E_SHAPE;
    if (rows > 0 && !norm_w) return BDLM_E_NULL;
    return aligned(norm_w, 16) ? BDLM_OK : BDLM_E_ALIGN;
}
// An input matrix and its stride.
int check_rows(const void *p, int64_t rows, int64_t ld) {
    TRY(check_in(p, rows));
    return ld < 0 || ld > kMaxStride ? BDLM_E_SHAPE : BDLM_OK;
}
int64_t scales_of(int64_t width, int64_t block) { return block ? (width + block - 1) / block : 1; }

int64_t norm_space(int64_t rows, int64_t width) {
    return up(int64_t(bdlm::add_norm_grad_blocks(rows, width)) * width * 4, 256);
}

}  // namespace

extern "C" {

int bdlm_check_add_rmsnorm(int64_t rows, int64_t width, int32_t x_dtype, const void *x, int64_t x_stride,
                           int32_t residual_dtype, const void *residual, int64_t residual_stride, const void *sum,
                           int64_t sum_stride, const float *norm_w, float eps, int32_t out_dtype, const void *out,
                           int64_t out_stride, const float *scale, int64_t scale_block) {
    if (!known(x_dtype) || (residual && !known(residual_dtype)) || (!known(out_dtype) && out_dtype != BDLM_DTYPE_E4M3))
        return BDLM_E_DTYPE;
    const bool e4m3 = out_dtype == BDLM_DTYPE_E4M3;
    TRY(check_norm(rows, width, norm_w, eps));
    if (scale_block != 0 && (!e4m3 || scale_block != kScaleBlock)) return BDLM_E_SHAPE;
    TRY(check_rows(x, rows, x_stride));
    if (residual) TRY(check_rows(residual, rows, residual_stride));
    if (sum && !residual) return BDLM_E_NULL;
    if (sum) TRY(check_out(sum, rows, width, sum_stride));
    TRY(check_out(out, rows, width, out_stride));
    if (e4m3 && rows > 0 && !scale) return BDLM_E_NULL;
    if (!aligned(scale, 4)) return BDLM_E_ALIGN;
    const int64_t ex = size_of(x_dtype), er = residual ? size_of(residual_dtype) : 0;
    const Span sx(x, rows, width, x_stride, ex), sr(residual, rows, width, residual_stride, er),
        ss(sum, rows, width, sum_stride, er), sw(norm_w, 1, width, 0, 4),
        so(out, rows, width, out_stride, size_of(out_dtype)),
        sc(e4m3 ? scale : nullptr, 1, rows * scales_of(width, scale_block), 0, 4);
    // (each element is read by the lane that writes it)
    const bool stream_in_place = sum && sum == residual && sum_stride == residual_stride;
    const bool x_in_place = out == x && out_stride == x_stride && out_dtype == x_dtype;
    if ((!x_in_place && so.meets(sx)) || (!stream_in_place && ss.meets(sr))) return BDLM_E_SHAPE;
    if (!apart(so, sr, ss, sw, sc) || !apart(ss, sx, sw, sc) || !apart(sc, sx, sr, sw)) return BDLM_E_SHAPE;
    return BDLM_OK;
}

int bdlm_add_rmsnorm(int64_t rows, int64_t width, int32_t x_dtype, const void *x, int64_t x_stride,
                     int32_t residual_dtype, const void *residual, int64_t residual_stride, void *sum,
                     int64_t sum_stride, const float *norm_w, float eps, int32_t out_dtype, void *out,
                     int64_t out_stride, float *scale, int64_t scale_block, void *stream) {
    TRY(bdlm_check_add_rmsnorm(rows, width, x_dtype, x, x_stride, residual_dtype, residual, residual_stride, sum,
                               sum_stride, norm_w, eps, out_dtype, out, out_stride, scale, scale_block));
    AddNormArgs a{};
    a.x = x;
    a.residual = residual;
    a.sum = sum;
    a.out = out;
    a.w = norm_w;
    a.scale = scale;
    a.ldx = x_stride;
    a.ldr = residual_stride;
    a.lds = sum_stride;
    a.ldo = out_stride;
    a.rows = static_cast<int32_t>(rows);
    a.width = static_cast<int32_t>(width);
    a.x_bf16 = x_dtype == BDLM_DTYPE_BF16;
    a.res_bf16 = residual_dtype == BDLM_DTYPE_BF16;
    a.out_dtype = out_dtype;
    a.blocks = static_cast<int32_t>(scales_of(width, scale_block));
    a.by_block = scale_block != 0;
    a.eps = eps;
    return launch_add_norm(a, stream);
}

int bdlm_add_rmsnorm_backward_workspace(int64_t rows, int64_t width, int64_t *bytes) {
    if (rows < 0 || width <= 0 || rows > kMaxSize || width > kMaxSize) return BDLM_E_SHAPE;
    if (!bytes) return BDLM_E_NULL;
    *bytes = norm_space(rows, width);
    return BDLM_OK;
}

int bdlm_check_add_rmsnorm_backward(int64_t rows, int64_t width, int32_t dy_dtype, const void *dy, int64_t dy_stride,
                                    int32_t s_dtype, const void *s, int64_t s_stride, const float *norm_w, float eps,
                                    int32_t ds_dtype, const void *dsum, int64_t dsum_stride, const void *ds,
                                    int64_t ds_stride, const float *dw, const void *ws, int64_t ws_bytes) {
    if (!known(dy_dtype) || !known(s_dtype) || !known(ds_dtype)) return BDLM_E_DTYPE;
    TRY(check_norm(rows, width, norm_w, eps));
    TRY(check_rows(dy, rows, dy_stride));
    TRY(check_rows(s, rows, s_stride));
    if (dsum) TRY(check_rows(dsum, rows, dsum_stride));
    if (ds) TRY(check_out(ds, rows, width, ds_stride));
    if (!aligned(dw, 4)) return BDLM_E_ALIGN;
    const int64_t ed = size_of(ds_dtype), need = dw ? norm_space(rows, width) : 0;
    if (need > 0 && (!ws || ws_bytes < need)) return BDLM_E_WORKSPACE;
    if (need > 0 && !aligned(ws, 256)) return BDLM_E_ALIGN;
    const Span sy(dy, rows, width, dy_stride, size_of(dy_dtype)), sx(s, rows, width, s_stride, size_of(s_dtype)),
        sb(dsum, rows, width, dsum_stride, ed), so(ds, rows, width, ds_stride, ed), sw(norm_w, 1, width, 0, 4),
        sg(dw, 1, width, 0, 4), ss(need > 0 ? ws : nullptr, 1, ws_bytes, 0, 1);
    const bool in_place = dsum && ds == dsum && ds_stride == dsum_stride;
    if (!in_place && so.meets(sb)) return BDLM_E_SHAPE;
    if (!apart(so, sy, sx, sw, sg) || !apart(sg, sy, sx, sb, sw)) return BDLM_E_SHAPE;
    return apart(ss, sy, sx, sb, so, sw, sg) ? BDLM_OK : BDLM_E_WORKSPACE;
}

int bdlm_add_rmsnorm_backward(int64_t rows, int64_t width, int32_t dy_dtype, const void *dy, int64_t dy_stride,
                              int32_t s_dtype, const void *s, int64_t s_stride, const float *norm_w, float eps,
                              int32_t ds_dtype, const void *dsum, int64_t dsum_stride, void *ds, int64_t ds_stride,
                              float *dw, void *ws, int64_t ws_bytes, void *stream) {
    TRY(bdlm_check_add_rmsnorm_backward(rows, width, dy_dtype, dy, dy_stride, s_dtype, s, s_stride, norm_w, eps, ds_dtype,
                                        dsum, dsum_stride, ds, ds_stride, dw, ws, ws_bytes));
    if (!ds && !dw) return BDLM_OK;
    AddNormGradArgs a{};
    a.dy = dy;
    a.s = s;
    a.dsum = dsum;
    a.ds = ds;
    a.w = norm_w;
    a.part = dw ? static_cast<float *>(ws) : nullptr;
    a.ldy = dy_stride;
    a.lds = s_stride;
    a.ldt = dsum_stride;
    a.ldd = ds_stride;
    a.rows = static_cast<int32_t>(rows);
    a.width = static_cast<int32_t>(width);
    a.dy_bf16 = dy_dtype == BDLM_DTYPE_BF16;
    a.s_bf16 = s_dtype == BDLM_DTYPE_BF16;
    a.ds_bf16 = ds_dtype == BDLM_DTYPE_BF16;
    a.eps = eps;
    TRY(launch_add_norm_grad(a, stream));
    return dw ? launch_colsum(a.part, add_norm_grad_blocks(rows, width), a.width, dw, stream) : BDLM_OK;
}

}  // extern "C"
