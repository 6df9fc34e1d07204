// bdlm_sublayer_api.cpp -- the C ABI of the operators of a sublayer (include/bdlm.h): the norm at its entry, with
// the residual's addition, the gated product of an MLP, and their gradients.  Argument checks, the plan of a call
// and its launches; a plan depends on the descriptor alone.
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

// Partial sums of dw, unless one workgroup writes dw itself.
int64_t norm_space(int64_t rows, int64_t width) {
    const int64_t blocks = bdlm::add_norm_grad_blocks(rows, width);
    return blocks > 1 ? up(blocks * width * 4, 256) : 0;
}

// From one operand to the other, in elements.
int64_t between(const Mat &a, const Mat &b) {
    return static_cast<int64_t>(reinterpret_cast<uintptr_t>(b.p) - reinterpret_cast<uintptr_t>(a.p)) / 2;
}

struct GatedPlan {
    bool skinny;
    Space ws;
    Operand x, wg, wu;         // (laid out anew, the weights lie one behind the other)
    Shape shape;
    float *part;
    GatedPlan(const bdlm_dense_desc_t &d, const void *px, const void *pg, const void *pu, void *p)
        : skinny(few(d)), ws(p),
          x(px, skinny ? 0 : d.rows, d.in_features, d.x_stride, d.in_dtype, false, ws),
          wg(pg, skinny ? 0 : d.out_features, d.in_features, d.w_stride, d.in_dtype, false, ws),
          wu(pu, skinny ? 0 : d.out_features, d.in_features, d.w_stride, d.in_dtype, false, ws) {
        const int64_t cols = gated_columns(d.out_features);
        shape = skinny ? Shape{false, 1, true}
                       : shape_of(d.rows, cols, steps_of(d.in_features, pairs_of(d.in_dtype)), true);
        part = ws.take<float>(part_size(shape, d.rows, cols));
    }
    bool fits() const { return shape.fits; }
};

// The gradients by both factors lie side by side, [terms][rows][2 ldz]: one product over both for dx, and one whose rows
// are those of both weights.
struct GatedBackwardPlan {
    Space ws;
    Operand x, wg, wu;
    int64_t ldz, plane;
    Shape sx, sw;
    uint16_t *dz;
    float *part, *sum_gate, *sum_up;
    GatedBackwardPlan(const bdlm_dense_desc_t &d, const void *px, const void *pg, const void *pu, void *p)
        : ws(p), x(px, d.rows, d.in_features, d.x_stride, d.in_dtype, false, ws),
          wg(pg, d.out_features, d.in_features, d.w_stride, d.in_dtype, false, ws),
          wu(pu, d.out_features, d.in_features, d.w_stride, d.in_dtype, false, ws) {
        const int32_t np = grad_pairs(grad_terms(d));
        ldz = up(d.out_features, 64);
        plane = up(d.rows, 64) * 2 * ldz;
        const int64_t both = ldz + d.out_features;
        // (reading one operand across its rows costs small tiles about what reading both does: 768 x 1,024 x 832 took 37.4 us by
        // the other figures, 34.8 so)
        sx = shape_of(d.rows, d.in_features, steps_of(d.out_features, 2 * np), true, true);
        sw = shape_of(both, d.in_features, steps_of(d.rows, np), true, true);
        dz = ws.take<uint16_t>(grad_terms(d) * plane);
        const int64_t sums = int64_t(pack_row_blocks(static_cast<int32_t>(d.rows))) * d.out_features;
        sum_gate = ws.take<float>(sums);
        sum_up = ws.take<float>(sums);
        part = ws.take<float>(std::max(part_size(sx, d.rows, d.in_features), part_size(sw, both, d.in_features)));
    }
    bool fits() const { return sx.fits && sw.fits; }
};

template <class P>
int gated_query(const bdlm_dense_desc_t *d, int64_t *bytes) {
    TRY(check_desc(d));
    if (!bytes) return BDLM_E_NULL;
    *bytes = P(*d, nullptr, nullptr, nullptr, nullptr).ws.used;
    return BDLM_OK;
}
template <class P>
int gated_space(const bdlm_dense_desc_t *d, const void *ws, int64_t bytes) {
    const P plan(*d, nullptr, nullptr, nullptr, nullptr);
    if (!plan.fits()) return BDLM_E_SHAPE;
    if (plan.ws.used == 0) return BDLM_OK;
    if (!ws || bytes < plan.ws.used) return BDLM_E_WORKSPACE;
    return aligned(ws, 256) ? BDLM_OK : BDLM_E_ALIGN;
}
// A product stored without an epilogue, split and joined where its shape says so: rows below two_rows go to s.out, those
// from two_at on to two_out.
int store_plain(TileArgs a, const StoreArgs &s, void *two_out, int32_t two_rows, int32_t two_at, float *part, void *stream) {
    a.store = s;
    a.two_out = two_out;
    a.two_rows = two_rows;
    a.two_at = two_at;
    a.out = a.splits > 1 ? kTilePartial : kTileTwo;
    a.part = part;
    TRY(launch_tile(a, stream));
    return a.splits > 1 ? launch_join_two(part, a.splits, a.nrow, a.ncol, two_out, two_rows, two_at, s, stream) : BDLM_OK;
}
int check_act(int32_t act) { return act < BDLM_ACT_NONE || act > BDLM_ACT_GELU ? BDLM_E_SHAPE : BDLM_OK; }

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
    const int32_t blocks = add_norm_grad_blocks(rows, width);
    a.part = dw && blocks > 1 ? static_cast<float *>(ws) : dw;
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
    return dw && blocks != 1 ? launch_colsum(a.part, blocks, a.width, dw, stream) : BDLM_OK;
}

int bdlm_gated_projection_workspace(const bdlm_dense_desc_t *d, int64_t *bytes) { return gated_query<GatedPlan>(d, bytes); }
int bdlm_gated_projection_backward_workspace(const bdlm_dense_desc_t *d, int64_t *bytes) {
    return gated_query<GatedBackwardPlan>(d, bytes);
}

int bdlm_check_gated_projection(const bdlm_dense_desc_t *d, int32_t act, int32_t out_dtype, const void *x,
                                const void *w_gate, const void *w_up, const float *bias_gate, const float *bias_up,
                                const void *out, int64_t out_stride, const void *pre_gate, const void *pre_up,
                                int64_t pre_stride, const void *ws, int64_t ws_bytes) {
    TRY(check_desc(d));
    if (!known(out_dtype)) return BDLM_E_DTYPE;
    TRY(check_act(act));
    TRY(check_inputs(d, x, w_gate));
    TRY(check_in(w_up, d->out_features));
    if (!aligned(bias_gate, 4) || !aligned(bias_up, 4)) return BDLM_E_ALIGN;
    TRY(check_out(out, d->rows, d->out_features, out_stride));
    if (!pre_gate != !pre_up) return BDLM_E_NULL;
    if (pre_gate) {
        TRY(check_out(pre_gate, d->rows, d->out_features, pre_stride));
        TRY(check_out(pre_up, d->rows, d->out_features, pre_stride));
    }
    const int64_t es = elem_size(d->in_dtype);
    const Span so(out, d->rows, d->out_features, out_stride, elem_size(out_dtype)),
        pg(pre_gate, d->rows, d->out_features, pre_stride, es), pu(pre_up, d->rows, d->out_features, pre_stride, es),
        bg(bias_gate, 1, d->out_features, 0, 4), bu(bias_up, 1, d->out_features, 0, 4), sx = span_x(d, x),
        wg = span_w(d, w_gate), wu = span_w(d, w_up);
    TRY(gated_space<GatedPlan>(d, ws, ws_bytes));
    const Span ss(ws, 1, ws_bytes, 0, 1);
    if (!apart(so, sx, wg, wu, bg, bu, pg, pu) || !apart(pg, sx, wg, wu, bg, bu, pu) || !apart(pu, sx, wg, wu, bg, bu))
        return BDLM_E_SHAPE;
    return apart(ss, so, pg, pu, sx, wg, wu, bg, bu) ? BDLM_OK : BDLM_E_WORKSPACE;
}

int bdlm_gated_projection(const bdlm_dense_desc_t *d, int32_t act, int32_t out_dtype, const void *x, const void *w_gate,
                          const void *w_up, const float *bias_gate, const float *bias_up, void *out, int64_t out_stride,
                          void *pre_gate, void *pre_up, int64_t pre_stride, void *ws, int64_t ws_bytes, void *stream) {
    TRY(bdlm_check_gated_projection(d, act, out_dtype, x, w_gate, w_up, bias_gate, bias_up, out, out_stride, pre_gate,
                                    pre_up, pre_stride, ws, ws_bytes));
    if (d->rows == 0) return BDLM_OK;
    GatedPlan p(*d, x, w_gate, w_up, ws);
    const GatedArgs g{out, bias_gate, bias_up, pre_gate, pre_up, out_stride, pre_stride, out_dtype == BDLM_DTYPE_BF16,
                      d->in_dtype == BDLM_DTYPE_BF16, act, static_cast<int32_t>(d->out_features)};
    if (p.skinny) {
        SkinnyArgs a = few_rows(*d, x, w_gate, kTileGated);
        a.w2 = w_up;
        a.gated = g;
        return launch_skinny(a, stream);
    }
    TRY(lay_all(stream, p.x, p.wg, p.wu));
    TileArgs a = product(p.x.mat, false, p.wg.mat, false, d->rows, gated_columns(d->out_features), d->in_features,
                         pairs_of(d->in_dtype), p.shape);
    a.col_duo = between(p.wg.mat, p.wu.mat);
    a.gated = g;
    a.out = p.shape.splits > 1 ? kTileGatedPart : kTileGated;
    a.part = p.part;
    TRY(launch_tile(a, stream));
    return p.shape.splits > 1 ? launch_join_gated(p.part, p.shape.splits, a.nrow, g, stream) : BDLM_OK;
}

int bdlm_check_gated_projection_backward(const bdlm_dense_desc_t *d, int32_t act, int32_t dh_dtype, const void *dh,
                                         int64_t dh_stride, const void *x, const void *w_gate, const void *w_up,
                                         const void *pre_gate, const void *pre_up, int64_t pre_stride, const void *dx,
                                         int64_t dx_stride, const void *dw_gate, const void *dw_up, int64_t dw_stride,
                                         const float *db_gate, const float *db_up, const void *ws, int64_t ws_bytes) {
    TRY(check_desc(d));
    if (!known(dh_dtype)) return BDLM_E_DTYPE;
    TRY(check_act(act));
    // x is read for the weights' gradients alone, the weights for dx alone
    TRY(check_in(x, dw_gate || dw_up ? d->rows : 0));
    TRY(check_in(w_gate, dx ? d->out_features : 0));
    TRY(check_in(w_up, dx ? d->out_features : 0));
    TRY(check_rows(dh, d->rows, dh_stride));
    TRY(check_rows(pre_gate, d->rows, pre_stride));
    TRY(check_rows(pre_up, d->rows, pre_stride));
    if (dx) TRY(check_out(dx, d->rows, d->in_features, dx_stride));
    if (dw_gate) TRY(check_out(dw_gate, d->out_features, d->in_features, dw_stride));
    if (dw_up) TRY(check_out(dw_up, d->out_features, d->in_features, dw_stride));
    if (!aligned(db_gate, 4) || !aligned(db_up, 4)) return BDLM_E_ALIGN;
    const int64_t es = elem_size(d->in_dtype), n = d->out_features, k = d->in_features;
    const Span sx = span_x(d, x), wg = span_w(d, w_gate), wu = span_w(d, w_up),
               sh(dh, d->rows, n, dh_stride, elem_size(dh_dtype)), pg(pre_gate, d->rows, n, pre_stride, es),
               pu(pre_up, d->rows, n, pre_stride, es), gx(dx, d->rows, k, dx_stride, es),
               gg(dw_gate, n, k, dw_stride, es), gu(dw_up, n, k, dw_stride, es), bg(db_gate, 1, n, 0, 4),
               bu(db_up, 1, n, 0, 4);
    TRY(gated_space<GatedBackwardPlan>(d, ws, ws_bytes));
    const Span ss(ws, 1, ws_bytes, 0, 1);
    if (!apart(gx, sx, wg, wu, sh, pg, pu, gg, gu, bg, bu) || !apart(gg, sx, wg, wu, sh, pg, pu, gu, bg, bu) ||
        !apart(gu, sx, wg, wu, sh, pg, pu, bg, bu) || !apart(bg, sx, wg, wu, sh, pg, pu, bu) ||
        !apart(bu, sx, wg, wu, sh, pg, pu))
        return BDLM_E_SHAPE;
    return apart(ss, sx, wg, wu, sh, pg, pu, gx, gg, gu, bg, bu) ? BDLM_OK : BDLM_E_WORKSPACE;
}

int bdlm_gated_projection_backward(const bdlm_dense_desc_t *d, int32_t act, int32_t dh_dtype, const void *dh,
                                   int64_t dh_stride, const void *x, const void *w_gate, const void *w_up,
                                   const void *pre_gate, const void *pre_up, int64_t pre_stride, void *dx,
                                   int64_t dx_stride, void *dw_gate, void *dw_up, int64_t dw_stride, float *db_gate,
                                   float *db_up, void *ws, int64_t ws_bytes, void *stream) {
    TRY(bdlm_check_gated_projection_backward(d, act, dh_dtype, dh, dh_stride, x, w_gate, w_up, pre_gate, pre_up,
                                             pre_stride, dx, dx_stride, dw_gate, dw_up, dw_stride, db_gate, db_up, ws,
                                             ws_bytes));
    if (!dx && !dw_gate && !dw_up && !db_gate && !db_up) return BDLM_OK;
    GatedBackwardPlan p(*d, x, w_gate, w_up, ws);
    const int terms = grad_terms(*d);
    const int32_t np = grad_pairs(terms), n = static_cast<int32_t>(d->out_features);
    GatedPackArgs g{};
    g.dh = dh;
    g.gate = pre_gate;
    g.up = pre_up;
    g.ld_dh = dh_stride;
    g.ld_pre = pre_stride;
    g.ldz = p.ldz;
    g.plane = p.plane;
    g.rows = static_cast<int32_t>(d->rows);
    g.n = n;
    g.dh_bf16 = dh_dtype == BDLM_DTYPE_BF16;
    g.pre_bf16 = d->in_dtype == BDLM_DTYPE_BF16;
    g.terms = terms;
    g.act = act;
    g.dst = dx || dw_gate || dw_up ? p.dz : nullptr;
    g.sum_gate = db_gate ? p.sum_gate : nullptr;
    g.sum_up = db_up ? p.sum_up : nullptr;
    TRY(launch_gated_pack(g, stream));
    TRY(launch_colsum2(p.sum_gate, p.sum_up, pack_row_blocks(g.rows), n, db_gate, db_up, stream));
    // (what both products need, in one launch)
    const bool wanted = dw_gate || dw_up, for_dx = dx && d->rows > 0;
    if (for_dx && wanted) TRY(lay_all(stream, p.wg, p.wu, p.x));
    else if (for_dx) TRY(lay_all(stream, p.wg, p.wu));
    else if (wanted) TRY(lay_all(stream, p.x));
    const Mat dz{p.dz, 2 * p.ldz, p.plane};
    if (for_dx) {
        TileArgs a = product(dz, false, p.wg.mat, true, d->rows, d->in_features, n, 2 * np, p.sx);
        a.half = np;
        a.row_duo = p.ldz;
        a.col_duo = between(p.wg.mat, p.wu.mat);
        TRY(store_plain(a, plain_store(dx, dx_stride, d->in_dtype), nullptr, a.nrow, a.nrow, p.part, stream));
    }
    if (!wanted) return BDLM_OK;
    if (!dw_gate || !dw_up) {
        const Mat one{p.dz + (dw_gate ? 0 : p.ldz), dz.ld, dz.plane};
        return store_plain(product(one, true, p.x.mat, true, n, d->in_features, d->rows, np, p.sw),
                           plain_store(dw_gate ? dw_gate : dw_up, dw_stride, d->in_dtype), nullptr, n, n, p.part, stream);
    }
    return store_plain(product(dz, true, p.x.mat, true, p.ldz + n, d->in_features, d->rows, np, p.sw),
                       plain_store(dw_gate, dw_stride, d->in_dtype), dw_up, n, static_cast<int32_t>(p.ldz), p.part, stream);
}

}  // extern "C"
