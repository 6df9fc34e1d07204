// bdlm_dense_api.cpp -- the C ABI of the dense operators (include/bdlm.h): argument checks, the plan
// of a call (which operands are laid out anew, tiles, splits, pieces of the vocabulary) and its
// launches.  A plan depends on the descriptor alone, so the size a workspace query returns is
// the size the call uses.
#include <stdint.h>

#include <algorithm>

#include "bdlm.h"
#include "bdlm_dense.h"
#include "bdlm_dense_plan.h"

namespace {

struct ProjectionPlan {
    bool skinny;
    Space ws;
    Operand x, w;
    Shape shape;
    float *part;
    ProjectionPlan(const bdlm_dense_desc_t &d, const void *px, const void *pw, void *p)
        : skinny(few(d)), ws(p),
          x(px, skinny ? 0 : d.rows, d.in_features, d.x_stride, d.in_dtype, false, ws),
          w(pw, skinny ? 0 : d.out_features, d.in_features, d.w_stride, d.in_dtype, false, ws) {
        shape = skinny ? Shape{false, 1, true}
                       : shape_of(d.rows, d.out_features, steps_of(d.in_features, pairs_of(d.in_dtype)), true);
        part = ws.take<float>(part_size(shape, d.rows, d.out_features));
    }
    bool fits() const { return shape.fits; }
};

struct BackwardPlan {
    Space ws;
    Operand x, w;
    Shape sx, sw;
    uint16_t *dz;
    int64_t ld_dz;
    float *part, *sums;
    BackwardPlan(const bdlm_dense_desc_t &d, const void *px, const void *pw, void *p)
        : ws(p), x(px, d.rows, d.in_features, d.x_stride, d.in_dtype, false, ws),
          w(pw, d.out_features, d.in_features, d.w_stride, d.in_dtype, false, ws) {
        const int32_t np = grad_pairs(grad_terms(d));
        sx = shape_of(d.rows, d.in_features, steps_of(d.out_features, np), true);
        sw = shape_of(d.out_features, d.in_features, steps_of(d.rows, np), true, true);
        ld_dz = up(d.out_features, 64);
        dz = ws.take<uint16_t>(grad_terms(d) * up(d.rows, 64) * ld_dz);
        sums = ws.take<float>(int64_t(pack_row_blocks(static_cast<int32_t>(d.rows))) * d.out_features);
        part = ws.take<float>(std::max(part_size(sx, d.rows, d.in_features),
                                       part_size(sw, d.out_features, d.in_features)));
    }
    bool fits() const { return sx.fits && sw.fits; }
};

// The rows that count of a masked loss.
struct Rows {
    int32_t *count, *row_of, *label;
    float *weight, *loss, *lse, *scale;
    Rows(int64_t n, bool backward, Space &ws) {
        count = ws.take<int32_t>(1);
        row_of = ws.take<int32_t>(n);
        label = ws.take<int32_t>(n);
        weight = loss = lse = scale = nullptr;
        if (!backward) return;
        weight = ws.take<float>(n);
        loss = ws.take<float>(n);
        lse = ws.take<float>(n);
        scale = ws.take<float>(n);
    }
};

struct SelectPlan {
    bool skinny;
    Space ws;
    Operand x, w;
    Shape shape;
    Records rec;
    SelectPlan(const bdlm_dense_desc_t &d, const void *px, const void *pw, void *p)
        : skinny(few(d)), ws(p),
          x(px, skinny ? 0 : d.rows, d.in_features, d.x_stride, d.in_dtype, false, ws),
          w(pw, skinny ? 0 : d.out_features, d.in_features, d.w_stride, d.in_dtype, false, ws),
          shape(shape_of(d.rows, d.out_features, steps_of(d.in_features, pairs_of(d.in_dtype)), false)),
          rec(d.rows, d.out_features, skinny ? skinny_cols(d.out_features) : tile_edge(shape.big), ws) {}
    bool fits() const { return skinny || shape.fits; }
};

struct LossPlan {
    bool skinny;
    Space ws;
    Rows rows;
    Operand x, w;
    Shape shape;
    Records rec;
    float *label_logit;
    LossPlan(const bdlm_dense_desc_t &d, const void *px, const void *pw, void *p)
        : skinny(few(d)), ws(p), rows(d.rows, false, ws),
          x(px, skinny ? 0 : d.rows, d.in_features, d.x_stride, d.in_dtype, true, ws),
          w(pw, skinny ? 0 : d.out_features, d.in_features, d.w_stride, d.in_dtype, false, ws),
          shape(shape_of(d.rows, d.out_features, steps_of(d.in_features, pairs_of(d.in_dtype)), false)),
          rec(d.rows, d.out_features, skinny ? skinny_cols(d.out_features) : tile_edge(shape.big), ws),
          label_logit(ws.take<float>(d.rows)) {}
    bool fits() const { return skinny || shape.fits; }
};

// The vocabulary goes in pieces whose logit gradients (rows x piece, bf16 terms) stay within 512 MB, or have 4,096
// columns where those take more (bf16 above 65,536 rows, 2^22 rows 34 GB; fp32 above 21,845, 2^22 rows 103 GB): they
// are written once and read twice, mostly from the memory-side cache where half of the rows count.  The number of rows that count is known on the device alone, so the product over the
// vocabulary (dx) is split there.
struct LossBackwardPlan {
    Space ws;
    Rows rows;
    bool scaled;               // the rows of P are divided by their labels' entries
    Operand x, w, xs;          // xs: x times what they were divided by
    int64_t piece;
    Shape sp, sx, sw;
    uint16_t *p;
    float *part_x, *part_w;
    LossBackwardPlan(const bdlm_dense_desc_t &d, const void *px, const void *pw, void *mem)
        : ws(mem), rows(d.rows, true, ws), scaled(grad_terms(d) == 1),
          x(px, d.rows, d.in_features, d.x_stride, d.in_dtype, true, ws),
          w(pw, d.out_features, d.in_features, d.w_stride, d.in_dtype, false, ws),
          xs(px, scaled ? d.rows : 0, d.in_features, d.x_stride, d.in_dtype, true, ws) {
        const int32_t np = grad_pairs(grad_terms(d));
        const int64_t per = std::max<int64_t>(d.rows, 1) * 2 * grad_terms(d);
        piece = std::max<int64_t>((int64_t(512) << 20) / per / 256 * 256, 4096);
        piece = std::min(piece, up(d.out_features, 256));
        // pieces of nearly equal width
        const int64_t n = (d.out_features + piece - 1) / piece;
        piece = up((d.out_features + n - 1) / n, 256);
        sp = shape_of(d.rows, piece, steps_of(d.in_features, pairs_of(d.in_dtype)), false);
        // (few rows: the small tile, half of which they would leave empty in the large one)
        const bool big = d.rows > tile_edge(false);
        const int64_t e = tile_edge(big), cols = (d.in_features + e - 1) / e;
        sx = Shape{big, 0, launch_fits((d.rows + e - 1) / e * cols)};
        sw = shape_of(piece, d.in_features, steps_of(d.rows, np), true, true);
        p = ws.take<uint16_t>(grad_terms(d) * up(d.rows, 64) * piece);
        // summed over the pieces: what the splits of any number of rows take
        part_x = ws.take<float>(std::max(d.rows, std::min(d.rows * kMostSplits, kChip / std::min<int64_t>(cols, kChip) * e)) * d.in_features);
        part_w = ws.take<float>(part_size(sw, piece, d.in_features));
    }
    bool fits() const { return sp.fits && sx.fits && sw.fits; }
};

}  // namespace

extern "C" {

int bdlm_dense_desc_init(bdlm_dense_desc_t *d, int64_t rows, int64_t in_features, int64_t out_features,
                         int32_t in_dtype) {
    if (!d) return BDLM_E_NULL;
    *d = bdlm_dense_desc_t{rows, in_features, out_features, in_features, in_features, in_dtype, 0};
    return BDLM_OK;
}

int bdlm_projection_workspace(const bdlm_dense_desc_t *d, int64_t *bytes) { return query<ProjectionPlan>(d, bytes); }
int bdlm_projection_backward_workspace(const bdlm_dense_desc_t *d, int64_t *bytes) {
    return query<BackwardPlan>(d, bytes);
}
int bdlm_head_loss_workspace(const bdlm_dense_desc_t *d, int64_t *bytes) { return query<LossPlan>(d, bytes); }
int bdlm_head_loss_backward_workspace(const bdlm_dense_desc_t *d, int64_t *bytes) {
    return query<LossBackwardPlan>(d, bytes);
}
int bdlm_head_select_workspace(const bdlm_dense_desc_t *d, int64_t *bytes) { return query<SelectPlan>(d, bytes); }

int bdlm_check_projection(const bdlm_dense_desc_t *d, int32_t act, int32_t out_dtype, const void *x, const void *w,
                          const float *bias, const void *residual, int64_t residual_stride, const void *out,
                          int64_t out_stride, const void *pre, int64_t pre_stride, const void *ws,
                          int64_t ws_bytes) {
    TRY(check_desc(d));
    if (!known(out_dtype)) return BDLM_E_DTYPE;
    if (act < BDLM_ACT_NONE || act > BDLM_ACT_GELU) return BDLM_E_SHAPE;
    TRY(check_inputs(d, x, w));
    if (bias && !aligned(bias, 4)) return BDLM_E_ALIGN;
    TRY(check_out(out, d->rows, d->out_features, out_stride));
    if (pre) TRY(check_out(pre, d->rows, d->out_features, pre_stride));
    if (residual) {
        if (!aligned(residual, 16)) return BDLM_E_ALIGN;
        if (residual_stride < 0 || residual_stride > kMaxStride) return BDLM_E_SHAPE;
    }
    const int64_t es = elem_size(d->in_dtype), eo = elem_size(out_dtype);
    const Span so(out, d->rows, d->out_features, out_stride, eo), sp(pre, d->rows, d->out_features, pre_stride, es),
        sr(residual, d->rows, d->out_features, residual_stride, eo), sb(bias, 1, d->out_features, 0, 4),
        sx = span_x(d, x), sw = span_w(d, w);
    TRY(check_workspace<ProjectionPlan>(d, ws, ws_bytes));
    const Span ss(ws, 1, ws_bytes, 0, 1);
    // out may be residual itself (each element is read by the thread that writes it)
    const bool in_place = residual && residual == out && residual_stride == out_stride;
    if (!apart(so, sx, sw, sb, sp) || !apart(sp, sx, sw, sb, sr) || (!in_place && so.meets(sr)))
        return BDLM_E_SHAPE;
    return apart(ss, so, sp, sx, sw, sb, sr) ? BDLM_OK : BDLM_E_WORKSPACE;
}

int bdlm_projection(const bdlm_dense_desc_t *d, int32_t act, int32_t out_dtype, const void *x, const void *w,
                    const float *bias, const void *residual, int64_t residual_stride, void *out,
                    int64_t out_stride, void *pre, int64_t pre_stride, void *ws, int64_t ws_bytes, void *stream) {
    TRY(bdlm_check_projection(d, act, out_dtype, x, w, bias, residual, residual_stride, out, out_stride, pre,
                              pre_stride, ws, ws_bytes));
    if (d->rows == 0) return BDLM_OK;
    ProjectionPlan p(*d, x, w, ws);
    StoreArgs s = plain_store(out, out_stride, out_dtype);
    s.bias = bias;
    s.residual = residual;
    s.ld_res = residual_stride;
    s.pre = pre;
    s.ld_pre = pre_stride;
    s.pre_bf16 = d->in_dtype == BDLM_DTYPE_BF16;
    s.act = act;
    if (p.skinny) {
        SkinnyArgs a = few_rows(*d, x, w, kTileStore);
        a.store = s;
        return launch_skinny(a, stream);
    }
    TRY(p.x.lay(stream));
    TRY(p.w.lay(stream));
    return store_product(product(p.x.mat, false, p.w.mat, false, d->rows, d->out_features, d->in_features,
                                 pairs_of(d->in_dtype), p.shape),
                         s, p.part, stream);
}

int bdlm_check_projection_backward(const bdlm_dense_desc_t *d, int32_t act, int32_t dy_dtype, const void *dy,
                                   int64_t dy_stride, const void *x, const void *w, const void *pre,
                                   int64_t pre_stride, const void *dx, int64_t dx_stride, const void *dw,
                                   int64_t dw_stride, const float *db, const void *ws, int64_t ws_bytes) {
    TRY(check_desc(d));
    if (!known(dy_dtype)) return BDLM_E_DTYPE;
    if (act < BDLM_ACT_NONE || act > BDLM_ACT_GELU) return BDLM_E_SHAPE;
    // x is read for dw alone, w for dx alone
    TRY(check_in(x, dw ? d->rows : 0));
    TRY(check_in(w, dx ? d->out_features : 0));
    TRY(check_in(dy, d->rows));
    if (dy_stride < 0 || dy_stride > kMaxStride || pre_stride < 0 || pre_stride > kMaxStride) return BDLM_E_SHAPE;
    if (act != BDLM_ACT_NONE) TRY(check_in(pre, d->rows));
    if (dx) TRY(check_out(dx, d->rows, d->in_features, dx_stride));
    if (dw) TRY(check_out(dw, d->out_features, d->in_features, dw_stride));
    if (!aligned(db, 4)) return BDLM_E_ALIGN;
    const int64_t es = elem_size(d->in_dtype);
    const Span sx = span_x(d, x), sw = span_w(d, w),
               sy(dy, d->rows, d->out_features, dy_stride, elem_size(dy_dtype)),
               sp(act != BDLM_ACT_NONE ? pre : nullptr, d->rows, d->out_features, pre_stride, es),
               gx(dx, d->rows, d->in_features, dx_stride, es), gw(dw, d->out_features, d->in_features, dw_stride, es),
               gb(db, 1, d->out_features, 0, 4);
    TRY(check_workspace<BackwardPlan>(d, ws, ws_bytes));
    const Span ss(ws, 1, ws_bytes, 0, 1);
    if (!apart(gx, sx, sw, sy, sp, gw, gb) || !apart(gw, sx, sw, sy, sp, gb) || !apart(gb, sx, sw, sy, sp))
        return BDLM_E_SHAPE;
    return apart(ss, sx, sw, sy, sp, gx, gw, gb) ? BDLM_OK : BDLM_E_WORKSPACE;
}

int bdlm_projection_backward(const bdlm_dense_desc_t *d, int32_t act, int32_t dy_dtype, const void *dy,
                             int64_t dy_stride, const void *x, const void *w, const void *pre, int64_t pre_stride,
                             void *dx, int64_t dx_stride, void *dw, int64_t dw_stride, float *db, void *ws,
                             int64_t ws_bytes, void *stream) {
    TRY(bdlm_check_projection_backward(d, act, dy_dtype, dy, dy_stride, x, w, pre, pre_stride, dx, dx_stride, dw,
                                       dw_stride, db, ws, ws_bytes));
    BackwardPlan p(*d, x, w, ws);
    // dy as it is, where it can be an operand; else dz (a bf16 dy without an activation is one term)
    const bool exact = act == BDLM_ACT_NONE && d->in_dtype == BDLM_DTYPE_BF16 && dy_dtype == BDLM_DTYPE_BF16;
    const int terms = exact ? 1 : grad_terms(*d);
    const bool direct = exact && d->out_features % 64 == 0 && d->rows % 64 == 0 && dy_stride % 8 == 0 &&
                        dy_stride <= kMaxDirect;
    const int32_t np = grad_pairs(terms);
    Mat dz{p.dz, p.ld_dz, up(d->rows, 64) * p.ld_dz};
    if (direct) dz = Mat{static_cast<const uint16_t *>(dy), dy_stride, 0};
    if (!direct || db) {
        PackArgs a{};
        a.src = dy;
        a.ld = dy_stride;
        a.rows = static_cast<int32_t>(d->rows);
        a.cols = static_cast<int32_t>(d->out_features);
        a.src_bf16 = dy_dtype == BDLM_DTYPE_BF16;
        a.dst = direct || (!dx && !dw) ? nullptr : p.dz;
        a.ld_dst = p.ld_dz;
        a.plane = dz.plane;
        a.terms = terms;
        a.act = act;
        a.pre = pre;
        a.ld_pre = pre_stride;
        a.pre_bf16 = d->in_dtype == BDLM_DTYPE_BF16;
        a.colsum = db ? p.sums : nullptr;
        TRY(launch_pack(a, stream));
        if (db)
            TRY(launch_colsum(p.sums, pack_row_blocks(a.rows), a.cols, db, stream));
    }
    if (dx && d->rows > 0) {
        TRY(p.w.lay(stream));
        TRY(store_product(product(dz, false, p.w.mat, true, d->rows, d->in_features, d->out_features, np, p.sx),
                          plain_store(dx, dx_stride, d->in_dtype), p.part, stream));
    }
    if (dw) {
        TRY(p.x.lay(stream));
        TRY(store_product(product(dz, true, p.x.mat, true, d->out_features, d->in_features, d->rows, np, p.sw),
                          plain_store(dw, dw_stride, d->in_dtype), p.part, stream));
    }
    return BDLM_OK;
}

int bdlm_check_head_loss(const bdlm_dense_desc_t *d, const int64_t *labels, int64_t exclude, const void *x,
                         const void *w, const float *loss, const float *lse, const void *ws, int64_t ws_bytes) {
    TRY(check_head(d, exclude, x, w));
    if (d->rows > 0 && (!labels || !loss || !lse)) return BDLM_E_NULL;
    if (!aligned(labels, 8) || !aligned(loss, 4) || !aligned(lse, 4)) return BDLM_E_ALIGN;
    TRY(check_workspace<LossPlan>(d, ws, ws_bytes));
    const Span sx = span_x(d, x), sw = span_w(d, w), sl(labels, 1, d->rows, 0, 8), so(loss, 1, d->rows, 0, 4),
               se(lse, 1, d->rows, 0, 4), ss(ws, 1, ws_bytes, 0, 1);
    if (!apart(so, sx, sw, sl, se) || !apart(se, sx, sw, sl)) return BDLM_E_SHAPE;
    return apart(ss, sx, sw, sl, so, se) ? BDLM_OK : BDLM_E_WORKSPACE;
}

int bdlm_head_loss(const bdlm_dense_desc_t *d, const int64_t *labels, int64_t exclude, const void *x, const void *w,
                   float *loss, float *lse, void *ws, int64_t ws_bytes, void *stream) {
    TRY(bdlm_check_head_loss(d, labels, exclude, x, w, loss, lse, ws, ws_bytes));
    if (d->rows == 0) return BDLM_OK;
    LossPlan p(*d, x, w, ws);
    const int32_t rows = static_cast<int32_t>(d->rows), vocab = static_cast<int32_t>(d->out_features);
    const int32_t none = token_or_none(d, exclude);
    TRY(launch_rows(RowsArgs{labels, rows, vocab, exclude, p.rows.count, p.rows.row_of, p.rows.label, nullptr,
                             nullptr, nullptr, nullptr, nullptr, nullptr, nullptr},
                    stream));
    const BestArgs best{p.rec.top, p.rec.others, p.rec.at, p.label_logit, p.rows.label, p.rec.ntile, none};
    if (p.skinny) {
        SkinnyArgs a = few_rows(*d, x, w, kTileBest);
        a.nrow_dev = p.rows.count;
        a.row_of = p.rows.row_of;
        a.best = best;
        TRY(launch_skinny(a, stream));
    } else {
        TRY(p.x.lay(stream, p.rows.row_of, p.rows.count));
        TRY(p.w.lay(stream));
        TileArgs a = product(p.x.mat, false, p.w.mat, false, d->rows, vocab, d->in_features, pairs_of(d->in_dtype),
                             p.shape);
        a.nrow_dev = p.rows.count;
        a.out = kTileBest;
        a.best = best;
        TRY(launch_tile(a, stream));
    }
    return launch_finish(FinishArgs{p.rec.top, p.rec.others, p.rec.at, p.rec.ntile, rows, vocab, none, p.rows.count,
                                    p.rows.row_of, labels, p.label_logit, loss, lse, nullptr, nullptr},
                         stream);
}

int bdlm_check_head_loss_backward(const bdlm_dense_desc_t *d, const int64_t *labels, int64_t exclude,
                                  const void *x, const void *w, const float *loss, const float *lse,
                                  const float *dloss, const void *dx, int64_t dx_stride, const void *dw,
                                  int64_t dw_stride, const void *ws, int64_t ws_bytes) {
    TRY(check_head(d, exclude, x, w));
    if (d->rows > 0 && (!labels || !loss || !lse || !dloss)) return BDLM_E_NULL;
    if (!aligned(labels, 8) || !aligned(loss, 4) || !aligned(lse, 4) || !aligned(dloss, 4)) return BDLM_E_ALIGN;
    if (dx) TRY(check_out(dx, d->rows, d->in_features, dx_stride));
    if (dw) TRY(check_out(dw, d->out_features, d->in_features, dw_stride));
    TRY(check_workspace<LossBackwardPlan>(d, ws, ws_bytes));
    const int64_t es = elem_size(d->in_dtype);
    const Span sx = span_x(d, x), sw = span_w(d, w), sl(labels, 1, d->rows, 0, 8), so(loss, 1, d->rows, 0, 4),
               se(lse, 1, d->rows, 0, 4), sd(dloss, 1, d->rows, 0, 4),
               gx(dx, d->rows, d->in_features, dx_stride, es), gw(dw, d->out_features, d->in_features, dw_stride, es),
               ss(ws, 1, ws_bytes, 0, 1);
    if (!apart(gx, sx, sw, sl, so, se, sd, gw) || !apart(gw, sx, sw, sl, so, se, sd)) return BDLM_E_SHAPE;
    return apart(ss, sx, sw, sl, so, se, sd, gx, gw) ? BDLM_OK : BDLM_E_WORKSPACE;
}

int bdlm_head_loss_backward(const bdlm_dense_desc_t *d, const int64_t *labels, int64_t exclude, const void *x,
                            const void *w, const float *loss, const float *lse, const float *dloss, void *dx,
                            int64_t dx_stride, void *dw, int64_t dw_stride, void *ws, int64_t ws_bytes,
                            void *stream) {
    TRY(bdlm_check_head_loss_backward(d, labels, exclude, x, w, loss, lse, dloss, dx, dx_stride, dw, dw_stride, ws,
                                      ws_bytes));
    if (!dx && !dw) return BDLM_OK;
    LossBackwardPlan p(*d, x, w, ws);
    const int32_t rows = static_cast<int32_t>(d->rows), vocab = static_cast<int32_t>(d->out_features);
    const int32_t none = token_or_none(d, exclude), terms = grad_terms(*d), np = grad_pairs(terms);
    const int64_t K = d->in_features;
    TRY(launch_rows(RowsArgs{labels, rows, vocab, exclude, p.rows.count, p.rows.row_of, p.rows.label, dloss, loss,
                             lse, p.rows.weight, p.rows.loss, p.rows.lse, p.rows.scale},
                    stream));
    TRY(p.x.lay(stream, p.rows.row_of, p.rows.count));
    TRY(p.w.lay(stream));
    if (dw) TRY(p.xs.lay(stream, p.rows.row_of, p.rows.count, p.rows.scale));   // (of no rows: nothing)
    const Mat pm{p.p, p.piece, up(rows, 64) * p.piece};
    for (int64_t v0 = 0; v0 < vocab; v0 += p.piece) {
        const int64_t n = std::min(p.piece, vocab - v0);
        const Mat w_at{p.w.mat.p + v0 * p.w.mat.ld, p.w.mat.ld, p.w.mat.plane};
        TileArgs a = product(p.x.mat, false, w_at, false, rows, n, K, pairs_of(d->in_dtype), p.sp);
        a.nrow_dev = p.rows.count;
        a.out = kTileProb;
        a.prob = ProbArgs{p.p, pm.ld, pm.plane, terms, p.rows.lse, p.rows.loss, p.rows.weight, p.rows.label, none,
                          static_cast<int32_t>(v0), static_cast<int32_t>(up(n, 64))};
        TRY(launch_tile(a, stream));
        if (dx) {
            // w's row of the excluded token is not read: whatever it holds, it has no part in dx
            const int64_t x = none >= v0 && none < v0 + n ? none - v0 : -1;
            TileArgs b = product(pm, false, w_at, true, rows, K, x == n - 1 ? n - 1 : n, np, p.sx);
            b.skip = static_cast<int32_t>(x == n - 1 ? -1 : x);
            b.nrow_dev = p.rows.count;
            b.out = kTilePartial;
            b.part = p.part_x;
            b.add = v0 > 0;
            TRY(launch_tile(b, stream));
        }
        if (dw) {
            TileArgs c = product(pm, true, p.scaled ? p.xs.mat : p.x.mat, true, n, K, rows, np, p.sw);
            c.k_dev = p.rows.count;
            TRY(store_product(c, plain_store(static_cast<char *>(dw) + v0 * dw_stride * elem_size(d->in_dtype),
                                             dw_stride, d->in_dtype),
                              p.part_w, stream));
        }
    }
    if (dx) {
        StoreArgs s = plain_store(dx, dx_stride, d->in_dtype);
        s.row_of = p.rows.row_of;
        TRY(launch_join(p.part_x, 0, p.sx.big, rows, static_cast<int32_t>(K), p.rows.count,
                        p.scaled ? p.rows.scale : nullptr, s, stream));
        TRY(launch_zero_rows(labels, exclude, vocab, rows, dx, dx_stride, static_cast<int32_t>(K),
                             d->in_dtype == BDLM_DTYPE_BF16, stream));
    }
    return BDLM_OK;
}

int bdlm_check_head_select(const bdlm_dense_desc_t *d, int64_t exclude, const void *x, const void *w,
                           const int64_t *token, const float *logprob, const void *ws, int64_t ws_bytes) {
    TRY(check_head(d, exclude, x, w));
    if (d->rows > 0 && (!token || !logprob)) return BDLM_E_NULL;
    if (!aligned(token, 8) || !aligned(logprob, 4)) return BDLM_E_ALIGN;
    TRY(check_workspace<SelectPlan>(d, ws, ws_bytes));
    const Span sx = span_x(d, x), sw = span_w(d, w), st(token, 1, d->rows, 0, 8), sl(logprob, 1, d->rows, 0, 4),
               ss(ws, 1, ws_bytes, 0, 1);
    if (!apart(st, sx, sw, sl) || !apart(sl, sx, sw)) return BDLM_E_SHAPE;
    return apart(ss, sx, sw, st, sl) ? BDLM_OK : BDLM_E_WORKSPACE;
}

int bdlm_head_select(const bdlm_dense_desc_t *d, int64_t exclude, const void *x, const void *w, int64_t *token,
                     float *logprob, void *ws, int64_t ws_bytes, void *stream) {
    TRY(bdlm_check_head_select(d, exclude, x, w, token, logprob, ws, ws_bytes));
    if (d->rows == 0) return BDLM_OK;
    SelectPlan p(*d, x, w, ws);
    const int32_t rows = static_cast<int32_t>(d->rows), vocab = static_cast<int32_t>(d->out_features);
    const BestArgs best{p.rec.top, p.rec.others, p.rec.at, nullptr, nullptr, p.rec.ntile, token_or_none(d, exclude)};
    if (p.skinny) {
        SkinnyArgs a = few_rows(*d, x, w, kTileBest);
        a.best = best;
        TRY(launch_skinny(a, stream));
    } else {
        TRY(p.x.lay(stream));
        TRY(p.w.lay(stream));
        TileArgs a = product(p.x.mat, false, p.w.mat, false, rows, vocab, d->in_features, pairs_of(d->in_dtype),
                             p.shape);
        a.out = kTileBest;
        a.best = best;
        TRY(launch_tile(a, stream));
    }
    FinishArgs f{};
    f.top = p.rec.top;
    f.others = p.rec.others;
    f.at = p.rec.at;
    f.ntile = p.rec.ntile;
    f.rows = rows;
    f.vocab = vocab;
    f.exclude = best.exclude;
    f.token = token;
    f.logprob = logprob;
    return launch_finish(f, stream);
}

}  // extern "C"
