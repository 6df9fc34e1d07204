// bdlm_logprobs_api.cpp -- the C ABI of the head's log-probabilities (include/bdlm.h): argument checks, the plan of a call
// and its launches.  A plan depends on the descriptor and the number of alternatives alone.
#include <stdint.h>

#include "bdlm.h"
#include "bdlm_dense.h"
#include "bdlm_dense_plan.h"

namespace {

// Few rows' weights stream past; few tiles' contraction is split and the logits joined from partial sums, in memory; else
// the logits stay in the tiles.
struct LogprobsPlan {
    bool skinny, joined;
    Space ws;
    Operand x, w;
    Shape shape;
    int32_t ngroup, width;     // groups of columns, and values of one that are kept
    float *top, *others, *slope, *token_logit, *value, *part;
    int32_t *column;
    LogprobsPlan(const bdlm_dense_desc_t &d, int64_t n_top, const void *px, const void *pw, void *p)
        : skinny(few(d)), ws(p),
          x(px, skinny ? 0 : d.rows, d.in_features, d.x_stride, d.in_dtype, false, ws),
          w(pw, skinny ? 0 : d.out_features, d.in_features, d.w_stride, d.in_dtype, false, ws),
          shape(shape_of(d.rows, d.out_features, steps_of(d.in_features, pairs_of(d.in_dtype)), !skinny)) {
        joined = !skinny && shape.splits > 1;
        const int64_t edge = skinny ? skinny_cols(d.out_features) : joined ? kJoinGroup : tile_edge(shape.big);
        ngroup = static_cast<int32_t>((d.out_features + edge - 1) / edge);
        width = static_cast<int32_t>(n_top == 0 ? 0 : skinny || joined ? edge : n_top);
        const int64_t records = d.rows * ngroup;
        top = ws.take<float>(records);
        others = ws.take<float>(records);
        slope = ws.take<float>(records);
        token_logit = ws.take<float>(d.rows);
        value = ws.take<float>(records * width);
        column = ws.take<int32_t>(skinny || joined ? 0 : records * width);
        part = ws.take<float>(joined ? part_size(shape, d.rows, d.out_features) : 0);
    }
    bool fits() const { return skinny || shape.fits; }
};

int check_top(const bdlm_dense_desc_t *d, int64_t n_top, int64_t exclude) {
    const int64_t there = d->out_features - (exclude >= 0 && exclude < d->out_features ? 1 : 0);
    return n_top < 0 || n_top > BDLM_MAX_TOP || n_top > there ? BDLM_E_SHAPE : BDLM_OK;
}

}  // namespace

extern "C" {

int bdlm_head_logprobs_workspace(const bdlm_dense_desc_t *d, int64_t n_top, int64_t *bytes) {
    TRY(check_desc(d));
    if (!bytes) return BDLM_E_NULL;
    TRY(check_top(d, n_top, -1));
    *bytes = LogprobsPlan(*d, n_top, nullptr, nullptr, nullptr).ws.used;
    return BDLM_OK;
}

int bdlm_check_head_logprobs(const bdlm_dense_desc_t *d, const int64_t *tokens, int64_t exclude, int64_t n_top,
                             const void *x, const void *w, const float *logprob, const float *entropy,
                             const int64_t *top_token, const float *top_logprob, const void *ws, int64_t ws_bytes) {
    TRY(check_head(d, exclude, x, w));
    TRY(check_top(d, n_top, exclude));
    const int64_t listed = n_top > 0 ? d->rows * n_top : 0;
    if (d->rows > 0 && (!tokens != !logprob || (n_top > 0 && (!top_token || !top_logprob)))) return BDLM_E_NULL;
    if (!aligned(tokens, 8) || !aligned(logprob, 4) || !aligned(entropy, 4) || !aligned(top_token, 8) ||
        !aligned(top_logprob, 4))
        return BDLM_E_ALIGN;
    const LogprobsPlan plan(*d, n_top, nullptr, nullptr, nullptr);
    if (!plan.fits()) return BDLM_E_SHAPE;
    if (plan.ws.used > 0) {
        if (!ws || ws_bytes < plan.ws.used) return BDLM_E_WORKSPACE;
        if (!aligned(ws, 256)) return BDLM_E_ALIGN;
    }
    const Span sx = span_x(d, x), sw = span_w(d, w), st(tokens, 1, d->rows, 0, 8), sl(logprob, 1, d->rows, 0, 4),
               se(entropy, 1, d->rows, 0, 4), tt(top_token, 1, listed, 0, 8), tl(top_logprob, 1, listed, 0, 4),
               ss(ws, 1, ws_bytes, 0, 1);
    if (!apart(sl, sx, sw, st, se, tt, tl) || !apart(se, sx, sw, st, tt, tl) || !apart(tt, sx, sw, st, tl) ||
        !apart(tl, sx, sw, st))
        return BDLM_E_SHAPE;
    return apart(ss, sx, sw, st, sl, se, tt, tl) ? BDLM_OK : BDLM_E_WORKSPACE;
}

int bdlm_head_logprobs(const bdlm_dense_desc_t *d, const int64_t *tokens, int64_t exclude, int64_t n_top, const void *x,
                       const void *w, float *logprob, float *entropy, int64_t *top_token, float *top_logprob, void *ws,
                       int64_t ws_bytes, void *stream) {
    TRY(bdlm_check_head_logprobs(d, tokens, exclude, n_top, x, w, logprob, entropy, top_token, top_logprob, ws, ws_bytes));
    if (d->rows == 0 || (!tokens && !entropy && n_top == 0)) return BDLM_OK;
    LogprobsPlan p(*d, n_top, x, w, ws);
    const int32_t vocab = static_cast<int32_t>(d->out_features), list = static_cast<int32_t>(n_top);
    const TopArgs top{p.top, p.others, p.slope, p.token_logit, tokens, p.ngroup, token_or_none(d, exclude), list, p.value, p.column};
    if (p.skinny) {
        SkinnyArgs a = few_rows(*d, x, w, kTileTop);
        a.top = top;
        TRY(launch_skinny(a, stream));
    } else {
        TRY(lay_all(stream, p.x, p.w));
        TileArgs a = product(p.x.mat, false, p.w.mat, false, d->rows, vocab, d->in_features, pairs_of(d->in_dtype), p.shape);
        a.out = p.joined ? kTilePartial : kTileTop;
        a.part = p.part;
        if (!p.joined) a.top = top;
        TRY(launch_tile(a, stream));
        if (p.joined) TRY(launch_join_top(p.part, p.shape.splits, a.nrow, vocab, top, stream));
    }
    LogprobsArgs f{};
    f.top = p.top;
    f.others = p.others;
    f.slope = p.slope;
    f.ngroup = p.ngroup;
    f.rows = static_cast<int32_t>(d->rows);
    f.vocab = vocab;
    f.token = tokens;
    f.token_logit = p.token_logit;
    f.logprob = logprob;
    f.entropy = entropy;
    f.list = list;
    f.width = p.width;
    f.value = p.value;
    f.column = p.skinny || p.joined ? nullptr : p.column;
    f.top_token = top_token;
    f.top_logprob = top_logprob;
    return launch_logprobs(f, stream);
}

}  // extern "C"
