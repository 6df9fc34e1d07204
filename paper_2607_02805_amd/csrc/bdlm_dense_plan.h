// bdlm_dense_plan.h -- what the entry points of the dense operators share (bdlm_dense_api.cpp,
// bdlm_sublayer_api.cpp): argument checks, workspaces, and the plan of a product (which operands are laid out anew, tiles,
// splits).  Internal, plain C++.
#pragma once

#include <stdint.h>

#include <algorithm>

#include "bdlm.h"
#include "bdlm_dense.h"

namespace {

using namespace bdlm;

constexpr int64_t kMaxSize = int64_t(1) << 22;      // rows and features: grids stay within 32 bits
constexpr int64_t kMaxStride = int64_t(1) << 40;
constexpr int64_t kMaxDirect = int64_t(1) << 22;    // stride (elements) that 32-bit offsets in a tile reach

inline bool aligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline int64_t elem_size(int32_t dt) { return dt == BDLM_DTYPE_BF16 ? 2 : 4; }
inline bool known(int32_t dt) { return dt == BDLM_DTYPE_F32 || dt == BDLM_DTYPE_BF16; }
inline int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

// The memory of rows x cols elements with a row stride: `row` bytes every `ld`, `bytes` in all (unsigned: the largest
// rows and strides come to a little less than 2^64).
struct Span {
    uintptr_t p, bytes, row, ld;
    Span(const void *q, int64_t rows, int64_t cols, int64_t stride, int64_t es)
        : p(reinterpret_cast<uintptr_t>(q)),
          bytes(q && rows > 0 && cols > 0
                    ? (static_cast<uintptr_t>(rows - 1) * static_cast<uintptr_t>(stride) + static_cast<uintptr_t>(cols)) *
                          static_cast<uintptr_t>(es)
                    : 0),
          row(static_cast<uintptr_t>(cols * es)), ld(static_cast<uintptr_t>(stride * es)) {}
    bool meets(const Span &o) const {
        if (!bytes || !o.bytes || (o.p >= p ? o.p - p >= bytes : p - o.p >= o.bytes)) return false;
        if (ld != o.ld || ld == 0) return true;
        // column slices of one matrix: apart if the other's columns lie between this one's rows
        const uintptr_t at = o.p >= p ? (o.p - p) % ld : (ld - (p - o.p) % ld) % ld;
        return at < row || at + o.row > ld;
    }
};

inline int check_desc(const bdlm_dense_desc_t *d) {
    if (!d) return BDLM_E_NULL;
    if (!known(d->in_dtype) || d->reserved != 0) return BDLM_E_DTYPE;
    if (d->rows < 0 || d->in_features <= 0 || d->out_features <= 0 || d->rows > kMaxSize ||
        d->in_features > kMaxSize || d->out_features > kMaxSize)
        return BDLM_E_SHAPE;
    if (d->x_stride < 0 || d->w_stride < 0 || d->x_stride > kMaxStride || d->w_stride > kMaxStride)
        return BDLM_E_SHAPE;
    return BDLM_OK;
}
// An input whose rows may coincide (stride 0) or overlap.
inline int check_in(const void *p, int64_t rows) {
    if (rows > 0 && !p) return BDLM_E_NULL;
    return aligned(p, 16) ? BDLM_OK : BDLM_E_ALIGN;
}
// An output: its rows must not overlap.
inline int check_out(const void *p, int64_t rows, int64_t cols, int64_t ld) {
    if (rows > 0 && !p) return BDLM_E_NULL;
    if (!aligned(p, 16)) return BDLM_E_ALIGN;
    if (ld < 0 || ld > kMaxStride || (rows > 1 && ld < cols)) return BDLM_E_SHAPE;
    return BDLM_OK;
}

// ------------------------------------------------------------------ plans
// Takes pieces of the workspace in turn.
struct Space {
    char *base;
    int64_t used = 0;
    explicit Space(void *p) : base(static_cast<char *>(p)) {}
    template <class T>
    T *take(int64_t n) {
        T *p = base ? reinterpret_cast<T *>(base + used) : nullptr;
        used += up(n * int64_t(sizeof(T)), 256);
        return p;
    }
};

// A call whose rows the weights stream past.
inline bool few(const bdlm_dense_desc_t &d) { return d.rows <= skinny_rows(d.in_dtype == BDLM_DTYPE_BF16); }
constexpr int64_t kFewRows = 64;   // whose gradients keep two terms

inline int terms_of(int32_t dtype) { return dtype == BDLM_DTYPE_BF16 ? 1 : 3; }

// Tiles of a product and how its contraction is split over workgroups.  steps: contraction
// steps of 64 indices over all term pairs.
struct Shape {
    bool big;
    int32_t splits;
    bool fits = true;   // in one launch (fewer than 2^32 threads)
};
inline bool launch_fits(int64_t tiles) { return tiles * kTileThreads < int64_t(1) << 32; }
// The tiles and splits of the least time, as measured: a step of a large tile takes 1.75 us where
// every CU has one and 1.1 where few have (the clock), two of small tiles on a CU 0.92, one alone
// 0.38 to 0.52 (a third more where both operands' contraction index is the slow one: twice as many
// reads from LDS), and a tile 5 to 7 steps more to begin and to end.  16,384 x 4,096 over 1,024 takes
// 158 us in large tiles and 188 in small ones, 4,096 x 832 over 1,664 takes 43 and 20.  Partial
// sums are written and read again at 4 TB/s, by a launch of their own: 448 x 1,934 over 16,384
// takes 110 us whole and 50 in four splits, 512 x 4,384 over 1,024 takes 14 and 24 in two.
inline Shape shape_of(int64_t nrow, int64_t ncol, int64_t steps, bool may_split, bool both_slow = false) {
    const double small = both_slow ? 1.35 : 1.0;
    Shape best{true, 1, false};
    double least = 1e300;
    for (int big = 0; big < 2; ++big) {
        const int64_t e = tile_edge(big);
        const int64_t tiles = ((nrow + e - 1) / e) * ((ncol + e - 1) / e);
        for (int s = 1; s <= (may_split ? kMostSplits : 1); ++s) {
            if ((s > 1 && steps / s < 4) || !launch_fits(tiles * s)) break;
            const double deep = double((steps + s - 1) / s);
            // whole rounds of the chip, and what is left
            const int64_t per = big ? kChip : 2 * kChip, left = tiles * s % per;
            const double share = double(left) / kChip;
            double us = double(tiles * s / per) * (big ? (deep + 5.0) * 1.75 : (deep + 6.0) * 0.92 * small);
            if (left) us += big ? (deep + 5.0) * (1.1 + 0.65 * share)
                                : (share > 1.0 ? (deep + 6.0) * 0.92 : (deep + 7.0) * (0.38 + 0.14 * share)) * small;
            if (s > 1) us += 3.0 + double(s + 1) * nrow * ncol * 4.0 / 4.0e6;
            if (us < least) {
                least = us;
                best = Shape{big != 0, s, true};
            }
        }
    }
    return best;
}

// An operand [rows][cols] of a tiled product: as it lies, or laid out anew as bf16 terms (gathered,
// fp32, or of strides and widths that the tiles do not take: whole buffers of 64 columns).
struct Operand {
    const void *src;
    int64_t rows, cols, ld;
    int32_t dtype;
    bool direct;
    Mat mat{};
    uint16_t *copy = nullptr;

    Operand(const void *p, int64_t r, int64_t c, int64_t s, int32_t dt, bool gather, Space &ws)
        : src(p), rows(r), cols(c), ld(s), dtype(dt) {
        direct = !gather && dt == BDLM_DTYPE_BF16 && s % 8 == 0 && c % 64 == 0 && s <= kMaxDirect;
        if (direct) {
            mat = Mat{static_cast<const uint16_t *>(p), s, 0};
        } else {
            const int64_t w = up(c, 64);
            copy = ws.take<uint16_t>(terms_of(dt) * up(r, 64) * w);
            mat = Mat{copy, w, up(r, 64) * w};
        }
    }
    PackArgs pack(const int32_t *row_of = nullptr, const int32_t *rows_dev = nullptr, const float *scale = nullptr) const {
        PackArgs a{};
        a.src = src;
        a.ld = ld;
        a.rows = static_cast<int32_t>(rows);
        a.cols = static_cast<int32_t>(cols);
        a.src_bf16 = dtype == BDLM_DTYPE_BF16;
        a.rows_dev = rows_dev;
        a.row_of = row_of;
        a.scale = scale;
        a.dst = copy;
        a.ld_dst = mat.ld;
        a.plane = mat.plane;
        a.terms = terms_of(dtype);
        return a;
    }
    int lay(void *stream, const int32_t *row_of = nullptr, const int32_t *rows_dev = nullptr,
            const float *scale = nullptr) const {
        return direct ? BDLM_OK : launch_pack(pack(row_of, rows_dev, scale), stream);
    }
};

// Lays out those of the operands (of one type) that need it, in one launch.
template <class... O>
int lay_all(void *stream, const O &...operands) {
    PackArgs a[sizeof...(operands)];
    int32_t n = 0;
    for (const Operand *o : {&operands...})
        if (!o->direct) a[n++] = o->pack();
    return launch_pack_some(a, n, stream);
}

inline TileArgs product(const Mat &row, bool row_t, const Mat &col, bool col_t, int64_t nrow, int64_t ncol, int64_t k,
                 int32_t npair, const Shape &s) {
    TileArgs a{};
    a.row = row;
    a.col = col;
    a.nrow = static_cast<int32_t>(nrow);
    a.ncol = static_cast<int32_t>(ncol);
    a.k = static_cast<int32_t>(k);
    a.npair = npair;
    a.half = npair;
    a.row_t = row_t;
    a.col_t = col_t;
    a.skip = -1;
    a.big = s.big;
    a.splits = s.splits;
    return a;
}
// Terms of a gradient's first operand (dz, or the logits' gradients).  With bf16 inputs they are
// rounded to bf16, as the activations of the forward products are: the outputs of 16,384 x 1,024 x 4,096 are then
// off by 0.0023 of their size, where their own rounding makes 0.0017 of it, and a second term would double both
// products (277 of 352 us).  A gated product's gradients are off by 0.00235 so, whatever the sizes (the factors' gradients are rounded as the outputs are,
// 0.00166 each), and with a second term by 0.00166, but take 1,140 us instead of 606 there, 175 instead of 110 of 2,048 rows, 63 instead of 45 of 512, 38 instead
// of 31 of 65.  Of few rows, where an output's errors do not average out and the weights' bytes
// bound the products, two terms are kept; fp32 inputs keep three, and are the choice of a caller who needs more.
inline int grad_terms(const bdlm_dense_desc_t &d) {
    return d.in_dtype != BDLM_DTYPE_BF16 ? 3 : d.rows <= kFewRows ? 2 : 1;
}
inline int32_t grad_pairs(int terms) { return terms == 3 ? 6 : terms; }
inline int32_t pairs_of(int32_t dtype) { return dtype == BDLM_DTYPE_BF16 ? 1 : 6; }
inline int64_t steps_of(int64_t k, int32_t npair) { return (k + 63) / 64 * npair; }

// A product stored through `s`, split and joined where its shape says so.
inline int store_product(TileArgs a, const StoreArgs &s, float *part, void *stream) {
    if (a.splits == 1) {
        a.out = kTileStore;
        a.store = s;
        return launch_tile(a, stream);
    }
    a.out = kTilePartial;
    a.part = part;
    const int rc = launch_tile(a, stream);
    return rc != BDLM_OK ? rc : launch_join(part, a.splits, a.big, a.nrow, a.ncol, a.nrow_dev, nullptr, s, stream);
}
inline int64_t part_size(const Shape &s, int64_t nrow, int64_t ncol) { return s.splits > 1 ? s.splits * nrow * ncol : 0; }

inline StoreArgs plain_store(void *out, int64_t ld, int32_t dtype) {
    StoreArgs s{};
    s.out = out;
    s.ld_out = ld;
    s.out_bf16 = dtype == BDLM_DTYPE_BF16;
    s.act = BDLM_ACT_NONE;
    return s;
}

// Records of a softmax over the vocabulary.
struct Records {
    float *top, *others;
    int32_t *at;
    int32_t ntile;
    Records(int64_t rows, int64_t vocab, int64_t edge, Space &ws) {
        ntile = static_cast<int32_t>((vocab + edge - 1) / edge);
        top = ws.take<float>(rows * ntile);
        others = ws.take<float>(rows * ntile);
        at = ws.take<int32_t>(rows * ntile);
    }
};

inline SkinnyArgs few_rows(const bdlm_dense_desc_t &d, const void *x, const void *w, int32_t out) {
    SkinnyArgs a{};
    a.x = x;
    a.w = w;
    a.ldx = d.x_stride;
    a.ldw = d.w_stride;
    a.nrow = static_cast<int32_t>(d.rows);
    a.ncol = static_cast<int32_t>(d.out_features);
    a.k = static_cast<int32_t>(d.in_features);
    a.bf16 = d.in_dtype == BDLM_DTYPE_BF16;
    a.out = out;
    return a;
}

template <class P>
inline int query(const bdlm_dense_desc_t *d, int64_t *bytes) {
    const int rc = check_desc(d);
    if (rc != BDLM_OK) return rc;
    if (!bytes) return BDLM_E_NULL;
    *bytes = P(*d, nullptr, nullptr, nullptr).ws.used;
    return BDLM_OK;
}
template <class P>
inline int check_workspace(const bdlm_dense_desc_t *d, const void *ws, int64_t bytes) {
    const P plan(*d, nullptr, nullptr, nullptr);
    if (!plan.fits()) return BDLM_E_SHAPE;
    const int64_t need = plan.ws.used;
    if (need == 0) return BDLM_OK;
    if (!ws || bytes < need) return BDLM_E_WORKSPACE;
    return aligned(ws, 256) ? BDLM_OK : BDLM_E_ALIGN;
}

#define TRY(call)                             \
    do {                                      \
        const int rc_ = (call);               \
        if (rc_ != BDLM_OK) return rc_;       \
    } while (0)

inline int check_inputs(const bdlm_dense_desc_t *d, const void *x, const void *w) {
    TRY(check_desc(d));
    TRY(check_in(x, d->rows));
    return check_in(w, d->out_features);
}
inline Span span_x(const bdlm_dense_desc_t *d, const void *x) {
    return Span(x, d->rows, d->in_features, d->x_stride, elem_size(d->in_dtype));
}
inline Span span_w(const bdlm_dense_desc_t *d, const void *w) {
    return Span(w, d->out_features, d->in_features, d->w_stride, elem_size(d->in_dtype));
}
// An output (and the workspace) meets none of the other memory of the call.
template <class... S>
inline bool apart(const Span &out, const S &...others) {
    return !(out.meets(others) || ...);
}
inline int check_head(const bdlm_dense_desc_t *d, int64_t exclude, const void *x, const void *w) {
    TRY(check_inputs(d, x, w));
    // the softmax has a token to range over
    if (exclude == 0 && d->out_features == 1) return BDLM_E_SHAPE;
    return BDLM_OK;
}
inline int32_t token_or_none(const bdlm_dense_desc_t *d, int64_t t) {
    return t >= 0 && t < d->out_features ? static_cast<int32_t>(t) : -1;
}

}  // namespace
