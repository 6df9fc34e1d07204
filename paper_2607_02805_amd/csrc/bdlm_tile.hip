// bdlm_tile.hip -- gfx950 tiled matrix products of the dense operators: acc[row][col] = sum over k
// of row(row, k) * col(col, k) in bf16 terms with fp32 accumulation, and what becomes of a tile
// (bdlm_dense.h: the epilogue of a projection, partial sums, softmax records, loss gradients).
//
// One workgroup per tile (and split).  The operands go straight from memory to LDS in 16-byte
// pieces, a stage of 64 contraction indices at a time into one of two buffers (or four).  `col` is
// the first MFMA operand, so a lane holds groups of four consecutive columns of one row.
//
// Bound by the matrix unit and the clock that it can hold: 8,192 x 8,192 x 8,192 in bf16 takes
// 860 to 960 us by the card (1,280 to 1,145 TFLOP/s), with the matrix unit busy in 0.76 of the
// cycles and the clock at 1.4 to 2.0 GHz under that load.  A tile of 256 x 256
// reads a byte of its operands for 128 operations; tiles of 128 x 128 need twice the LDS reads and
// copies and are for launches that large tiles would leave partly idle.  The epilogue of a large tile is not hidden, as its
// buffers leave a CU one workgroup: GELU with the pre-activation kept costs 40 of the 204 us of
// 16,384 x 1,024 x 4,096 in bf16 (164 without either, 195 with GELU alone).
// Built and measured slower at 8,192^3: four waves of 128 x 128 (900 to 1,080 us), operands
// staged through registers, a ring of four stages of 32, a stage's copies all in one group,
// nontemporal or streaming copies.
//
// An operand whose contraction index is contiguous lies in LDS as [row][64] (eight pieces a
// row) and is read 16 bytes a lane; one whose contraction index is the slow one lies as
// [64][row] and is read with the LDS transpose read.  Both are permuted by the piece so that a
// quarter wave meets every bank once (no conflicts counted); as the copy writes LDS in lane order,
// the permutation is of the addresses in memory that the lanes read.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "bdlm.h"
#include "bdlm_dense.h"
#include "bdlm_dense_device.h"
#include "bdlm_store.h"

namespace bdlm {
namespace {

constexpr int kDepth = 64;    // contraction indices of a stage (a cache line of an operand's row)
constexpr int kGroups = kDepth / 16;   // of products

typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// 16 bytes a lane from base + off + AT to LDS at `to` + AT, lane by lane (the instruction adds its
// offset to both).  Written out because the compiler makes every LDS transpose read wait for the
// copies it knows of; nothing is returned in registers, and group() waits for the copies before
// the barrier that hands a buffer over.
template <int AT>
__device__ __forceinline__ void copy16(const char *base, uint32_t off, uint32_t to) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 offset:%3"
                 :
                 : "v"(off), "s"(base), "s"(to), "n"(AT)
                 : "memory", "m0");
}
__device__ __forceinline__ bf16x8 frag(const char *lds) {
    return __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4 *>(lds));
}
__device__ __forceinline__ s16x4 read_tr(const char *lds) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(const_cast<char *>(lds)));
}
typedef float f32x16 __attribute__((ext_vector_type(16)));

// c += a b, in place: written out so that the accumulators stay in their registers (given the
// builtin, the compiler rotates them through copies).  The wait states cover an operand that the
// compiler has just moved; the
// matrix pipeline is busy for longer than that.  At every edge of the control flow, where the
// compiler may move accumulators, settle() waits for the last products' results.
// 32 x 32 outputs a product: a wave issues an instruction every four cycles or so, and products of
// 16 x 16 take 16 cycles, which leaves too few in between for the reads and copies.
__device__ __forceinline__ void mma(bf16x8 a, bf16x8 b, f32x16 &c) {
    asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
}
// A product's results may be read by other instructions after at most 19 wait states.
template <int FC, int FR>
__device__ __forceinline__ void settle(f32x16 (&acc)[FC][FR]) {
    asm volatile("s_nop 15\n\ts_nop 3");
#pragma unroll
    for (int i = 0; i < FC; ++i)
#pragma unroll
        for (int j = 0; j < FR; ++j) asm volatile("" : "+a"(acc[i][j]));
}

// The permutation of a contraction row's pieces (an operand whose contraction index is slow).
__device__ __forceinline__ int piece_of(int t) { return 4 * (t & 3) ^ 2 * ((t >> 3) & 1); }

// One operand's share of a tile: R rows (or columns) from `first` on, a stage deep.  REPEAT (T
// only): contraction indices past the operand's end, and the index `skip`, read another row again,
// as the other operand is zero there.
template <int R, bool T, int WAVES, bool REPEAT>
struct Stage {
    static constexpr int kPieces = R * kDepth / 8;        // 16-byte pieces of a stage
    static constexpr int kLoads = kPieces / (64 * WAVES);   // per lane
    static_assert(kLoads * 64 * WAVES == kPieces, "whole loads");
    static constexpr int kLast = (kLoads - 1) * 1024;   // a wave's pieces lie together: its last 64 from its first
    static_assert(kLast < 4096, "the instruction's offset");
    const char *base;      // the operand at (first, 0) of its first plane, less kLast
    int64_t ld2;           // bytes of a row
    uint32_t off[kLoads];    // this lane's bytes from base, less the instruction's offset
    int32_t at[T ? kLoads : 1];   // T: contraction index of the piece within the stage

    // rows past the operand's end repeat its last row, columns past it its first piece
    __device__ __forceinline__ void init(const Mat &m, int64_t first, int64_t size, int wave, int lane) {
        ld2 = m.ld * 2;
        base = reinterpret_cast<const char *>(m.p) + (T ? first * 2 : first * ld2) - kLast;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int piece = (wave * kLoads + i) * 64 + lane, more = kLast - i * 1024;
            if constexpr (T) {
                constexpr int kRow = R / 8;
                const int t = piece / kRow, pos = piece % kRow;
                int c = pos ^ piece_of(t);
                if (first + 8 * c >= size) c = 0;
                at[i] = t;
                off[i] = static_cast<uint32_t>(t * ld2 + c * 16) + more;
            } else {
                const int r = piece >> 3, c = (piece & 7) ^ ((r >> 1) & 7);
                const int64_t rr = first + r < size ? r : size - 1 - first;
                off[i] = static_cast<uint32_t>(rr * ld2 + c * 16) + more;
            }
        }
    }
    // Rows of two matrices in turn, 32 of either (GatedArgs): a wave copies rows of one of them.  first: the tile's first
    // column of the product; size: rows of either matrix.
    __device__ __forceinline__ void init_gated(const Mat &m, int64_t duo, int64_t first, int64_t size, int wave, int lane) {
        static_assert(!T && kLoads * 8 <= 32 && 32 % (kLoads * 8) == 0, "a wave's rows are of one matrix");
        ld2 = m.ld * 2;
        const int up = (wave * kLoads * 8 >> 5) & 1;
        first >>= 1;
        base = reinterpret_cast<const char *>(m.p + (up ? duo : 0)) + first * ld2 - kLast;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int piece = (wave * kLoads + i) * 64 + lane, more = kLast - i * 1024;
            const int r = piece >> 3, c = (piece & 7) ^ ((r >> 1) & 7), own = (r >> 6) * 32 + (r & 31);
            const int64_t rr = first + own < size ? own : size - 1 - first;
            off[i] = static_cast<uint32_t>(rr * ld2 + c * 16) + more;
        }
    }
    __device__ __forceinline__ const char *at_step(int64_t plane, int kt) const {
        return base + plane * 2 + kt * stride();
    }
    __device__ __forceinline__ int64_t stride() const { return T ? kDepth * ld2 : 2 * kDepth; }   // of a stage
    // left, skip: contraction indices from the stage's first to the operand's end, and to the one that
    // is not read (never the only one of a stage)
    // lds: the wave's pieces of the stage
    template <int I>
    __device__ __forceinline__ void copy(const char *from, uint32_t lds, int left, int skip) const {
        constexpr int i = I;
        uint32_t o = off[i];
        if constexpr (T && REPEAT)
            o = at[i] < left && at[i] != skip ? o : o + static_cast<uint32_t>(((skip == 0) - at[i]) * ld2);
        copy16<I * 1024>(from, o, lds);
    }
};

// Operand reads: fragment i, 32 rows from `row0` + 32 i, of group `first` + g of the stage (16
// indices; G groups).  Lane: row lane & 31, indices 8 (lane >> 5) .. + 7.
template <int R, bool T, int F, int G>
struct Reader {
    int off[T ? F : G];
    __device__ __forceinline__ void init(int row0, int first, int lane) {
        if constexpr (T) {
            const int s = lane & 15, t = 8 * (lane >> 5) + (s >> 2);
#pragma unroll
            for (int i = 0; i < F; ++i) {
                const int c = (row0 + 32 * i + (lane & 16)) / 8 + ((s & 3) >> 1);
                off[i] = (t * (R / 8) + (c ^ piece_of(t))) * 16 + (s & 1) * 8 + first * (16 * 2 * R);
            }
        } else {
            const int r = row0 + (lane & 31);
#pragma unroll
            for (int g = 0; g < G; ++g) off[g] = r * 128 + (((2 * (first + g) + (lane >> 5)) ^ ((r >> 1) & 7)) * 16);
        }
    }
    __device__ __forceinline__ bf16x8 get(const char *lds, int i, int g) const {
        if constexpr (T) {
            const char *p = lds + off[i] + g * (16 * 2 * R);
            const s16x4 a = read_tr(p), b = read_tr(p + 4 * 2 * R);
            return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            return frag(lds + off[g] + i * (32 * 128));
        }
    }
};

// Pair i of planes multiplies term row_term(i) of `row` and col_term(i) of `col`: of two fp32
// operands the six of weight 2^-16 or more, of a `row` in two terms and a bf16 `col` both.
__device__ __forceinline__ int row_term(int npair, int i) { return npair == 6 ? static_cast<int>(0x010210ll >> (4 * i)) & 15 : i; }
__device__ __forceinline__ int col_term(int npair, int i) { return npair == 6 ? static_cast<int>(0x102010ll >> (4 * i)) & 15 : 0; }

template <int V>
struct Int {
    static constexpr int value = V;
};
// f(Int<0>) .. f(Int<N - 1>)
template <int N, class F>
__device__ __forceinline__ void repeat(F f) {
    if constexpr (N > 0) {
        repeat<N - 1>(f);
        f(Int<N - 1>{});
    }
}

// What the epilogue needs of a row, kept in LDS from the start of the kernel.
struct RowData {
    float lse, g, hot;   // kTileProb: lse, weight, the label's gradient
    int label;           // kTileProb, kTileBest
};

// Four columns of a row that goes to one of two matrices, or to neither.
__device__ __forceinline__ void store_two(const StoreArgs &s, void *two_out, int two_rows, int two_at, f32x4 v, int64_t r, int c,
                                          int ncol) {
    const int n = ncol - c < 4 ? ncol - c : 4;
    if (n <= 0 || (r >= two_rows && r < two_at)) return;
    const bool second = r >= two_at;
    put4(second ? two_out : s.out, (second ? r - two_at : r) * s.ld_out + c, s.ld_out, n, s.out_bf16, v);
}

// Four columns of one row of a tile, in their place.
template <int OUT>
__device__ __forceinline__ void tile_quad(const TileArgs &a, f32x4 v, f32x4 bias, const RowData &d, int64_t r, int c,
                                          int nrow, int split) {
    if constexpr (OUT == kTileStore) {
        store4(a.store, v, bias, r, c, a.ncol);
    } else if constexpr (OUT == kTilePartial || OUT == kTileGatedPart) {
        float *to = a.part + (int64_t(split) * (a.splits ? a.nrow : nrow) + r) * a.ncol + c;
        if (c + 4 <= a.ncol) {   // (at any alignment)
            if (a.add) v += *reinterpret_cast<const f32x4_a4 *>(to);
            *reinterpret_cast<f32x4_a4 *>(to) = v;
        } else {
            for (int e = 0; e < 4; ++e)
                if (c + e < a.ncol) to[e] = a.add ? to[e] + v[e] : v[e];
        }
    } else {
        const ProbArgs &b = a.prob;
        if (c >= b.width) return;
        if (b.terms == 3) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = d.g * expf(v[e] - d.lse);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = d.g * __builtin_amdgcn_exp2f((v[e] - d.lse) * kLog2e);
        }
        // few quads hold a label, the excluded token or columns past the end
        const unsigned label = d.label - c, exclude = b.exclude - b.col0 - c;
        if (label < 4u || exclude < 4u || c + 4 > a.ncol) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (label == static_cast<unsigned>(e)) v[e] = d.hot;
                if (c + e >= a.ncol || exclude == static_cast<unsigned>(e)) v[e] = 0.f;
            }
        }
        uint16_t *to = b.p + r * b.ld + c;
        if (b.terms == 1) {
            *reinterpret_cast<uint2 *>(to) = uint2{cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3])};
        } else {
            uint16_t h[4][3];
#pragma unroll
            for (int e = 0; e < 4; ++e) split_terms(v[e], h[e]);
#pragma unroll
            for (int k = 0; k < 3; ++k)
                if (k < b.terms)
                    *reinterpret_cast<uint2 *>(to + k * b.plane) =
                        uint2{h[0][k] | uint32_t(h[1][k]) << 16, h[2][k] | uint32_t(h[3][k]) << 16};
        }
    }
}

// The softmax record of a row's columns col1 .. + cols - 1, which lie in LDS as quads permuted by
// `swap`.  The largest value's place is overwritten, so that the others are all the rest.
__device__ __forceinline__ Best row_best(const TileArgs &a, f32x4 *row, int swap, int cols, int col1) {
    int n = a.ncol - col1 < cols ? a.ncol - col1 : cols;   // columns that there are
    n = n < 0 ? 0 : n;
    const int nq = (n + 3) >> 2;
    auto place = [&](int c) { return reinterpret_cast<float *>(row + ((c >> 2) ^ swap)) + (c & 3); };
    for (int c = n; c < 4 * nq; ++c) *place(c) = -INFINITY;
    const int x = a.best.exclude - col1;
    if (x >= 0 && x < n) *place(x) = -INFINITY;
    Best m{-INFINITY, 0.f, kNoColumn};
    int first = -1;
#pragma unroll 8
    for (int q = 0; q < nq; ++q) {
        const f32x4 v = row[q ^ swap];
        const float t = fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3]));   // (passes over a NaN)
        first = t > m.top ? q : first;
        m.top = fmaxf(m.top, t);
    }
    if (first >= 0) {
        const f32x4 v = row[first ^ swap];
        const int e = v[0] == m.top ? 0 : v[1] == m.top ? 1 : v[2] == m.top ? 2 : 3;
        m.at = col1 + 4 * first + e;
        *place(4 * first + e) = -INFINITY;
    }
    // -infinities add nothing, also where there is nothing else
    const float ref = m.top == -INFINITY ? 0.f : m.top;
#pragma unroll 8
    for (int q = 0; q < nq; ++q) {
        const f32x4 v = row[q ^ swap];
        float s[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] = __builtin_amdgcn_exp2f((v[e] - ref) * kLog2e);
        m.others += (s[0] + s[1]) + (s[2] + s[3]);
    }
    return m;
}

// Largest value and sum of four consecutive lanes, in each.
template <int CTRL>
__device__ __forceinline__ float quad_other(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(v), __float_as_int(v), CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ float quad_largest(float v) {
    v = fmaxf(v, quad_other<0xb1>(v));
    return fmaxf(v, quad_other<0x4e>(v));
}
__device__ __forceinline__ float quad_sum(float v) {
    v += quad_other<0xb1>(v);
    return v + quad_other<0x4e>(v);
}

// The record of a row and with b.list > 0 its largest values in order (the lower column first of equals), by four consecutive
// lanes: each has the row's 8 OCTS columns from col1 on, which lie in LDS as quads row[(at + q) ^ swap].  Every step takes the largest
// value out, some 80 instructions: the lane that has it finds it by the maxima of its groups of eight columns, which are kept in
// registers, and puts -infinity in its place.  o: the row's place in the records, or less than 0 (nothing is written).
// (With a lane for 64 columns of a row, and the waves' lists merged by a lane a row, 512 rows of 50,257 of 1,024 with five listed
// took 88 us instead of 83, with sixteen 120 instead of 108, and 1,800 of 25,757 of 254, in small tiles, 156 instead of 125.)
template <int OCTS>
__device__ __forceinline__ void row_top(const TopArgs &b, int ncol, f32x4 *row, int at, int swap, int col1, int lane, int64_t o) {
    constexpr int kCols = 8 * OCTS;
    auto place = [&](int c) { return reinterpret_cast<float *>(row + ((at + (c >> 2)) ^ swap)) + (c & 3); };
    int n = ncol - col1 < kCols ? ncol - col1 : kCols;
    n = n < 0 ? 0 : n;
    for (int c = n; c < kCols; ++c) *place(c) = -INFINITY;
    const int x = b.exclude - col1;
    if (x >= 0 && x < n) *place(x) = -INFINITY;
    float most[OCTS];
#pragma unroll
    for (int q = 0; q < OCTS; ++q) {
        const f32x4 u = row[(at + 2 * q) ^ swap], v = row[(at + 2 * q + 1) ^ swap];
        most[q] = fmaxf(fmaxf(fmaxf(u[0], u[1]), fmaxf(u[2], u[3])), fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])));
        most[q] = fmaxf(most[q], -INFINITY);   // (nothing but NaN)
    }
    const int s = lane & 3;
    auto take = [&](int j) {
        float own = most[0];
#pragma unroll
        for (int q = 1; q < OCTS; ++q) own = fmaxf(own, most[q]);
        const float m = quad_largest(own);
        // the lowest of the lanes that hold it (numbers that are exact as floats)
        const float first = -quad_largest(own == m ? -static_cast<float>(s) : -4.f);
        if (first == static_cast<float>(s)) {
            int g = 0;
#pragma unroll
            for (int q = OCTS - 1; q >= 0; --q) g = most[q] == m ? q : g;
            const f32x4 u = row[(at + 2 * g) ^ swap], v = row[(at + 2 * g + 1) ^ swap];
            const float w[8] = {u[0], u[1], u[2], u[3], v[0], v[1], v[2], v[3]};
            int e = 0;
#pragma unroll
            for (int k = 7; k >= 0; --k) e = w[k] == m ? k : e;
            float rest = -INFINITY;
#pragma unroll
            for (int k = 0; k < 8; ++k) rest = fmaxf(rest, k == e ? -INFINITY : w[k]);
            if (m > -INFINITY) *place(8 * g + e) = -INFINITY;
#pragma unroll
            for (int q = 0; q < OCTS; ++q) most[q] = q == g ? rest : most[q];
            if (j < b.list && o >= 0) {
                b.value[o * b.list + j] = m;
                b.column[o * b.list + j] = m > -INFINITY ? col1 + 8 * g + e : kNoColumn;
            }
        }
        return m;
    };
    const float top = take(0);
    const float ref = top == -INFINITY ? 0.f : top;
    float others = 0.f, slope = 0.f;
#pragma unroll
    for (int q = 0; q < 2 * OCTS; ++q) {
        const f32x4 v = row[(at + q) ^ swap];
        float t[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) t[e] = __builtin_amdgcn_exp2f((v[e] - ref) * kLog2e);
        others += (t[0] + t[1]) + (t[2] + t[3]);
        slope += (slope_of(t[0], v[0] - ref) + slope_of(t[1], v[1] - ref)) + (slope_of(t[2], v[2] - ref) + slope_of(t[3], v[3] - ref));
    }
    others = quad_sum(others);
    slope = quad_sum(slope);
    if (s == 0 && o >= 0) {
        b.top[o] = top;
        b.others[o] = others;
        b.slope[o] = slope;
    }
    for (int j = 1; j < b.list; ++j) take(j);
}

// WR x WC waves of (E / WR) x (E / WC) outputs: of 128 x 64 in a tile of 256, of 64 x 64 in one of
// 128, where KS = 2 such sets of waves take half of a stage's contraction each and add up at the
// end.  (With one set a SIMD has a wave too few: instructions come at most every four cycles from a
// wave, some ten a product, and a product takes 32.  512 x 1,024 x 4,384 takes 14.5 us instead of
// 17.1, 1,500 x 832 x 16,001 in fp32 276 instead of 286.  Large tiles have two waves a SIMD, and no
// registers for more.)  A stage is four groups of products, or a wave's two of them, each from one
// of two sets of registers while the other fills with the next group's operands from LDS.  With
// the last group's operands read, and the next stage arrived in its buffer, the waves meet; then the
// stage that takes this buffer over is copied into it, from the last group on and through the next
// stage's first.
//
// E 256: two waves on each SIMD, 128 accumulators a lane.  E 128 with two buffers: two workgroups on
// a CU, so that one's epilogue meets the other's products.
template <int E, int WR, int WC, int KS, int BUFS, bool ROWT, bool COLT, int OUT>
__global__ void __launch_bounds__(64 * WR * WC * KS, KS * (BUFS == 2 ? 2 : 1)) bdlm_tile_kernel(const TileArgs a) {
    static_assert(64 * WR * WC * KS == kTileThreads, "what the launch has, and the host's check counts on");
    constexpr int WAVES = WR * WC * KS, kWaveGroups = kGroups / KS, FR = E / WR / 32, FC = E / WC / 32;   // fragments of a wave
    constexpr int kBuf = E * kDepth / 8;                 // pieces of an operand's stage
    constexpr bool kTop = OUT == kTileTop;
    constexpr int kRec = OUT == kTileBest ? E : 1;
    __shared__ uint4 sm[BUFS][2 * kBuf];                 // [buffer][col, then row]
    __shared__ RowData rows[OUT == kTileProb || OUT == kTileBest || kTop ? E : 1];
    __shared__ float top[WC][kRec], others[WC][kRec];    // softmax records of the waves' columns
    __shared__ int at[WC][kRec];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int nrow = a.nrow_dev ? *a.nrow_dev : a.nrow;
    const int K = a.k_dev ? *a.k_dev : a.k;
    const int tr = (nrow + E - 1) / E, tc = (a.ncol + E - 1) / E;
    // Consecutive workgroups go to the eight XCDs in turn: each XCD takes a run of the tile
    // order, four tile rows by all columns at a time, so that the tiles that run together on it
    // share rows and columns in its L2.
    const int splits = a.splits ? a.splits : split_count(int64_t(tr) * tc);
    const uint32_t total = static_cast<uint32_t>(tr) * tc * splits;
    const uint32_t id = blockIdx.x;
    if (id >= total) return;
    const uint32_t q = total >> 3, rem = total & 7, xcd = id & 7;
    uint32_t t = xcd * q + (xcd < rem ? xcd : rem) + (id >> 3);
    const int split = t / (static_cast<uint32_t>(tr) * tc);
    t -= split * static_cast<uint32_t>(tr) * tc;
    const uint32_t panel = t / (4u * tc);
    const int ph = tr - 4 * static_cast<int>(panel) < 4 ? tr - 4 * panel : 4;
    const uint32_t in = t - panel * 4u * tc;
    const int tile_c = in / ph, tile_r = 4 * panel + in % ph;
    const int64_t row0 = int64_t(tile_r) * E, col0 = int64_t(tile_c) * E;

    const int nkt = (K + kDepth - 1) / kDepth;
    // (below 2^31: 2^16 stages, twelve pairs, 16 splits)
    const uint32_t steps = static_cast<uint32_t>(nkt) * a.npair;
    int it0 = 0, n = static_cast<int>(steps);
    if (splits > 1) {
        it0 = static_cast<int>(steps * split / splits);
        n = static_cast<int>(steps * (split + 1) / splits) - it0;
    }

    Stage<E, COLT, WAVES, true> sc;
    Stage<E, ROWT, WAVES, false> sr;
    constexpr bool kGated = OUT == kTileGated || OUT == kTileGatedPart;
    if constexpr (kGated) sc.init_gated(a.col, a.col_duo, col0, a.gated.n, wave, lane);
    else sc.init(a.col, col0, a.ncol, wave, lane);
    sr.init(a.row, row0, nrow, wave, lane);
    const int wr = wave % WR, wc = wave / WR % WC, half = wave / (WR * WC);
    Reader<E, COLT, FC, kWaveGroups> rc;
    Reader<E, ROWT, FR, kWaveGroups> rr;
    rc.init(wc * (E / WC), half * kWaveGroups, lane);
    rr.init(wr * (E / WR), half * kWaveGroups, lane);

    if constexpr (OUT == kTileProb) {
        const ProbArgs &b = a.prob;
        for (int x = threadIdx.x; x < E; x += 64 * WAVES) {
            // rows past the last one up to a multiple of 64 are zeros: they are summed over as they lie
            const int64_t r = row0 + x;
            RowData d{INFINITY, 0.f, 0.f, -1};
            if (r < nrow) {
                const float g = b.weight[r], rest = expm1f(-b.loss[r]);   // the label's probability less one
                d = RowData{b.lse[r], g, g * rest, b.label[r] - b.col0};
                // one term: divided by the label's entry (where that is 0, the row's factor is as well)
                if (b.terms == 1) d = RowData{rest == 0.f ? INFINITY : d.lse + logf(-rest), -1.f, 1.f, d.label};
            }
            rows[x] = d;
        }
    } else if constexpr (OUT == kTileBest) {
        if (a.best.label)
            for (int x = threadIdx.x; x < E; x += 64 * WAVES) rows[x].label = row0 + x < nrow ? a.best.label[row0 + x] : -1;
    }

    if constexpr (kTop) {
        if (a.top.token)
            for (int x = threadIdx.x; x < E; x += 64 * WAVES) {
                const int64_t token = row0 + x < nrow ? a.top.token[row0 + x] : -1;
                rows[x].label = token >= 0 && token < a.ncol ? static_cast<int>(token) : -1;
            }
    }

    f32x16 acc[FC][FR];   // [column fragment][row fragment]
#pragma unroll
    for (int i = 0; i < FC; ++i)
#pragma unroll
        for (int j = 0; j < FR; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

    // where the next stage's contents come from
    struct From {
        const char *c, *r;
        int left, skip;
    };
    int pair = it0 > 0 ? it0 / nkt : 0, kt = it0 - pair * nkt;
    // (second parts are met in a product over both factors of a gated one alone: the other kernels do without the choice)
    constexpr bool kParts = COLT && !ROWT && (OUT == kTilePartial || OUT == kTileTwo);
    auto col_at = [&](int i) {
        if (kParts && i >= a.half) return a.col_duo + col_term(a.half, i - a.half) * a.col.plane;
        return col_term(kParts ? a.half : a.npair, i) * a.col.plane;
    };
    auto row_at = [&](int i) {
        if (kParts && i >= a.half) return a.row_duo + row_term(a.half, i - a.half) * a.row.plane;
        return row_term(kParts ? a.half : a.npair, i) * a.row.plane;
    };
    From next{sc.at_step(col_at(pair), kt), sr.at_step(row_at(pair), kt), K - kt * kDepth, a.skip - kt * kDepth};
    auto advance = [&]() {   // (past the last stage: to addresses that are not read)
        next = From{next.c + sc.stride(), next.r + sr.stride(), next.left - kDepth, next.skip - kDepth};
        if (++kt == nkt) {   // (more than one pair of planes)
            kt = 0;
            ++pair;
            next = From{sc.at_step(col_at(pair), 0), sr.at_step(row_at(pair), 0), K, a.skip};
        }
    };
    constexpr int kLoads = Stage<E, COLT, WAVES, true>::kLoads;   // of either operand
    const uint32_t lds = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_void *)sm)) + wave * kLoads * 1024;
    auto copy = [&](auto i_, int buf) {
        constexpr int i = decltype(i_)::value;
        const uint32_t to = lds + buf * int(sizeof(sm[0]));
        if constexpr (i < kLoads) sc.template copy<i>(next.c, to, next.left, next.skip);
        else sr.template copy<i - kLoads>(next.r, to + kBuf * 16, 0, -1);
    };
    bf16x8 fc[2][FC], fr[2][FR];
    // in the order that products use them: column 0, the rows, the other columns
    auto order = [](int k) { return k == 0 ? 0 : k <= FR ? FC + k - 1 : k - FR; };
    auto read = [&](int x, int buf, int g) {
        if (x < FC) fc[g & 1][x] = rc.get(reinterpret_cast<const char *>(sm[buf]), x, g);
        else fr[g & 1][x - FC] = rr.get(reinterpret_cast<const char *>(sm[buf] + kBuf), x - FC, g);
    };
    constexpr int kProducts = FC * FR, kReads = FC + FR;   // of a group
    // Copies of a stage, in parts: in the last group of the stage whose buffer it takes, where that
    // becomes free, and in the next stage's first group, or two of four.  All at once they would
    // come faster than they are served (64 bytes a cycle), and the products would wait.
    constexpr int kCopies = 2 * kLoads, kPart1 = kCopies * (KS == 1 ? 7 : 8) / 16, kPart2 = KS == 1 ? kPart1 : 0;
    constexpr int kPart0 = kCopies - kPart1 - kPart2;
    // Group g of the stage in buffer `buf`.  Between its products: the reads of the next group (of the
    // last one: the next stage's first, or nothing's where there is none), and, if it has some,
    // a part of a stage's copies.  No product lies in a branch, so that no accumulator is moved.
    auto group = [&](auto g_, int s) {
        constexpr int g = decltype(g_)::value;
        constexpr bool last = g == kWaveGroups - 1;
        constexpr int part = (g + 1) % kWaveGroups;
        const int buf = s % BUFS, after = (s + 1) % BUFS, before = (s + BUFS - 1) % BUFS;
        constexpr int copies_from = part == 0 ? 0 : part == 1 ? kPart0 : kPart0 + kPart1;
        constexpr int count = part == 0 ? kPart0 : part == 1 ? kPart1 : part == 2 ? kPart2 : 0;
        const bool copies = last ? s + BUFS < n : s + BUFS - 1 < n;
        // in the group before the last, after its copies: on to the next stage
        constexpr int kStep = KS == 1 ? kProducts / 2 : kProducts - 1;
        __builtin_amdgcn_sched_barrier(0);
        constexpr int kMeet = kProducts * 6 / 16;   // products before the waves meet, in that group
#pragma unroll
        for (int x = 0; x < kProducts; ++x) {
            mma(fc[g & 1][x / FR], fr[g & 1][x % FR], acc[x / FR][x % FR]);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (last) {
                if (x + 1 == kMeet) {
                    // the next stage has arrived: only later ones' copies may be on their way
                    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((BUFS - 2) * kCopies) : "memory");
                    if (BUFS > 2 && s + BUFS > n) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                    __builtin_amdgcn_s_barrier();
                    asm volatile("" ::: "memory");
                }
            }
            constexpr int from = last ? kMeet - 1 : 0, slots = kProducts - from;
            const int slot = x - from;
            if (slot >= 0) {
#pragma unroll
                for (int k = 0; k < kReads; ++k)
                    if (k * slots / kReads == slot) read(order(k), last ? after : buf, (g + 1) % kWaveGroups);
                if (copies)
                    repeat<count>([&](auto k) {
                        constexpr int v = decltype(k)::value;
                        if (v * slots / count == slot) copy(Int<copies_from + v>{}, last ? buf : before);
                    });
            }
            if (g == kWaveGroups - 2 && x == kStep) advance();
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    if (n > 0) {
        // all of the first stages, and a first part of the one in the last buffer
#pragma unroll
        for (int s = 0; s < BUFS; ++s) {
            if (s >= n) break;
            if (s > 0) advance();
            repeat<kPart0>([&](auto k) { copy(k, s); });
            if (s + 1 < BUFS) repeat<kCopies - kPart0>([&](auto k) { copy(Int<kPart0 + decltype(k)::value>{}, s); });
        }
        if (n >= BUFS) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((BUFS - 2) * kCopies + kPart0) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
#pragma unroll
        for (int x = 0; x < kReads; ++x) read(x, 0, 0);
    }
    for (int s = 0; s < n; ++s) {
        // stage s + BUFS is copied over stage s: from the last group on, through the next stage's first
        group(Int<0>{}, s);
        group(Int<1>{}, s);
        if constexpr (KS == 1) {
            group(Int<2>{}, s);
            group(Int<3>{}, s);
        }
        settle(acc);
    }
    __syncthreads();   // every wave has read the last stage

    // 64 rows of the wave at a time through LDS (a region of its own): consecutive lanes then store
    // consecutive columns, or a lane has a whole row, or four lanes one (kTileTop); quads are permuted by the row, and then by
    // the wave, against bank conflicts.
    constexpr int kCols = E / WC, kQuads = kCols / 4, kRows = 64 / kQuads;   // rows of one pass of the wave
    static_assert(WR * WC * 64 * kCols * 4 <= int(sizeof(sm)), "the waves' regions fit");
    f32x4 *mine = reinterpret_cast<f32x4 *>(sm) + (wave % (WR * WC)) * 64 * kQuads;   // (both halves')
    const int rows_out = OUT == kTileProb ? (nrow + 63) / 64 * 64 : nrow;
    const int col1 = static_cast<int>(col0) + wc * kCols;   // the wave's first column
    const int quad = lane % kQuads, sub = lane / kQuads;
    f32x4 bias = {0.f, 0.f, 0.f, 0.f};
    if constexpr (OUT == kTileStore) bias = load_bias(a.store, col1 + 4 * quad, a.ncol);
    // gated: lanes of eight quads, whose columns are half of the wave's
    const int gate_quad = lane & 7, gate_sub = lane >> 3, gate_col = (col1 >> 1) + 4 * gate_quad;
    f32x4 bias_up = {0.f, 0.f, 0.f, 0.f};
    if constexpr (OUT == kTileGated) {
        bias = gated_bias(a.gated.bias_gate, gate_col, a.gated.n);
        bias_up = gated_bias(a.gated.bias_up, gate_col, a.gated.n);
    }
    auto part = [&](auto j0_) {
        constexpr int j0 = decltype(j0_)::value;
        const int r1 = wr * (E / WR) + 32 * j0;   // the part's first row in the tile
        auto put = [&](bool add) {
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int i = 0; i < FC; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const f32x16 &v = acc[i][j0 + j];
                        f32x4 *to = mine + (32 * j + (lane & 31)) * kQuads + ((8 * i + 2 * e + (lane >> 5)) ^ (lane & 15) ^ (kTop ? 4 * wc : 0));
                        const f32x4 u = {v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]};
                        *to = add ? u + *to : u;
                    }
        };
        // (with kTileTop the waves meet again, so all of them stay)
        const bool live = row0 + r1 < rows_out;
        if constexpr (KS == 1) {
            if (!kTop && !live) return;
            put(false);
            __builtin_amdgcn_wave_barrier();
        } else {
            // the second half's sums, then the first half's added onto them
            if (half == 1) put(false);
            __syncthreads();
            if (half == 0) put(true);
            __syncthreads();
            if (!kTop && !live) return;
        }
        if constexpr (kTop) {
            // four lanes a row of all the waves' columns
            static_assert(64 * WAVES == 4 * 64 * WR && E / WC == 64, "four lanes for each of the part's rows; a wave's columns");
            if constexpr (KS == 1) __syncthreads();
            const TopArgs &b = a.top;
            const int r = threadIdx.x >> 2, s = threadIdx.x & 3, x = r & 63;
            const int tile_row = (r >> 6) * (E / WR) + 32 * j0 + x;
            constexpr int kOcts = E / 32;   // of a lane
            const int w = kOcts == 8 ? s : s >> 1, at = kOcts == 8 ? 0 : 8 * (s & 1), swap = (x & 15) ^ (4 * w);
            f32x4 *row = reinterpret_cast<f32x4 *>(sm) + (((r >> 6) + WR * w) * 64 + x) * kQuads;
            const int mine1 = static_cast<int>(col0) + 8 * kOcts * s;
            const bool counts = row0 + tile_row < nrow;
            if (b.token) {
                const int token = rows[tile_row].label, y = token - mine1;
                if (counts && y >= 0 && y < 8 * kOcts)
                    b.token_logit[row0 + tile_row] = token == b.exclude ? -INFINITY : row[(at + (y >> 2)) ^ swap][y & 3];
            }
            row_top<kOcts>(b, a.ncol, row, at, swap, mine1, lane, counts ? (row0 + tile_row) * b.ngroup + tile_c : -1);
            if constexpr (KS == 1) __syncthreads();   // before the next part's sums take the place
            return;
        }
        if constexpr (OUT == kTileBest) {
            if (half != 0) return;
            const Best m = row_best(a, mine + lane * kQuads, lane & 15, kCols, col1);
            top[wc][r1 + lane] = m.top;
            others[wc][r1 + lane] = m.others;
            at[wc][r1 + lane] = m.at;
            if (a.best.label) {
                const int label = rows[r1 + lane].label, x = label - col1;
                if (x >= 0 && x < kCols && label < a.ncol) {
                    // (the largest value is no longer in its place)
                    const float v = mine[lane * kQuads + ((x >> 2) ^ (lane & 15))][x & 3];
                    a.best.label_logit[row0 + r1 + lane] = label == m.at ? m.top : v;
                }
            }
        } else if constexpr (OUT == kTileGated) {
            static_assert(kCols == 64, "a fragment of either matrix");
            const int most = static_cast<int>(rows_out - row0) - r1;
            // (rows eight apart in a pass: their quads lie in both halves of the banks)
            constexpr int kBatch = 4;
            // Of large tiles, what is kept goes first, one matrix after the other: at sizes of a power of two the three lie at the same places of
            // memory's banks, and stores to them in turn wait for each other (16,384 x 1,024 x 4,096 took 374 us so, 340 one by one, 320 on
            // another card, and 303 where they lie 1 KiB further from each other, as the binding allocates them, and 306 one by one).
            // Rows of other lengths do not meet so and read LDS once: 3,279 x 448 x 1,934 takes 27.4 us, 29.8 one by one, and small
            // tiles 1,000 x 832 x 2,048 13.2 and 13.9.
            const bool first = KS == 1 && a.gated.pre_gate && a.gated.ld_pre % 512 == 0;
            GatedArgs g = a.gated;
            if (first) g.pre_gate = nullptr;
            if (first) {
#pragma unroll
                for (int which = 0; which < 2; ++which) {
#pragma unroll
                    for (int k = 0; k < 8 / KS; ++k) {
                        const int x = half * (8 / KS) + k + 8 * gate_sub;
                        const f32x4 v = mine[x * kQuads + ((gate_quad + 8 * which) ^ (x & 15))] + (which ? bias_up : bias);
                        const int n = a.gated.n - gate_col < 4 ? a.gated.n - gate_col : 4;
                        if (x < most && n > 0)
                            put4(which ? a.gated.pre_up : a.gated.pre_gate, (row0 + r1 + x) * a.gated.ld_pre + gate_col, a.gated.ld_pre, n,
                                 a.gated.pre_bf16, v);
                    }
                }
            }
#pragma unroll
            for (int k0 = 0; k0 < 8 / KS; k0 += kBatch) {
                f32x4 gate[kBatch], up[kBatch];
                const int x0 = half * (8 / KS) + k0 + 8 * gate_sub;
#pragma unroll
                for (int k = 0; k < kBatch; ++k) {
                    const f32x4 *from = mine + (x0 + k) * kQuads;
                    gate[k] = from[gate_quad ^ ((x0 + k) & 15)] + bias;
                    up[k] = from[(gate_quad + 8) ^ ((x0 + k) & 15)] + bias_up;
                }
                gated4(g, gate, up, row0 + r1 + x0, most - x0, gate_col);
            }
        } else if constexpr (OUT == kTileTwo) {
            // (four rows' reads, then their stores)
            const int most = static_cast<int>(rows_out - row0) - r1;
            constexpr int kBatch = 4, kTurns = 64 / KS / kRows;
            static_assert(kTurns % kBatch == 0, "whole batches");
#pragma unroll
            for (int t = 0; t < kTurns; t += kBatch) {
                const int x0 = sub + half * (64 / KS) + t * kRows;
                f32x4 v[kBatch];
#pragma unroll
                for (int k = 0; k < kBatch; ++k) v[k] = mine[(x0 + k * kRows) * kQuads + (quad ^ ((x0 + k * kRows) & 15))];
#pragma unroll
                for (int k = 0; k < kBatch; ++k) {
                    const int x = x0 + k * kRows;
                    if (x < most) store_two(a.store, a.two_out, a.two_rows, a.two_at, v[k], row0 + r1 + x, col1 + 4 * quad, a.ncol);
                }
            }
        } else {
            const int most = static_cast<int>(rows_out - row0) - r1;
#pragma unroll 4
            for (int x = sub + half * (64 / KS); x < (half + 1) * (64 / KS); x += kRows) {
                const f32x4 v = mine[x * kQuads + (quad ^ (x & 15))];
                RowData d{};
                if constexpr (OUT == kTileProb) d = rows[r1 + x];
                if (x < most) tile_quad<OUT>(a, v, bias, d, row0 + r1 + x, col1 + 4 * quad, nrow, split);
            }
        }
        __builtin_amdgcn_wave_barrier();
    };
    part(Int<0>{});
    if constexpr (FR > 2) part(Int<2>{});
    static_assert(FR == 2 || (FR == 4 && KS == 1), "parts of 64 rows, one where the halves meet");
    if constexpr (OUT == kTileBest) {
        __syncthreads();
        for (int x = threadIdx.x; x < E; x += 64 * WAVES) {
            if (row0 + x >= nrow) continue;
            Best m{top[0][x], others[0][x], at[0][x]};
#pragma unroll
            for (int w = 1; w < WC; ++w) m = merge(m, Best{top[w][x], others[w][x], at[w][x]});
            const int64_t o = (row0 + x) * a.best.ntile + tile_c;
            a.best.top[o] = m.top;
            a.best.others[o] = m.others;
            a.best.at[o] = m.at;
        }
    }
}

template <bool ROWT, bool COLT, int OUT>
hipError_t launch_one(const TileArgs &a, dim3 g, hipStream_t s) {
    // Small tiles that leave a CU one workgroup take four buffers, so that copies have three stages to
    // arrive (a stage of theirs is 512 cycles of products).
    if (a.big) hipLaunchKernelGGL((bdlm_tile_kernel<256, 2, 4, 1, 2, ROWT, COLT, OUT>), g, dim3(kTileThreads), 0, s, a);
    else if (g.x <= static_cast<unsigned>(kChip))
        hipLaunchKernelGGL((bdlm_tile_kernel<128, 2, 2, 2, 4, ROWT, COLT, OUT>), g, dim3(kTileThreads), 0, s, a);
    else hipLaunchKernelGGL((bdlm_tile_kernel<128, 2, 2, 2, 2, ROWT, COLT, OUT>), g, dim3(kTileThreads), 0, s, a);
    return hipGetLastError();
}

// out = epilogue(sum of the slices), four columns per thread
__global__ void __launch_bounds__(256) bdlm_join_kernel(const float *part, int splits, int edge, int nrow, int ncol,
                                                        const int32_t *nrow_dev, const float *scale, const StoreArgs s) {
    const int quads = (ncol + 3) / 4;
    const int64_t rows = nrow_dev ? *nrow_dev : nrow;
    const int64_t slice = (splits ? int64_t(nrow) : rows) * ncol;
    if (splits == 0) splits = split_count(((rows + edge - 1) / edge) * ((ncol + edge - 1) / edge));
    for (int64_t x = blockIdx.x * int64_t(256) + threadIdx.x; x < rows * quads; x += gridDim.x * int64_t(256)) {
        const int64_t r = x / quads;
        const int c = static_cast<int>(x - r * quads) * 4;
        const float *p = part + r * ncol + c;
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
        if (c + 4 <= ncol) {
            v = sum_slices(p, slice, splits);
        } else {
            for (int k = 0; k < splits; ++k)
                for (int e = 0; e < 4; ++e)
                    if (c + e < ncol) v[e] += p[k * slice + e];
        }
        if (scale) v *= scale[r];
        store4(s, v, load_bias(s, c, ncol), r, c, ncol);
    }
}

__global__ void __launch_bounds__(256) bdlm_join_two_kernel(const float *part, int splits, int nrow, int ncol, void *two_out,
                                                            int two_rows, int two_at, const StoreArgs s) {
    const int quads = (ncol + 3) / 4;
    const int64_t slice = int64_t(nrow) * ncol, all = int64_t(nrow) * quads;
    for (int64_t x = blockIdx.x * int64_t(256) + threadIdx.x; x < all; x += gridDim.x * int64_t(256)) {
        const int64_t r = x / quads;
        const int c = static_cast<int>(x - r * quads) * 4;
        const float *p = part + r * ncol + c;
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
        if (c + 4 <= ncol) {
            v = sum_slices(p, slice, splits);
        } else {
            for (int k = 0; k < splits; ++k)
                for (int e = 0; e < 4; ++e)
                    if (c + e < ncol) v[e] += p[k * slice + e];
        }
        store_two(s, two_out, two_rows, two_at, v, r, c, ncol);
    }
}

__global__ void __launch_bounds__(256) bdlm_join_gated_kernel(const float *part, int splits, int nrow, const GatedArgs g) {
    const int quads = (g.n + 3) / 4;
    const int64_t ncol = int64_t(g.n + 31) / 32 * 64, slice = nrow * ncol, all = int64_t(nrow) * quads;
    for (int64_t x = blockIdx.x * int64_t(256) + threadIdx.x; x < all; x += gridDim.x * int64_t(256)) {
        const int64_t r = x / quads;
        const int c = static_cast<int>(x - r * quads) * 4;
        const float *p = part + r * ncol + (c >> 5) * 64 + (c & 31);
        const f32x4 gate = sum_slices(p, slice, splits), up = sum_slices(p + 32, slice, splits);
        f32x4 both[2][1] = {{gate + gated_bias(g.bias_gate, c, g.n)}, {up + gated_bias(g.bias_up, c, g.n)}};
        gated4(g, both[0], both[1], r, 1, c);
    }
}

}  // namespace

int launch_tile(const TileArgs &a, void *stream) {
    if (a.nrow <= 0 || a.ncol <= 0) return BDLM_OK;
    const int64_t e = tile_edge(a.big);
    int64_t tiles = ((a.nrow + e - 1) / e) * ((a.ncol + e - 1) / e);
    // (splits 0: fewer rows make more splits, never more than the chip holds)
    tiles = a.splits ? tiles * a.splits : tiles > kChip ? tiles : kChip;
    const dim3 g(static_cast<unsigned>(tiles));
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t r = hipErrorInvalidValue;
    const int lay = (a.row_t ? 2 : 0) + (a.col_t ? 1 : 0);   // 0: both contiguous, 1: col, 3: both slow
    if (a.out == kTileStore) {
        if (lay == 0) r = launch_one<false, false, kTileStore>(a, g, s);
        else if (lay == 1) r = launch_one<false, true, kTileStore>(a, g, s);
        else if (lay == 3) r = launch_one<true, true, kTileStore>(a, g, s);
    } else if (a.out == kTilePartial) {
        if (lay == 0) r = launch_one<false, false, kTilePartial>(a, g, s);
        else if (lay == 1) r = launch_one<false, true, kTilePartial>(a, g, s);
        else if (lay == 3) r = launch_one<true, true, kTilePartial>(a, g, s);
    } else if (a.out == kTileTwo) {
        if (lay == 3) r = launch_one<true, true, kTileTwo>(a, g, s);
        else if (lay == 1) r = launch_one<false, true, kTileTwo>(a, g, s);
    } else if (lay == 0) {
        if (a.out == kTileBest) r = launch_one<false, false, kTileBest>(a, g, s);
        else if (a.out == kTileProb) r = launch_one<false, false, kTileProb>(a, g, s);
        else if (a.out == kTileGated) r = launch_one<false, false, kTileGated>(a, g, s);
        else if (a.out == kTileTop) r = launch_one<false, false, kTileTop>(a, g, s);
        else if (a.out == kTileGatedPart) r = launch_one<false, false, kTileGatedPart>(a, g, s);
    }
    return r == hipSuccess ? BDLM_OK : BDLM_E_LAUNCH;
}

int launch_join(const float *part, int32_t splits, int32_t big, int32_t nrow, int32_t ncol, const int32_t *nrow_dev,
                const float *scale, const StoreArgs &s, void *stream) {
    if (nrow <= 0 || ncol <= 0) return BDLM_OK;
    const int64_t blocks = (int64_t(nrow) * ((ncol + 3) / 4) + 255) / 256;
    const dim3 g(static_cast<unsigned>(blocks < 8192 ? blocks : 8192));
    hipLaunchKernelGGL(bdlm_join_kernel, g, dim3(256), 0, static_cast<hipStream_t>(stream), part, splits,
                       tile_edge(big), nrow, ncol, nrow_dev, scale, s);
    return hipGetLastError() == hipSuccess ? BDLM_OK : BDLM_E_LAUNCH;
}

int launch_join_two(const float *part, int32_t splits, int32_t nrow, int32_t ncol, void *two_out, int32_t two_rows,
                    int32_t two_at, const StoreArgs &s, void *stream) {
    if (nrow <= 0 || ncol <= 0) return BDLM_OK;
    const int64_t blocks = (int64_t(nrow) * ((ncol + 3) / 4) + 255) / 256;
    hipLaunchKernelGGL(bdlm_join_two_kernel, dim3(static_cast<unsigned>(blocks < 8192 ? blocks : 8192)), dim3(256), 0,
                       static_cast<hipStream_t>(stream), part, splits, nrow, ncol, two_out, two_rows, two_at, s);
    return hipGetLastError() == hipSuccess ? BDLM_OK : BDLM_E_LAUNCH;
}

int launch_join_gated(const float *part, int32_t splits, int32_t nrow, const GatedArgs &g, void *stream) {
    if (nrow <= 0 || g.n <= 0) return BDLM_OK;
    const int64_t blocks = (int64_t(nrow) * ((g.n + 3) / 4) + 255) / 256;
    hipLaunchKernelGGL(bdlm_join_gated_kernel, dim3(static_cast<unsigned>(blocks < 8192 ? blocks : 8192)), dim3(256), 0,
                       static_cast<hipStream_t>(stream), part, splits, nrow, g);
    return hipGetLastError() == hipSuccess ? BDLM_OK : BDLM_E_LAUNCH;
}

}  // namespace bdlm
