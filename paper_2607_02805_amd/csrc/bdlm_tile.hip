// bdlm_tile.hip -- gfx950 tiled matrix products of the dense operators: acc[row][col] = sum over k
// of row(row, k) * col(col, k) in bf16 terms with fp32 accumulation, and what becomes of a tile
// (bdlm_dense.h: the epilogue of a projection, partial sums, softmax records, loss gradients).
//
// One workgroup per tile (and split).  The operands go straight from memory to LDS in 16-byte
// pieces, 64 contraction indices at a time into one of two buffers: while a buffer is multiplied
// the next one fills.  `col` is the first MFMA operand, so a lane holds four consecutive
// columns of one row and stores them together.
//
// An operand whose contraction index is contiguous lies in LDS as [row][64] (eight pieces a
// row) and is read 16 bytes a lane; one whose contraction index is the slow one lies as
// [64][row] and is read with the LDS transpose read.  Both are permuted by the piece so that a
// quarter wave meets every bank once; as the copy writes LDS in lane order, the permutation
// is of the addresses in memory that the lanes read.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "bdlm.h"
#include "bdlm_dense.h"
#include "bdlm_dense_device.h"
#include "bdlm_store.h"

namespace bdlm {
namespace {

constexpr int kDepth = 64;   // contraction indices per buffer

typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(1))) const void g_void;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

__device__ __forceinline__ void copy16(const char *from, uint4 *to) {
    __builtin_amdgcn_global_load_lds((g_void *)from, (lds_void *)to, 16, 0, 0);
}
__device__ __forceinline__ bf16x8 frag(const char *lds) {
    return __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4 *>(lds));
}
__device__ __forceinline__ s16x4 read_tr(const char *lds) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(const_cast<char *>(lds)));
}
__device__ __forceinline__ f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// One operand's share of a tile: R rows (or columns) from `first` on, 64 indices deep.
template <int R, bool T, int WAVES>
struct Stage {
    static constexpr int kPieces = R * kDepth / 8;        // 16-byte pieces of a buffer
    static constexpr int kLoads = kPieces / (64 * WAVES);   // per lane
    static_assert(kLoads * 64 * WAVES == kPieces, "whole loads");
    const char *base;      // the operand at (first, 0) of its first plane
    int64_t ld2;           // bytes of a row
    uint32_t off[kLoads];    // this lane's bytes from base
    int32_t at[kLoads];      // contraction index of the piece within the buffer

    // rows past the operand's end repeat its last row, columns past it its first piece
    __device__ __forceinline__ void init(const Mat &m, int64_t first, int64_t size, int wave, int lane) {
        ld2 = m.ld * 2;
        base = reinterpret_cast<const char *>(m.p) + (T ? first * 2 : first * ld2);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int piece = (i * WAVES + wave) * 64 + lane;
            if constexpr (T) {
                constexpr int kRow = R / 8;
                const int t = piece / kRow, pos = piece % kRow;
                int c = pos ^ (2 * ((t & 3) | (((t >> 3) & 1) << 2)));
                if (first + 8 * c >= size) c = 0;
                at[i] = t;
                off[i] = static_cast<uint32_t>(t * ld2 + c * 16);
            } else {
                const int r = piece >> 3, c = (piece & 7) ^ ((r >> 1) & 7);
                const int64_t rr = first + r < size ? r : size - 1 - first;
                at[i] = 8 * c;
                off[i] = static_cast<uint32_t>(rr * ld2 + c * 16);
            }
        }
    }
    // left: contraction indices from this buffer's first to the operand's end
    __device__ __forceinline__ void load(uint4 *lds, int64_t plane, int kt, int left, int wave) const {
        const char *p = base + plane * 2 + (T ? kt * (kDepth * ld2) : kt * int64_t(2 * kDepth));
        if (left >= kDepth) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) copy16(p + off[i], lds + (i * WAVES + wave) * 64);
        } else {
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
                copy16(at[i] < left ? p + off[i] : reinterpret_cast<const char *>(&kZeroChunk),
                       lds + (i * WAVES + wave) * 64);
        }
    }
};

// Operand reads: fragment i (16 rows from `row0` + 16 i) of k step s (32 indices).
template <int R, bool T, int F>
struct Reader {
    int off[T ? F : 2];
    __device__ __forceinline__ void init(int row0, int lane) {
        const int kg = lane >> 4, s = lane & 15;
        if constexpr (T) {
            const int t = 8 * kg + (s >> 2);
            const int f = 2 * ((t & 3) | (((t >> 3) & 1) << 2));
#pragma unroll
            for (int i = 0; i < F; ++i) {
                const int c = row0 / 8 + 2 * i + ((s & 3) >> 1);
                off[i] = (t * (R / 8) + (c ^ f)) * 16 + (s & 1) * 8;
            }
        } else {
#pragma unroll
            for (int k = 0; k < 2; ++k) off[k] = (row0 + s) * 128 + (((4 * k + kg) ^ ((s >> 1) & 7)) * 16);
        }
    }
    __device__ __forceinline__ bf16x8 get(const char *lds, int i, int k) const {
        if constexpr (T) {
            const char *p = lds + off[i] + k * (32 * 2 * R);
            const s16x4 a = read_tr(p), b = read_tr(p + 4 * 2 * R);
            return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            return frag(lds + off[k] + i * (16 * 128));
        }
    }
};

// Plane pairs in order of weight: pair i multiplies term kRowTerm[i] of `row` and kColTerm[i] of
// `col`.  Three pairs: an fp32 row operand (gradients of the logits) with a bf16 one.
__device__ __forceinline__ int row_term(int npair, int i) { return npair == 6 ? (0x010210 >> (4 * i)) & 15 : i; }
__device__ __forceinline__ int col_term(int npair, int i) { return npair == 6 ? (0x102010 >> (4 * i)) & 15 : 0; }

// Four columns of one row of a tile, in its place.
template <int OUT>
__device__ __forceinline__ void tile_quad(const TileArgs &a, f32x4 v, int64_t r, int c, int split) {
    if constexpr (OUT == kTileStore) {
        store4(a.store, v, r, c, a.ncol);
    } else if constexpr (OUT == kTilePartial) {
        float *to = a.part + (int64_t(split) * a.nrow + r) * a.ncol + c;
        if (c + 4 <= a.ncol && a.ncol % 4 == 0) {
            if (a.add) v += *reinterpret_cast<const f32x4 *>(to);
            *reinterpret_cast<f32x4 *>(to) = v;
        } else {
            for (int e = 0; e < 4; ++e)
                if (c + e < a.ncol) to[e] = a.add ? to[e] + v[e] : v[e];
        }
    } else {
        const ProbArgs &b = a.prob;
        if (c >= b.width) return;
        const float lse = b.lse[r], g = b.weight[r];
        const int label = b.label[r] - b.col0, exclude = b.exclude - b.col0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float x = v[e] - lse;
            v[e] = g * (b.terms == 1 ? __expf(x) : expf(x));
            // the label's probability less one is exp(-loss) - 1, without cancellation
            if (c + e == label) v[e] = g * expm1f(-b.loss[r]);
            if (c + e >= a.ncol || c + e == exclude) v[e] = 0.f;
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
                *reinterpret_cast<uint2 *>(to + k * b.plane) =
                    uint2{h[0][k] | uint32_t(h[1][k]) << 16, h[2][k] | uint32_t(h[3][k]) << 16};
        }
    }
}

template <int E, int WR, int WC, bool ROWT, bool COLT, int OUT>
__global__ void __launch_bounds__(64 * WR * WC) bdlm_tile_kernel(const TileArgs a) {
    constexpr int WAVES = WR * WC;
    constexpr int FR = E / WR / 16, FC = E / WC / 16;   // fragments of a wave
    constexpr int kBuf = E * kDepth / 8;                 // pieces of an operand's buffer
    __shared__ uint4 sm[2][2 * kBuf];                    // [buffer][col, then row]
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int nrow = a.nrow_dev ? *a.nrow_dev : a.nrow;
    const int K = a.k_dev ? *a.k_dev : a.k;
    const int tr = (nrow + E - 1) / E, tc = (a.ncol + E - 1) / E;
    // Consecutive workgroups go to the eight XCDs in turn: each XCD takes a run of the tile
    // order, four tile rows by all columns at a time, so that the tiles that run together on it
    // share rows and columns in its L2.
    const uint32_t total = static_cast<uint32_t>(tr) * tc * a.splits;
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
    const int steps = nkt * a.npair;
    const int it0 = static_cast<int>(int64_t(steps) * split / a.splits);
    const int it1 = static_cast<int>(int64_t(steps) * (split + 1) / a.splits);

    Stage<E, COLT, WAVES> sc;
    Stage<E, ROWT, WAVES> sr;
    sc.init(a.col, col0, a.ncol, wave, lane);
    sr.init(a.row, row0, nrow, wave, lane);
    const int wr = wave % WR, wc = wave / WR;
    Reader<E, COLT, FC> rc;
    Reader<E, ROWT, FR> rr;
    rc.init(wc * (E / WC), lane);
    rr.init(wr * (E / WR), lane);

    f32x4 acc[FC][FR];
#pragma unroll
    for (int i = 0; i < FC; ++i)
#pragma unroll
        for (int j = 0; j < FR; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    int pair = it0 / (nkt > 0 ? nkt : 1), kt = it0 - pair * nkt;
    auto fill = [&](int buf) {
        const int left = K - kt * kDepth;
        sc.load(sm[buf], col_term(a.npair, pair) * a.col.plane, kt, left, wave);
        sr.load(sm[buf] + kBuf, row_term(a.npair, pair) * a.row.plane, kt, left, wave);
        if (++kt == nkt) {
            kt = 0;
            ++pair;
        }
    };
    if (it0 < it1) fill(0);
    for (int it = it0; it < it1; ++it) {
        const int buf = (it - it0) & 1;
        // this buffer's copies have landed in every wave, and every wave is done with the other
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (it + 1 < it1) fill(buf ^ 1);
        const char *lc = reinterpret_cast<const char *>(sm[buf]);
        const char *lr = reinterpret_cast<const char *>(sm[buf] + kBuf);
#pragma unroll
        for (int k = 0; k < kDepth / 32; ++k) {
            bf16x8 fc[FC], fr[FR];
#pragma unroll
            for (int i = 0; i < FC; ++i) fc[i] = rc.get(lc, i, k);
#pragma unroll
            for (int j = 0; j < FR; ++j) fr[j] = rr.get(lr, j, k);
#pragma unroll
            for (int i = 0; i < FC; ++i)
#pragma unroll
                for (int j = 0; j < FR; ++j) acc[i][j] = mma(fc[i], fr[j], acc[i][j]);
        }
    }

    // lane: row r0 + 16 j, columns c0 + 16 i .. + 3
    const int64_t r0 = row0 + wr * (E / WR) + (lane & 15);
    const int c0 = static_cast<int>(col0) + wc * (E / WC) + 4 * (lane >> 4);
    __syncthreads();   // every wave has read the last buffer
    if constexpr (OUT == kTileBest) {
        const BestArgs &b = a.best;
        float *top = reinterpret_cast<float *>(sm[0]);   // [WC][E], then others, at
        float *oth = top + WC * E;
        int *at = reinterpret_cast<int *>(oth + WC * E);
#pragma unroll
        for (int j = 0; j < FR; ++j) {
            const int64_t r = r0 + 16 * j;
            const int label = b.label && r < nrow ? b.label[r] : -1;
            Best m{-INFINITY, 0.f, kNoColumn};
#pragma unroll
            for (int i = 0; i < FC; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int c = c0 + 16 * i + e;
                    if (c >= a.ncol || c == b.exclude) acc[i][j][e] = -INFINITY;
                    else if (beats(acc[i][j][e], c, m)) m.top = acc[i][j][e], m.at = c;
                    if (c == label) b.label_logit[r] = acc[i][j][e];
                }
            // the four lane groups of a row
#pragma unroll
            for (int d = 16; d < 64; d *= 2) {
                const float v = __shfl_xor(m.top, d, 64);
                const int w = __shfl_xor(m.at, d, 64);
                if (beats(v, w, m)) m.top = v, m.at = w;
            }
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < FC; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (c0 + 16 * i + e != m.at) s += share(acc[i][j][e], m.top);
            s += __shfl_xor(s, 16, 64);
            s += __shfl_xor(s, 32, 64);
            if (lane < 16) {
                const int x = wc * E + wr * (E / WR) + 16 * j + lane;
                top[x] = m.top;
                oth[x] = s;
                at[x] = m.at;
            }
        }
        __syncthreads();
        for (int x = threadIdx.x; x < E; x += 64 * WAVES) {
            if (row0 + x >= nrow) continue;
            Best m{top[x], oth[x], at[x]};
#pragma unroll
            for (int w = 1; w < WC; ++w) m = merge(m, Best{top[w * E + x], oth[w * E + x], at[w * E + x]});
            const int64_t o = (row0 + x) * b.ntile + tile_c;
            b.top[o] = m.top;
            b.others[o] = m.others;
            b.at[o] = m.at;
        }
    } else {
        // Sixteen rows at a time through LDS (a region of the wave's own), so that whole rows of
        // the wave's columns are stored by consecutive lanes.
        constexpr int kCols = E / WC, kPitch = kCols + 4, kQuads = kCols / 4;
        static_assert(WAVES * 16 * kPitch * 4 <= int(sizeof(sm)), "the waves' regions fit");
        float *mine = reinterpret_cast<float *>(sm) + wave * 16 * kPitch;
        const int64_t wrow0 = row0 + wr * (E / WR);
        const int wcol0 = static_cast<int>(col0) + wc * kCols;
#pragma unroll
        for (int j = 0; j < FR; ++j) {
            if (wrow0 + 16 * j >= nrow) break;
#pragma unroll
            for (int i = 0; i < FC; ++i)
                *reinterpret_cast<f32x4 *>(mine + (lane & 15) * kPitch + 16 * i + 4 * (lane >> 4)) = acc[i][j];
            __builtin_amdgcn_wave_barrier();
#pragma unroll 1
            for (int x = lane; x < 16 * kQuads; x += 64) {
                const int64_t r = wrow0 + 16 * j + x / kQuads;
                const int c = wcol0 + x % kQuads * 4;
                if (r < nrow) tile_quad<OUT>(a, *reinterpret_cast<const f32x4 *>(mine + x / kQuads * kPitch + x % kQuads * 4), r, c, split);
            }
            __builtin_amdgcn_wave_barrier();
        }
    }
}

template <bool ROWT, bool COLT, int OUT>
hipError_t launch_one(const TileArgs &a, dim3 g, hipStream_t s) {
    if (a.big) hipLaunchKernelGGL((bdlm_tile_kernel<256, 2, 4, ROWT, COLT, OUT>), g, dim3(512), 0, s, a);
    else hipLaunchKernelGGL((bdlm_tile_kernel<128, 2, 2, ROWT, COLT, OUT>), g, dim3(256), 0, s, a);
    return hipGetLastError();
}

// out = epilogue(sum of the slices), four columns per thread
__global__ void __launch_bounds__(256) bdlm_join_kernel(const float *part, int splits, int nrow, int ncol,
                                                        const int32_t *nrow_dev, const StoreArgs s) {
    const int quads = (ncol + 3) / 4;
    const int64_t rows = nrow_dev ? *nrow_dev : nrow;
    const int64_t slice = int64_t(nrow) * ncol;
    for (int64_t x = blockIdx.x * int64_t(256) + threadIdx.x; x < rows * quads; x += gridDim.x * int64_t(256)) {
        const int64_t r = x / quads;
        const int c = static_cast<int>(x - r * quads) * 4;
        const float *p = part + r * ncol + c;
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
        if (ncol % 4 == 0) {
            for (int k = 0; k < splits; ++k) v += *reinterpret_cast<const f32x4 *>(p + k * slice);
        } else {
            for (int k = 0; k < splits; ++k)
                for (int e = 0; e < 4; ++e)
                    if (c + e < ncol) v[e] += p[k * slice + e];
        }
        store4(s, v, r, c, ncol);
    }
}

}  // namespace

int launch_tile(const TileArgs &a, void *stream) {
    if (a.nrow <= 0 || a.ncol <= 0) return BDLM_OK;
    const int64_t e = tile_edge(a.big);
    const int64_t tiles = ((a.nrow + e - 1) / e) * ((a.ncol + e - 1) / e) * a.splits;
    if (tiles > (int64_t(1) << 30)) return BDLM_E_SHAPE;
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
    } else if (lay == 0) {
        r = a.out == kTileBest ? launch_one<false, false, kTileBest>(a, g, s)
                               : launch_one<false, false, kTileProb>(a, g, s);
    }
    return r == hipSuccess ? BDLM_OK : BDLM_E_LAUNCH;
}

int launch_join(const float *part, int32_t splits, int32_t nrow, int32_t ncol, const int32_t *nrow_dev,
                const StoreArgs &s, void *stream) {
    if (nrow <= 0 || ncol <= 0) return BDLM_OK;
    const int64_t blocks = (int64_t(nrow) * ((ncol + 3) / 4) + 255) / 256;
    const dim3 g(static_cast<unsigned>(blocks < 8192 ? blocks : 8192));
    hipLaunchKernelGGL(bdlm_join_kernel, g, dim3(256), 0, static_cast<hipStream_t>(stream), part, splits, nrow,
                       ncol, nrow_dev, s);
    return hipGetLastError() == hipSuccess ? BDLM_OK : BDLM_E_LAUNCH;
}

}  // namespace bdlm
