// bdlm_skinny.hip -- gfx950 products of few rows (a single token, a small step) with a weight
// matrix: out[row][col] = sum over k of x[row][k] * w[col][k], at most 64 rows.
//
// Bound by the weights' bytes: every weight is read once, straight into the registers that the
// matrix instructions take it from (one row over 50,257 x 1,024 in bf16: 22.6 us with the launch,
// 4.56 TB/s; 4,384 x 1,024: 4.8 us, the launch).  A workgroup owns 16 or 32 columns; its waves share out the
// contraction in runs of 128 indices, so that a wave has 4 or 8 loads of 16 bytes a lane in flight
// and four lanes read 256 contiguous bytes of a weight row.  x is small and comes from the caches.
// The waves' partial tiles meet in LDS, in a fixed order.
//
// fp32: both operands are split in registers into three bf16 terms, six products each
// (bdlm_dense.h).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "bdlm.h"
#include "bdlm_dense.h"
#include "bdlm_dense_device.h"
#include "bdlm_store.h"

namespace bdlm {
namespace {

constexpr int kRun = 128;    // contraction indices of a wave's turn
constexpr int kSteps = kRun / 32;

// Eight consecutive elements from index k of a row of length K, as bf16 terms; zeros past K.
template <bool BF16>
struct Piece;
template <>
struct Piece<true> {
    u32x4 v;
    __device__ __forceinline__ void load(const void *row, int k, int K, bool whole) {
        const uint16_t *p = static_cast<const uint16_t *>(row) + k;
        if (whole || k + 8 <= K) {
            v = *(const __attribute__((address_space(1))) u32x4_a2 *)p;
        } else {
            uint32_t h[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) h[e] = k + e < K ? p[e] : 0u;
            v = u32x4{h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16};
        }
    }
    __device__ __forceinline__ void terms(bf16x8 (&t)[1]) const { t[0] = __builtin_bit_cast(bf16x8, v); }
};
template <>
struct Piece<false> {
    float f[8];
    __device__ __forceinline__ void load(const void *row, int k, int K, bool whole) {
        const float *p = static_cast<const float *>(row) + k;
        if (whole || k + 8 <= K) {
            const u32x4 a = *(const __attribute__((address_space(1))) u32x4_a4 *)p;
            const u32x4 b = *(const __attribute__((address_space(1))) u32x4_a4 *)(p + 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) f[e] = __uint_as_float(a[e]), f[4 + e] = __uint_as_float(b[e]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = k + e < K ? p[e] : 0.f;
        }
    }
    __device__ __forceinline__ void terms(bf16x8 (&t)[3]) const {
        s16x8 s[3];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            uint16_t h[3];
            split_terms(f[e], h);
#pragma unroll
            for (int k = 0; k < 3; ++k) s[k][e] = static_cast<short>(h[k]);
        }
#pragma unroll
        for (int k = 0; k < 3; ++k) t[k] = __builtin_bit_cast(bf16x8, s[k]);
    }
};

__device__ __forceinline__ f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// MT: tiles of 16 rows; G: groups of 16 columns.  Lane: weight column (lane & 15) of a group, or row (lane & 15) of x.
template <int MT, int G, bool BF16, int OUT>
__global__ void __launch_bounds__(BF16 ? 1024 : 512) bdlm_skinny_kernel(const SkinnyArgs a) {
    constexpr int kCols = 16 * G;
    constexpr int TERMS = BF16 ? 1 : 3;
    constexpr int kPitch = kCols + 4;                // floats of a row of sums
    extern __shared__ float part[];                        // [waves][16 MT][kPitch]
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int waves = blockDim.x >> 6;
    const int s = lane & 15, kg = lane >> 4;
    // gated: group 0 is 16 columns of the gate's weights, group 1 the same of the other's
    constexpr bool kGated = OUT == kTileGated;
    static_assert(!kGated || G == 2, "a group of either matrix");
    const int col0 = blockIdx.x * (kGated ? 16 : kCols);
    const int esz = BF16 ? 2 : 4;
    const int nrow = a.nrow_dev ? *a.nrow_dev : a.nrow;
    if (nrow <= 0) return;
    const char *wrow[G], *xrow[MT];
#pragma unroll
    for (int g = 0; g < G; ++g) {
        const int c = col0 + (kGated ? 0 : 16 * g) + s;
        wrow[g] = static_cast<const char *>(kGated && g == 1 ? a.w2 : a.w) + int64_t(c < a.ncol ? c : a.ncol - 1) * a.ldw * esz;
    }
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const int r = 16 * m + s;
        const int rr = r < nrow ? r : nrow - 1;
        xrow[m] = static_cast<const char *>(a.x) + int64_t(a.row_of ? a.row_of[rr] : rr) * a.ldx * esz;
    }
    f32x4 acc[G][MT];
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[g][m] = f32x4{0.f, 0.f, 0.f, 0.f};

    auto run = [&](int k0, bool whole) {
        Piece<BF16> w[G][kSteps];
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int u = 0; u < kSteps; ++u) w[g][u].load(wrow[g], k0 + 32 * u + 8 * kg, a.k, whole);
#pragma unroll
        for (int u = 0; u < kSteps; ++u) {
            bf16x8 wt[G][TERMS];
#pragma unroll
            for (int g = 0; g < G; ++g) w[g][u].terms(wt[g]);
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                Piece<BF16> x;
                x.load(xrow[m], k0 + 32 * u + 8 * kg, a.k, whole);
                bf16x8 xt[TERMS];
                x.terms(xt);
#pragma unroll
                for (int g = 0; g < G; ++g)
#pragma unroll
                    for (int i = 0; i < TERMS; ++i)
#pragma unroll
                        for (int j = 0; j + i < TERMS; ++j) acc[g][m] = mma(wt[g][i], xt[j], acc[g][m]);
            }
        }
    };
    for (int k0 = wave * kRun; k0 < a.k; k0 += waves * kRun) {
        if (k0 + kRun <= a.k) run(k0, true);
        else run(k0, false);
    }

    // lane: row 16 m + s, columns 16 g + 4 kg .. + 3
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int m = 0; m < MT; ++m)
            *reinterpret_cast<f32x4 *>(part + (wave * 16 * MT + 16 * m + s) * kPitch + 16 * g + 4 * kg) = acc[g][m];
    __syncthreads();
    if constexpr (kGated) {
        for (int x = threadIdx.x; x < 16 * MT * 4; x += blockDim.x) {
            const int r = x >> 2, c = (x & 3) * 4;
            f32x4 gate[1] = {gated_bias(a.gated.bias_gate, col0 + c, a.gated.n)}, up[1] = {gated_bias(a.gated.bias_up, col0 + c, a.gated.n)};
            for (int w = 0; w < waves; ++w) {
                const float *p = part + (w * 16 * MT + r) * kPitch + c;
                gate[0] += *reinterpret_cast<const f32x4 *>(p);
                up[0] += *reinterpret_cast<const f32x4 *>(p + 16);
            }
            gated4(a.gated, gate, up, r, nrow - r, col0 + c);
        }
        return;
    }
    constexpr int kQuads = kCols / 4;
    for (int x = threadIdx.x; x < 16 * MT * kQuads; x += blockDim.x) {
        const int r = x / kQuads, c = x % kQuads * 4;
        f32x4 v = *reinterpret_cast<const f32x4 *>(part + r * kPitch + c);
        for (int w = 1; w < waves; ++w) v += *reinterpret_cast<const f32x4 *>(part + (w * 16 * MT + r) * kPitch + c);
        if constexpr (OUT == kTileTop) {
            // kQuads consecutive lanes hold a row's columns
            const TopArgs &b = a.top;
            const int64_t token = b.token && r < nrow ? b.token[r] : -1;
            float top = -INFINITY;
            int at = kNoColumn;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int col = col0 + c + e;
                if (col >= a.ncol || col == b.exclude) v[e] = -INFINITY;
                if (v[e] > top) top = v[e], at = col;
                if (col < a.ncol && col == token) b.token_logit[r] = v[e];
            }
            if (b.list > 0 && r < nrow)
                *reinterpret_cast<f32x4 *>(b.value + (int64_t(r) * b.ngroup + blockIdx.x) * kCols + c) = v;
#pragma unroll
            for (int d = 1; d < kQuads; d *= 2) {
                const float t = __shfl_xor(top, d, 64);
                const int w = __shfl_xor(at, d, 64);
                if (t > top || (t == top && w < at)) top = t, at = w;
            }
            const float ref = top == -INFINITY ? 0.f : top;
            float sum = 0.f, slope = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (col0 + c + e == at) continue;
                const float s = __builtin_amdgcn_exp2f((v[e] - ref) * kLog2e);
                sum += s;
                slope += slope_of(s, v[e] - ref);
            }
#pragma unroll
            for (int d = 1; d < kQuads; d *= 2) sum += __shfl_xor(sum, d, 64), slope += __shfl_xor(slope, d, 64);
            if (c == 0 && r < nrow) {
                const int64_t o = int64_t(r) * b.ngroup + blockIdx.x;
                b.top[o] = top;
                b.others[o] = sum;
                b.slope[o] = slope;
            }
        } else if constexpr (OUT == kTileStore) {
            if (r < nrow) store4(a.store, v, load_bias(a.store, col0 + c, a.ncol), r, col0 + c, a.ncol);
        } else {
            // kQuads consecutive lanes hold a row's columns
            const BestArgs &b = a.best;
            const int label = b.label && r < nrow ? b.label[r] : -1;
            Best m{-INFINITY, 0.f, kNoColumn};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int col = col0 + c + e;
                if (col >= a.ncol || col == b.exclude) v[e] = -INFINITY;
                else if (beats(v[e], col, m)) m.top = v[e], m.at = col;
                if (col == label) b.label_logit[r] = v[e];
            }
#pragma unroll
            for (int d = 1; d < kQuads; d *= 2) {
                const float t = __shfl_xor(m.top, d, 64);
                const int w = __shfl_xor(m.at, d, 64);
                if (beats(t, w, m)) m.top = t, m.at = w;
            }
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (col0 + c + e != m.at) sum += share(v[e], m.top);
#pragma unroll
            for (int d = 1; d < kQuads; d *= 2) sum += __shfl_xor(sum, d, 64);
            if (c == 0 && r < nrow) {
                const int64_t o = int64_t(r) * b.ntile + blockIdx.x;
                b.top[o] = m.top;
                b.others[o] = sum;
                b.at[o] = m.at;
            }
        }
    }
}

template <int MT, int G, bool BF16>
hipError_t launch_cols_of(const SkinnyArgs &a, hipStream_t s) {
    // a run for every wave, as far as the workgroup goes
    int waves = (a.k + kRun - 1) / kRun;
    constexpr int kMost = BF16 ? 16 : 8, kRoom = 32 / (MT * G);   // registers; LDS
    constexpr int most = kMost < kRoom ? kMost : kRoom;
    waves = waves < 1 ? 1 : waves > most ? most : waves;
    const int across = G == 2 && a.out == kTileGated ? 16 : 16 * G;
    const dim3 g((a.ncol + across - 1) / across), blk(64 * waves);
    const size_t lds = size_t(waves) * 16 * MT * (16 * G + 4) * 4;   // at most 40 KB
    if constexpr (G == 2)   // (a group of either matrix)
        if (a.out == kTileGated) {
            hipLaunchKernelGGL((bdlm_skinny_kernel<MT, 2, BF16, kTileGated>), g, blk, lds, s, a);
            return hipGetLastError();
        }
    if (a.out == kTileStore) hipLaunchKernelGGL((bdlm_skinny_kernel<MT, G, BF16, kTileStore>), g, blk, lds, s, a);
    else if (a.out == kTileTop) hipLaunchKernelGGL((bdlm_skinny_kernel<MT, G, BF16, kTileTop>), g, blk, lds, s, a);
    else hipLaunchKernelGGL((bdlm_skinny_kernel<MT, G, BF16, kTileBest>), g, blk, lds, s, a);
    return hipGetLastError();
}
template <int MT, bool BF16>
hipError_t launch_rows_of(const SkinnyArgs &a, hipStream_t s) {
    return a.out == kTileGated || skinny_cols(a.ncol) == 32 ? launch_cols_of<MT, 2, BF16>(a, s) : launch_cols_of<MT, 1, BF16>(a, s);
}

}  // namespace

int launch_skinny(const SkinnyArgs &a, void *stream) {
    if (a.nrow <= 0 || a.ncol <= 0) return BDLM_OK;
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t r;
    if (a.bf16) r = a.nrow <= 16 ? launch_rows_of<1, true>(a, s) : launch_rows_of<2, true>(a, s);
    else
        r = a.nrow <= 16 ? launch_rows_of<1, false>(a, s) : a.nrow <= 32 ? launch_rows_of<2, false>(a, s)
                                                                        : launch_rows_of<4, false>(a, s);
    return r == hipSuccess ? BDLM_OK : BDLM_E_LAUNCH;
}

}  // namespace bdlm
