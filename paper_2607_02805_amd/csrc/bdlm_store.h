// bdlm_store.h -- the epilogues of a projection and of a gated one, four consecutive columns of a row at a time, shared by
// the kernels that end one (bdlm_tile.hip, bdlm_skinny.hip).  Internal.
#pragma once

#include "bdlm_dense_device.h"

namespace bdlm {
namespace {

__device__ __forceinline__ float load_elem(const void *p, int64_t i, bool bf16) {
    return bf16 ? bf16_to_f32(static_cast<const short *>(p)[i]) : static_cast<const float *>(p)[i];
}

__device__ __forceinline__ f32x4 load_bias(const StoreArgs &s, int col, int ncol) {
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (s.bias) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (col + e < ncol) v[e] = s.bias[col + e];
    }
    return v;
}

// Four consecutive columns of one row through a projection's epilogue.
__device__ __forceinline__ void store4(const StoreArgs &s, f32x4 v, f32x4 bias, int64_t row, int col, int ncol) {
    const int n = ncol - col < 4 ? ncol - col : 4;
    if (n <= 0) return;
    const int64_t ro = (s.row_of ? s.row_of[row] : row);
    v += bias;
    if (s.pre) {
        const int64_t o = ro * s.ld_pre + col;
        if (s.pre_bf16) {
            uint16_t *p = static_cast<uint16_t *>(s.pre) + o;
            if (n == 4 && s.ld_pre % 4 == 0)
                *reinterpret_cast<uint2 *>(p) = uint2{cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3])};
            else
                for (int e = 0; e < n; ++e) p[e] = static_cast<uint16_t>(bf16_bits(v[e]));
        } else {
            float *p = static_cast<float *>(s.pre) + o;
            if (n == 4 && s.ld_pre % 4 == 0) *reinterpret_cast<f32x4 *>(p) = v;
            else
                for (int e = 0; e < n; ++e) p[e] = v[e];
        }
    }
    // (the fine form costs fp32 outputs 1 %: 2,048 x 1,024 x 4,096 127 and 128 us; in bf16, where products are six times
    // cheaper, it would cost 16,384 x 1,024 x 4,096 217 instead of 206)
    if (s.act == BDLM_ACT_GELU && !s.out_bf16) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = act_value<true>(v[e], BDLM_ACT_GELU);
    } else if (s.act != BDLM_ACT_NONE) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = act_value<false>(v[e], s.act);
    }
    if (s.residual) {
        const int64_t o = ro * s.ld_res + col;
        if (n == 4 && s.ld_res % 4 == 0) {
            if (s.out_bf16) {
                const uint2 u = *reinterpret_cast<const uint2 *>(static_cast<const uint16_t *>(s.residual) + o);
                v += f32x4{__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u),
                           __uint_as_float(u.y << 16), __uint_as_float(u.y & 0xffff0000u)};
            } else {
                v += *reinterpret_cast<const f32x4 *>(static_cast<const float *>(s.residual) + o);
            }
        } else {
            for (int e = 0; e < n; ++e) v[e] += load_elem(s.residual, o + e, s.out_bf16);
        }
    }
    const int64_t o = ro * s.ld_out + col;
    if (s.out_bf16) {
        uint16_t *p = static_cast<uint16_t *>(s.out) + o;
        if (n == 4 && s.ld_out % 4 == 0)
            *reinterpret_cast<uint2 *>(p) = uint2{cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3])};
        else
            for (int e = 0; e < n; ++e) p[e] = static_cast<uint16_t>(bf16_bits(v[e]));
    } else {
        float *p = static_cast<float *>(s.out) + o;
        if (n == 4 && s.ld_out % 4 == 0) *reinterpret_cast<f32x4 *>(p) = v;
        else
            for (int e = 0; e < n; ++e) p[e] = v[e];
    }
}

// Four consecutive values to a row of bf16 or fp32, n of which there are.  Nontemporal: the launch does not read again what a tile
// stores, and its operands keep the L2.  1,024 x 4,096 in bf16, with plain stores and so, and together with the projection to 1,024
// that reads the output next:
//   16,384 rows   gated 281 and 261 us, kept 330 and 308   with the projection 424 and 412, kept 506 and 461
//    2,048 rows          35.3 and 33.8       42.0 and 40.3                       66.0 and 66.5       73.8 and 73.1
//      512 rows          14.7 and 14.5       16.5 and 15.2                       30.6 and 31.6       32.7 and 32.6
//       32 rows           6.9 and  7.2        7.3 and  7.5                       20.8 and 21.3       21.2 and 21.8
// Gradients gain 1 to 5 % (64 rows 35.6 and 34.0, 512 49 and 47, 16,384 623 and 618).  One rule for every size costs calls of few rows up to
// 4 % of themselves and 3 % of the pair, where the output would have stayed in the caches for its reader.
// Four of them are one store at any alignment (one by one, 3,136 x 152 x 314, kept, took 18.2 us instead of 14.9), but not past
// the caches where rows are not whole cache lines: 3,279 x 448 x 1,934, kept, took 47.5 us so, 28.8 with plain stores.
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef u32x2 __attribute__((aligned(2))) u32x2_a2;
__device__ __forceinline__ void put4(void *dst, int64_t o, int64_t ld, int n, bool bf16, f32x4 v) {
    const bool past = ld % 32 == 0;
    if (bf16) {
        uint16_t *p = static_cast<uint16_t *>(dst) + o;
        const u32x2 u = {cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3])};
        if (n == 4 && past) __builtin_nontemporal_store(u, reinterpret_cast<u32x2 *>(p));
        else if (n == 4) *reinterpret_cast<u32x2_a2 *>(p) = u;
        else
            for (int e = 0; e < n; ++e) p[e] = static_cast<uint16_t>(bf16_bits(v[e]));
    } else {
        float *p = static_cast<float *>(dst) + o;
        if (n == 4 && past) __builtin_nontemporal_store(v, reinterpret_cast<f32x4 *>(p));
        else if (n == 4) *reinterpret_cast<f32x4_a4 *>(p) = v;
        else
            for (int e = 0; e < n; ++e) p[e] = v[e];
    }
}
__device__ __forceinline__ f32x4 gated_bias(const float *bias, int col, int n) {
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (bias) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (col + e < n) v[e] = bias[col + e];
    }
    return v;
}
// Four consecutive columns of N consecutive rows (`there` of which there are) of a gated product, biases added already:
// act(gate) * up, of the unrounded ones.  All rows take a step before any takes the next: one after the other, whose chains of
// reads, exponentials and reciprocals wait for each, the end of a small tile took 2.4 us instead
// of 1.1 (512 x 1,024 x 4,096 13.7 instead of 12.3, 16,384 rows of it 273 instead of 250, timed in turn on one card; on others the first takes 13.3 to 14).
template <int N>
__device__ __forceinline__ void gated4(const GatedArgs &a, f32x4 (&gate)[N], f32x4 (&up)[N], int64_t row, int there, int col) {
    const int n = a.n - col < 4 ? a.n - col : 4;
    if (n <= 0 || there <= 0) return;
    if (a.pre_gate) {
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (k < there) {
                const int64_t o = (row + k) * a.ld_pre + col;
                put4(a.pre_gate, o, a.ld_pre, n, a.pre_bf16, gate[k]);
                put4(a.pre_up, o, a.ld_pre, n, a.pre_bf16, up[k]);
            }
    }
    if (a.act == BDLM_ACT_SILU) {
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) gate[k][e] = act_value<false>(gate[k][e], BDLM_ACT_SILU);
    } else if (a.act == BDLM_ACT_GELU && a.out_bf16) {
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) gate[k][e] = act_value<false>(gate[k][e], BDLM_ACT_GELU);
    } else if (a.act == BDLM_ACT_GELU) {
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) gate[k][e] = act_value<true>(gate[k][e], BDLM_ACT_GELU);
    }
#pragma unroll
    for (int k = 0; k < N; ++k)
        if (k < there) put4(a.out, (row + k) * a.ld_out + col, a.ld_out, n, a.out_bf16, gate[k] * up[k]);
}

// The sum of the slices at p, four columns, at any alignment.  Four slices are asked for at a time (one after the other, 128 x 1,024 in 16
// slices took 4 us more).
__device__ __forceinline__ f32x4 sum_slices(const float *p, int64_t slice, int splits) {
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    int k = 0;
    for (; k + 4 <= splits; k += 4) {
        f32x4 u[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) u[j] = *reinterpret_cast<const f32x4_a4 *>(p + (k + j) * slice);
#pragma unroll
        for (int j = 0; j < 4; ++j) v += u[j];
    }
    for (; k < splits; ++k) v += *reinterpret_cast<const f32x4_a4 *>(p + k * slice);
    return v;
}

}  // namespace
}  // namespace bdlm
