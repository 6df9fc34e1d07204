// bdlm_store.h -- the epilogue of a projection, four consecutive columns of a row at a time, shared by
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

}  // namespace
}  // namespace bdlm
