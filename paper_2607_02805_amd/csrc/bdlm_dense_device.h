// bdlm_dense_device.h -- device helpers of the dense operators: unaligned row pieces, activations and their
// derivatives, bf16 terms of fp32 values, and the merge of softmax records.  Internal.
#pragma once

#include "bdlm_dense.h"
#include "bdlm_device.h"

namespace bdlm {
namespace {

constexpr int kNoColumn = 0x7fffffff;

typedef u32x4 __attribute__((aligned(2))) u32x4_a2;
typedef u32x4 __attribute__((aligned(4))) u32x4_a4;

typedef f32x4 __attribute__((aligned(4))) f32x4_a4;

// Eight consecutive elements of a row as they lie, zeros past the n that there are.  The last ones of a row are loaded with
// those before them in the row (`before` of which there are) and moved down by settle(), which every load is followed by before
// its values are used: several rows' loads are on their way then.  (Taken one by one, each row's end was waited for: laying out
// 8,192 rows of 397 took 8.5 us instead of 6.1.)
// WHOLE: rows of whole eights, which have no such ends.
template <bool BF16, bool WHOLE = false>
struct Eight {
    u32x4 u[BF16 ? 1 : 2];
    int cut;
    __device__ __forceinline__ void load(const void *src, int64_t at, int n, int before) {
        cut = 0;
        if (!WHOLE && n > 0 && n < 8) {
            if (n + before < 8) {   // a row of fewer than eight
                uint32_t h[8];
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    h[e] = e >= n ? 0u : BF16 ? static_cast<const uint16_t *>(src)[at + e] : static_cast<const uint32_t *>(src)[at + e];
                if constexpr (BF16) {
                    u[0] = u32x4{h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16};
                } else {
                    u[0] = u32x4{h[0], h[1], h[2], h[3]};
                    u[1] = u32x4{h[4], h[5], h[6], h[7]};
                }
                return;
            }
            cut = 8 - n;
            at -= cut;
        }
        if (n > 0) {
            if constexpr (BF16) {
                u[0] = *reinterpret_cast<const u32x4_a2 *>(static_cast<const uint16_t *>(src) + at);
            } else {
                const float *p = static_cast<const float *>(src) + at;
                u[0] = *reinterpret_cast<const u32x4_a4 *>(p);
                u[1] = *reinterpret_cast<const u32x4_a4 *>(p + 4);
            }
        } else {
            for (auto &v : u) v = u32x4{0u, 0u, 0u, 0u};
        }
    }
    // Moves the elements down by `cut`, zeros after them.
    __device__ __forceinline__ void settle() {
        if (WHOLE || cut == 0) return;
        if constexpr (BF16) {
            uint64_t lo = u[0][0] | uint64_t(u[0][1]) << 32, hi = u[0][2] | uint64_t(u[0][3]) << 32;
            if (cut & 4) lo = hi, hi = 0;
            const int by = 16 * (cut & 3);
            if (by) lo = lo >> by | hi << (64 - by), hi >>= by;
            u[0] = u32x4{static_cast<uint32_t>(lo), static_cast<uint32_t>(lo >> 32), static_cast<uint32_t>(hi), static_cast<uint32_t>(hi >> 32)};
        } else {
#pragma unroll
            for (int by = 4; by >= 1; by /= 2)
                if (cut & by) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int from = e + by;
                        u[e >> 2][e & 3] = from < 8 ? u[from >> 2][from & 3] : 0u;
                    }
                }
        }
    }
    __device__ __forceinline__ float value(int e) const {
        if constexpr (BF16) return e & 1 ? __uint_as_float(u[0][e >> 1] & 0xffff0000u) : __uint_as_float(u[0][e >> 1] << 16);
        else return __uint_as_float(u[e >> 2][e & 3]);
    }
};

// v = t[0] + t[1] + t[2]: each term the rounded remainder of the ones before it, 24 bits together.
// A value whose rounding to bf16 would overflow keeps the largest finite first term, and an
// infinity or NaN is its first term alone (the remainders of an infinity would be NaN).
__device__ __forceinline__ void split_terms(float v, uint16_t (&t)[3]) {
    const bool finite = fabsf(v) <= 3.4028234e38f;
    const float top = __uint_as_float(0x7f7f0000u);   // largest bf16
    const float c = finite ? fminf(fmaxf(v, -top), top) : v;
    t[0] = static_cast<uint16_t>(bf16_bits(c));
    const float r1 = finite ? v - bf16_to_f32(static_cast<short>(t[0])) : 0.f;
    t[1] = static_cast<uint16_t>(bf16_bits(r1));
    t[2] = static_cast<uint16_t>(bf16_bits(r1 - bf16_to_f32(static_cast<short>(t[1]))));
}

// The normal distribution's Phi(z) and e = exp(-z^2 / 2) on the hardware's reciprocal and exponential.
// Phi(-a) = e R(t), t = 1 / (1 + p a), where R(t) = t (c0 + c1 t + ..) stands for erfcx(a / sqrt 2) / 2, which is
// smooth in t over 0 <= a <= 14; the polynomials are minimax fits made for this file.
// FINE, for what is kept in fp32: R's relative error stays below 4e-8, t is improved by a Newton step and e by
// the part of -z^2 / 2 that fp32 drops, so that Phi(z) is off by at most 4e-7 of itself, the tail included (emulated
// over 50,001 points; GELU of normal z by 3.7e-8, as with a correctly rounded erf near 0).
// Otherwise, for values that are rounded to bf16 (half a step is 3.9e-3) and slopes at a z that was (which moves
// Phi(z) by up to z^2 2^-8 of itself in the tail): a polynomial of degree 5, off by 1e-7 and in the tail by 2.9e-4 of
// itself; GELU is off by 2.5e-7 |z| at most, also where a residual cancels it.
template <bool FINE>
__device__ __forceinline__ float normal_cdf(float z, float &e) {
    const float a = FINE ? fminf(fabsf(z), 14.5f) : fabsf(z);   // (finite, as q is subtracted from itself)
    const float d = fmaf(FINE ? 0.42426407f : 0.28284271f, a, 1.f);
    float t = __builtin_amdgcn_rcpf(d), r;
    const float q = a * a, y = q * (-0.5f * kLog2e);
    e = __builtin_amdgcn_exp2f(y);
    if constexpr (FINE) {
        t = fmaf(t, fmaf(-d, t, 1.f), t);
        // what y lacks of -z^2 log2(e) / 2: the roundings of q and y, and the constant's
        constexpr float rest = static_cast<float>(-0.5 * 1.4426950408889634 - double(-0.5f * kLog2e));
        const float lack = fmaf(fmaf(a, a, -q), -0.5f * kLog2e, fmaf(q, rest, fmaf(q, -0.5f * kLog2e, -y)));
        e = fmaf(e, lack * 0.69314718f, e);
        r = fmaf(t, 0.03233261f, -0.15625919f);
        r = fmaf(t, r, 0.27504578f);
        r = fmaf(t, r, -0.16007753f);
        r = fmaf(t, r, -0.068789035f);
        r = fmaf(t, r, 0.032218184f);
        r = fmaf(t, r, 0.066111073f);
        r = fmaf(t, r, 0.14113246f);
        r = fmaf(t, r, 0.16901903f);
        r = fmaf(t, r, 0.16926664f);
    } else {
        r = fmaf(t, -0.096094035f, 0.338998735f);
        r = fmaf(t, r, -0.161798224f);
        r = fmaf(t, r, 0.216511309f);
        r = fmaf(t, r, 0.087330155f);
        r = fmaf(t, r, 0.115052164f);
    }
    const float h = t * r * e;
    return z > 0.f ? 1.f - h : h;
}
// Values and slopes at infinities are the limits; a NaN stays one.
template <bool FINE>
__device__ __forceinline__ float act_value(float z, int act) {
    if (act == BDLM_ACT_SILU) {
        const float s = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * z));
        return z < -87.f ? 0.f : z * s;
    }
    if (act == BDLM_ACT_GELU) {
        float e;
        const float p = normal_cdf<FINE>(z, e);
        return z < -14.f ? 0.f : z * p;
    }
    return z;
}
// d act / dz
template <bool FINE>
__device__ __forceinline__ float act_slope(float z, int act) {
    if (act == BDLM_ACT_SILU) {
        const float s = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * z));
        return z < -87.f ? 0.f : z > 87.f ? 1.f : s * fmaf(z, 1.f - s, 1.f);
    }
    if (act == BDLM_ACT_GELU) {
        float e;
        const float p = normal_cdf<FINE>(z, e);
        return z < -14.f ? 0.f : z > 14.f ? 1.f : fmaf(z * 0.39894228f, e, p);
    }
    return 1.f;
}

// act(z) and d act / dz together
template <bool FINE>
__device__ __forceinline__ void act_both(float z, int act, float &value, float &slope) {
    if (act == BDLM_ACT_SILU) {
        const float s = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * z));
        value = z < -87.f ? 0.f : z * s;
        slope = z < -87.f ? 0.f : z > 87.f ? 1.f : s * fmaf(z, 1.f - s, 1.f);
    } else if (act == BDLM_ACT_GELU) {
        float e;
        const float p = normal_cdf<FINE>(z, e);
        value = z < -14.f ? 0.f : z * p;
        slope = z < -14.f ? 0.f : z > 14.f ? 1.f : fmaf(z * 0.39894228f, e, p);
    } else {
        value = z;
        slope = 1.f;
    }
}

// A softmax record: the largest value, its column (the lowest of equals), and the sum over the
// other columns of exp(value - largest).  The largest one's own 1 stays out of the sum, so that a
// log-probability near 0, -log(1 + others), keeps its digits.
struct Best {
    float top, others;
    int at;
};
__device__ __forceinline__ bool beats(float v, int at, const Best &b) {
    return v > b.top || (v == b.top && at < b.at);
}
// A value of -infinity adds nothing; a NaN makes the sum NaN and is never the largest.
__device__ __forceinline__ float share(float v, float top) {
    return v == -INFINITY ? 0.f : __expf(v - top);
}
__device__ __forceinline__ Best merge(const Best &a, const Best &b) {
    const bool second = beats(b.top, b.at, a);
    const Best &hi = second ? b : a;
    const Best &lo = second ? a : b;
    // the lower record's own 1 only if it holds a column at all
    const float one = lo.at == kNoColumn ? 0.f : 1.f;
    const float f = share(lo.top, hi.top);
    Best r{hi.top, hi.others, hi.at};
    r.others += (one + lo.others) * f;
    if (lo.others != lo.others) r.others = lo.others;   // NaN times a share of 0 stays NaN
    return r;
}

// The same record with the slope of the sum: over the other columns the sum of exp(d) d, d = value - largest, of which an
// entropy is made without cancellation: log Z - slope / Z, Z = 1 + others, both terms positive.
struct Spread {
    float top, others, slope;
};
// exp(d) d of a value's own exp(d) = s: 0 where d is -infinity
__device__ __forceinline__ float slope_of(float s, float d) { return s * fmaxf(d, -1e30f); }

}  // namespace
}  // namespace bdlm
