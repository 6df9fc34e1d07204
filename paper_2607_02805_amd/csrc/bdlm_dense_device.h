// bdlm_dense_device.h -- device helpers of the dense operators: activations and their
// derivatives, bf16 terms of fp32 values, and the merge of softmax records.  Internal.
#pragma once

#include "bdlm_dense.h"
#include "bdlm_device.h"

namespace bdlm {
namespace {

constexpr int kNoColumn = 0x7fffffff;

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

}  // namespace
}  // namespace bdlm
