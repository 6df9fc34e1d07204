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

// The normal distribution's Phi(z), off by at most 3e-7, and e = exp(-z^2 / 2): with x = |z| / sqrt 2,
// erfc(x) = (a1 t + .. + a5 t^5) exp(-x^2), t = 1 / (1 + p x) (Abramowitz and Stegun 7.1.26), on
// the hardware's reciprocal and exponential.  The library's erfc costs three times as much, which
// shows where a tile's epilogue is not hidden behind products.
__device__ __forceinline__ float normal_cdf(float z, float &e) {
    const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f * 0.70710678f, fabsf(z), 1.f));
    e = __builtin_amdgcn_exp2f(z * z * (-0.5f * kLog2e));
    // half of erfc
    const float h = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 0.5f * 1.061405429f, 0.5f * -1.453152027f), 0.5f * 1.421413741f),
                                     0.5f * -0.284496736f), 0.5f * 0.254829592f) * e;
    return z > 0.f ? 1.f - h : h;
}
// Values and slopes at infinities are the limits; a NaN stays one.
__device__ __forceinline__ float act_value(float z, int act) {
    if (act == BDLM_ACT_SILU) {
        const float s = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * z));
        return z < -87.f ? 0.f : z * s;
    }
    if (act == BDLM_ACT_GELU) {
        float e;
        const float p = normal_cdf(z, e);
        return z < -14.f ? 0.f : z * p;
    }
    return z;
}
// d act / dz
__device__ __forceinline__ float act_slope(float z, int act) {
    if (act == BDLM_ACT_SILU) {
        const float s = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * z));
        return z < -87.f ? 0.f : z > 87.f ? 1.f : s * fmaf(z, 1.f - s, 1.f);
    }
    if (act == BDLM_ACT_GELU) {
        float e;
        const float p = normal_cdf(z, e);
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
