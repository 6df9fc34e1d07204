// bdlm_addnorm.hip -- gfx950 kernels of the root-mean-square norm at a sublayer's entry, with the residual's
// addition and an output in 8 bits with scales, and of its gradient:
//   s = x + residual,  n = s / sqrt(mean s^2 + eps),  y = w n;
//   ds = rstd (w dy - n mean(n w dy)) + dsum,  dw = sum over the rows of dy n.
//
// Bound by the bytes of the rows, and for few rows by the launch.  Rows lie in registers between the sums over them and
// the output, so that every element is read once: a wave has a row of up to 1,024 columns for itself (no
// barrier), four waves share one of up to 8,192, and longer rows are read once for each sum.
// Waves go on to further rows with the weights kept.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "bdlm.h"
#include "bdlm_dense.h"
#include "bdlm_dense_device.h"
#include "bdlm_sublayer.h"

namespace bdlm {
namespace {

constexpr int kWaves = 4;          // of a workgroup
constexpr float kE4m3Max = 448.f;

__device__ __forceinline__ float last_lane(float v) {
    return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), 63));
}
__device__ __forceinline__ float wave_sum(float v) { return last_lane(wave_inclusive_sum(v)); }
// Largest of values that are not negative (a NaN is passed over).
__device__ __forceinline__ float wave_largest(float v) {
    v = fmaxf(v, dpp<0x111, 0xf, true>(v));
    v = fmaxf(v, dpp<0x112, 0xf, true>(v));
    v = fmaxf(v, dpp<0x114, 0xf, true>(v));
    v = fmaxf(v, dpp<0x118, 0xf, true>(v));
    v = fmaxf(v, dpp<0x142, 0xa, false>(v));
    v = fmaxf(v, dpp<0x143, 0xc, false>(v));
    return last_lane(v);
}

// Sums (or largest values) over the W waves of a row.  Two places in turn: a wave writes one again only after a
// barrier that follows every wave's reads of it.
template <int W>
struct Row {
    float (*lds)[2][kWaves];
    int turn = 0;
    template <bool LARGEST>
    __device__ __forceinline__ float over(float v) {
        v = LARGEST ? wave_largest(v) : wave_sum(v);
        if constexpr (W > 1) {
            const int wave = threadIdx.x >> 6;
            if ((threadIdx.x & 63) == 0) (*lds)[turn][wave] = v;
            __syncthreads();
            const float *p = (*lds)[turn];
            v = LARGEST ? fmaxf(fmaxf(p[0], p[1]), fmaxf(p[2], p[3])) : (p[0] + p[1]) + (p[2] + p[3]);
            turn ^= 1;
        }
        return v;
    }
    __device__ __forceinline__ float sum(float v) { return over<false>(v); }
    __device__ __forceinline__ float largest(float v) { return over<true>(v); }
};

// 1 / sqrt(mean + eps), mean = sum of squares / width.  Where squares may leave fp32's range (a sum above 2^120, or
// mean + eps below 2^-96, where lost squares would count) they are taken again of s / 2^e, 2^e just above the largest |s|.
// each(f): f(s) for the lane's elements.  The same way for every lane of the row.
template <class R, class E>
__device__ __forceinline__ float row_rstd(R &row, float ss, float inv_width, float eps, E each) {
    const float mean = ss * inv_width;
    if (!(ss > 0x1p120f) && !(mean + eps < 0x1p-96f)) return 1.f / sqrtf(mean + eps);
    float top = 0.f;
    each([&](float v) { top = fmaxf(top, fabsf(v)); });
    top = row.largest(top);
    if (top == INFINITY) return 0.f;
    int e = 0;
    frexpf(top, &e);
    float again = 0.f;
    each([&](float v) {
        const float u = ldexpf(v, -e);
        again = fmaf(u, u, again);
    });
    again = row.sum(again);
    const double square = static_cast<double>(again) * inv_width * exp2(2.0 * e);
    return static_cast<float>(1.0 / sqrt(square + eps));
}

// Eight values to a row of bf16 or fp32, n of which there are.
__device__ __forceinline__ void put8(void *dst, int64_t at, int n, bool bf16, const float (&v)[8]) {
    if (bf16) {
        uint16_t *p = static_cast<uint16_t *>(dst) + at;
        const u32x4 u = {cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3]), cvt_pk_bf16(v[4], v[5]), cvt_pk_bf16(v[6], v[7])};
        if (n >= 8) *reinterpret_cast<u32x4_a2 *>(p) = u;
        else
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < n) p[e] = static_cast<uint16_t>(u[e >> 1] >> (16 * (e & 1)));
    } else {
        float *p = static_cast<float *>(dst) + at;
        if (n >= 8) {
            *reinterpret_cast<u32x4_a4 *>(p) = u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
            *reinterpret_cast<u32x4_a4 *>(p + 4) = u32x4{__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])};
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < n) p[e] = v[e];
        }
    }
}

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef u32x2 __attribute__((aligned(1))) u32x2_a1;

// Eight values as e4m3: v times 448 / top, rounded to nearest even.  (v * f is at most 448 and a rounding.)
__device__ __forceinline__ void put8_e4m3(void *dst, int64_t at, int n, float f, const float (&v)[8]) {
    float q[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        q[e] = v[e] * f;
        q[e] = fabsf(q[e]) > kE4m3Max ? copysignf(kE4m3Max, q[e]) : q[e];   // (a NaN stays one)
    }
    int lo = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], lo, true);
    int hi = __builtin_amdgcn_cvt_pk_fp8_f32(q[4], q[5], 0, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(q[6], q[7], hi, true);
    uint8_t *p = static_cast<uint8_t *>(dst) + at;
    if (n >= 8) *reinterpret_cast<u32x2_a1 *>(p) = u32x2{static_cast<uint32_t>(lo), static_cast<uint32_t>(hi)};
    else
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) p[e] = static_cast<uint8_t>((e < 4 ? lo : hi) >> (8 * (e & 3)));
}

// The scale of values up to `top`, and what they are multiplied with.  Zeros have a scale of 1.
__device__ __forceinline__ float scale_of(float top, float &f) {
    if (top == 0.f) {
        f = 1.f;
        return 1.f;
    }
    // (448 / top overflows below 2^-119: such values, far below eps's reach, keep the largest factor there is)
    f = fminf(kE4m3Max / top, 0x1p126f);
    return top < 0x1p-110f ? 1.f / f : top / kE4m3Max;
}

struct Types {
    static constexpr int kNone = 0, kBf16 = 1, kF32 = 2;
};

// W waves a row, C pieces of 8 columns a lane kept in registers (0: any width, read again for each sum).
template <int W, int C, bool X16, int RES>
__global__ void __launch_bounds__(64 * kWaves) bdlm_add_rmsnorm_kernel(const AddNormArgs a) {
    __shared__ float lds[2][kWaves];
    constexpr int kRows = kWaves / W, kAcross = 64 * W * 8, K = C ? C : 1;
    const int lane = threadIdx.x & (64 * W - 1), sub = threadIdx.x / (64 * W);
    const float inv_width = 1.f / static_cast<float>(a.width);
    Row<W> row{&lds};
    float w[K][8];
    auto load_w = [&](int c, float (&v)[8]) {
        Eight<false> t;
        t.load(a.w, c, a.width - c, c);
        t.settle();
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = t.value(e);
    };
    if constexpr (C > 0) {
#pragma unroll
        for (int k = 0; k < C; ++k) load_w(k * kAcross + lane * 8, w[k]);
    }
    struct Raw {
        Eight<X16> x;
        Eight<RES != Types::kF32> r;
    };
    auto load = [&](int64_t r, int c, Raw &t) {
        const int n = a.width - c;
        t.x.load(a.x, r * a.ldx + c, n, c);
        if constexpr (RES != Types::kNone) t.r.load(a.residual, r * a.ldr + c, n, c);
    };
    auto add = [&](Raw &t, float (&s)[8]) {
        t.x.settle();
        if constexpr (RES != Types::kNone) t.r.settle();
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            s[e] = t.x.value(e);
            if constexpr (RES != Types::kNone) s[e] += t.r.value(e);
        }
    };
    // y of eight columns, to memory in 8 bits with scale factors, or as it is
    auto put = [&](int64_t r, int c, const float (&y)[8], float f) {
        const int n = a.width - c;
        if (n <= 0) return;
        if (a.out_dtype == BDLM_DTYPE_E4M3) put8_e4m3(a.out, r * a.ldo + c, n, f, y);
        else put8(a.out, r * a.ldo + c, n, a.out_dtype == BDLM_DTYPE_BF16, y);
    };
    auto top_of = [&](const float (&y)[8]) {
        float t = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) t = fmaxf(t, fabsf(y[e]));
        return t;
    };
    // 16 consecutive lanes have a block of columns
    auto block_factor = [&](int64_t r, int c, const float (&y)[8], float rstd) {
        float t = top_of(y), f;
#pragma unroll
        for (int d = 1; d < 16; d *= 2) t = fmaxf(t, __shfl_xor(t, d, 64));
        const float scale = scale_of(t, f);
        if ((lane & 15) == 0 && c < a.width) a.scale[r * a.blocks + c / kScaleBlock] = rstd > 0.f ? scale : NAN;
        return f;
    };
    const bool e4m3 = a.out_dtype == BDLM_DTYPE_E4M3;
    for (int64_t r0 = int64_t(blockIdx.x) * kRows; r0 < a.rows; r0 += int64_t(gridDim.x) * kRows) {
        const int64_t r = r0 + sub;
        if (r >= a.rows) break;   // (a wave's own row: no barrier follows where kRows > 1)
        if constexpr (C > 0) {
            Raw raw[C];
#pragma unroll
            for (int k = 0; k < C; ++k) load(r, k * kAcross + lane * 8, raw[k]);
            float s[C][8], ss = 0.f;
#pragma unroll
            for (int k = 0; k < C; ++k) {
                add(raw[k], s[k]);
#pragma unroll
                for (int e = 0; e < 8; ++e) ss = fmaf(s[k][e], s[k][e], ss);
            }
            if (RES != Types::kNone && a.sum) {
#pragma unroll
                for (int k = 0; k < C; ++k) {
                    const int c = k * kAcross + lane * 8;
                    if (c < a.width) put8(a.sum, r * a.lds + c, a.width - c, RES == Types::kBf16, s[k]);
                }
            }
            ss = row.sum(ss);
            const float rstd = row_rstd(row, ss, inv_width, a.eps, [&](auto f) {
#pragma unroll
                for (int k = 0; k < C; ++k)
#pragma unroll
                    for (int e = 0; e < 8; ++e) f(s[k][e]);
            });
            float top = 0.f;
#pragma unroll
            for (int k = 0; k < C; ++k) {
#pragma unroll
                for (int e = 0; e < 8; ++e) s[k][e] = s[k][e] * rstd * w[k][e];
                if (e4m3) top = fmaxf(top, top_of(s[k]));
            }
            float f = 1.f;
            if (e4m3 && !a.by_block) {
                const float scale = scale_of(row.largest(top), f);
                if (lane == 0) a.scale[r] = rstd > 0.f ? scale : NAN;
            }
#pragma unroll
            for (int k = 0; k < C; ++k) {
                const int c = k * kAcross + lane * 8;
                if (e4m3 && a.by_block) f = block_factor(r, c, s[k], rstd);
                put(r, c, s[k], f);
            }
        } else {
            // every pass reads the row again; the lane that writes an element has read it before
            auto each = [&](auto f) {
                for (int c = lane * 8; c < a.width; c += kAcross) {
                    Raw raw;
                    float s[8];
                    load(r, c, raw);
                    add(raw, s);
#pragma unroll
                    for (int e = 0; e < 8; ++e) f(s[e]);
                }
            };
            float ss = 0.f;
            each([&](float v) { ss = fmaf(v, v, ss); });
            ss = row.sum(ss);
            const float rstd = row_rstd(row, ss, inv_width, a.eps, each);
            auto y_of = [&](int c, float (&s)[8], float (&y)[8]) {
                Raw raw;
                load(r, c, raw);
                add(raw, s);
                load_w(c, y);
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] *= s[e] * rstd;
            };
            float f = 1.f;
            if (e4m3 && !a.by_block) {
                float top = 0.f;
                for (int c = lane * 8; c < a.width; c += kAcross) {
                    float s[8], y[8];
                    y_of(c, s, y);
                    top = fmaxf(top, top_of(y));
                }
                const float scale = scale_of(row.largest(top), f);
                if (lane == 0) a.scale[r] = rstd > 0.f ? scale : NAN;
            }
            // (whole turns, so that the 16 lanes of a block meet)
            for (int c0 = 0; c0 < a.width; c0 += kAcross) {
                const int c = c0 + lane * 8;
                float s[8], y[8];
                y_of(c, s, y);
                if (e4m3 && a.by_block) f = block_factor(r, c, y, rstd);
                if (RES != Types::kNone && a.sum && c < a.width)
                    put8(a.sum, r * a.lds + c, a.width - c, RES == Types::kBf16, s);
                put(r, c, y, f);
            }
        }
    }
}

// The gradient.  A workgroup's rows add up its partial sums of dw in registers (C 0: in its row of `part`).
template <int W, int C, bool Y16, bool S16>
__global__ void __launch_bounds__(64 * kWaves) bdlm_add_rmsnorm_grad_kernel(const AddNormGradArgs a) {
    __shared__ float lds[2][kWaves];
    constexpr int kRows = kWaves / W, kAcross = 64 * W * 8, K = C ? C : 1;
    __shared__ float sums[W == 1 ? kWaves : 1][W == 1 ? K * kAcross : 1];
    const int lane = threadIdx.x & (64 * W - 1), sub = threadIdx.x / (64 * W);
    const float inv_width = 1.f / static_cast<float>(a.width);
    Row<W> row{&lds};
    auto load_w = [&](int c, float (&v)[8]) {
        Eight<false> t;
        t.load(a.w, c, a.width - c, c);
        t.settle();
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = t.value(e);
    };
    // what arrives on the stream from behind, bf16 or fp32, for eight columns
    struct Behind {
        Eight<true> h;
        Eight<false> f;
    };
    auto load_behind = [&](int64_t at, int n, int c, Behind &t) {
        if (!a.dsum) return;
        if (a.ds_bf16) t.h.load(a.dsum, at, n, c);
        else t.f.load(a.dsum, at, n, c);
    };
    auto settle_behind = [&](Behind &t) {
        if (!a.dsum) return;
        if (a.ds_bf16) t.h.settle();
        else t.f.settle();
    };
    auto value = [&](const Behind &t, int e) { return !a.dsum ? 0.f : a.ds_bf16 ? t.h.value(e) : t.f.value(e); };
    float *part = a.part ? a.part + int64_t(blockIdx.x) * a.width : nullptr;
    if constexpr (C > 0) {
        float w[C][8], dw[C][8];
#pragma unroll
        for (int k = 0; k < C; ++k) {
            load_w(k * kAcross + lane * 8, w[k]);
#pragma unroll
            for (int e = 0; e < 8; ++e) dw[k][e] = 0.f;
        }
        for (int64_t r0 = int64_t(blockIdx.x) * kRows; r0 < a.rows; r0 += int64_t(gridDim.x) * kRows) {
            const int64_t r = r0 + sub;
            if (r >= a.rows) break;   // (a wave's own row)
            Eight<S16> rs[C];
            Eight<Y16> ry[C];
            Behind rb[C];
#pragma unroll
            for (int k = 0; k < C; ++k) {
                const int c = k * kAcross + lane * 8, n = a.width - c;
                rs[k].load(a.s, r * a.lds + c, n, c);
                ry[k].load(a.dy, r * a.ldy + c, n, c);
                if (a.ds) load_behind(r * a.ldt + c, n, c, rb[k]);
            }
            float ss = 0.f;
#pragma unroll
            for (int k = 0; k < C; ++k) rs[k].settle(), ry[k].settle();
#pragma unroll
            for (int k = 0; k < C; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) ss = fmaf(rs[k].value(e), rs[k].value(e), ss);
            ss = row.sum(ss);
            const float rstd = row_rstd(row, ss, inv_width, a.eps, [&](auto f) {
#pragma unroll
                for (int k = 0; k < C; ++k)
#pragma unroll
                    for (int e = 0; e < 8; ++e) f(rs[k].value(e));
            });
            float dot = 0.f;
#pragma unroll
            for (int k = 0; k < C; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float n = rs[k].value(e) * rstd, dy = ry[k].value(e);
                    dot = fmaf(n, w[k][e] * dy, dot);
                    dw[k][e] = fmaf(n, dy, dw[k][e]);
                }
            if (!a.ds) continue;
            dot = row.sum(dot) * inv_width;
#pragma unroll
            for (int k = 0; k < C; ++k) {
                const int c = k * kAcross + lane * 8;
                float d[8];
                settle_behind(rb[k]);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float n = rs[k].value(e) * rstd;
                    d[e] = fmaf(rstd, fmaf(-n, dot, w[k][e] * ry[k].value(e)), value(rb[k], e));
                }
                if (c < a.width) put8(a.ds, r * a.ldd + c, a.width - c, a.ds_bf16, d);
            }
        }
        if (!part) return;
        if constexpr (W == 1) {
#pragma unroll
            for (int k = 0; k < C; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) sums[sub][k * kAcross + lane * 8 + e] = dw[k][e];
            __syncthreads();
            for (int c = threadIdx.x; c < a.width; c += 64 * kWaves)
                part[c] = (sums[0][c] + sums[1][c]) + (sums[2][c] + sums[3][c]);
        } else {
#pragma unroll
            for (int k = 0; k < C; ++k) {
                const int c = k * kAcross + lane * 8;
                if (c < a.width) put8(part, c, a.width - c, false, dw[k]);
            }
        }
    } else {
        for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
            auto each = [&](auto f) {
                for (int c = lane * 8; c < a.width; c += kAcross) {
                    Eight<S16> t;
                    t.load(a.s, r * a.lds + c, a.width - c, c);
                    t.settle();
#pragma unroll
                    for (int e = 0; e < 8; ++e) f(t.value(e));
                }
            };
            float ss = 0.f;
            each([&](float v) { ss = fmaf(v, v, ss); });
            ss = row.sum(ss);
            const float rstd = row_rstd(row, ss, inv_width, a.eps, each);
            float dot = 0.f;
            for (int c = lane * 8; c < a.width; c += kAcross) {
                Eight<S16> s;
                Eight<Y16> y;
                float w[8], d[8];
                s.load(a.s, r * a.lds + c, a.width - c, c);
                y.load(a.dy, r * a.ldy + c, a.width - c, c);
                load_w(c, w);
                s.settle();
                y.settle();
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float n = s.value(e) * rstd;
                    dot = fmaf(n, w[e] * y.value(e), dot);
                    d[e] = n * y.value(e);
                }
                if (part) {
                    if (r != static_cast<int64_t>(blockIdx.x)) {
                        Eight<false> before;   // (this lane's own writes)
                        before.load(part, c, a.width - c, c);
                        before.settle();
#pragma unroll
                        for (int e = 0; e < 8; ++e) d[e] += before.value(e);
                    }
                    put8(part, c, a.width - c, false, d);
                }
            }
            if (!a.ds) continue;
            dot = row.sum(dot) * inv_width;
            for (int c = lane * 8; c < a.width; c += kAcross) {
                Eight<S16> s;
                Eight<Y16> y;
                Behind b;
                float w[8], d[8];
                s.load(a.s, r * a.lds + c, a.width - c, c);
                y.load(a.dy, r * a.ldy + c, a.width - c, c);
                load_behind(r * a.ldt + c, a.width - c, c, b);
                load_w(c, w);
                s.settle();
                y.settle();
                settle_behind(b);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    d[e] = fmaf(rstd, fmaf(-s.value(e) * rstd, dot, w[e] * y.value(e)), value(b, e));
                put8(a.ds, r * a.ldd + c, a.width - c, a.ds_bf16, d);
            }
        }
    }
}

// Waves and pieces for a width: one wave a row up to 1,024 columns, then four; 0 pieces: longer than 8,192.
struct Way {
    int waves, pieces;
};
Way way_of(int64_t width) {
    if (width <= 512) return {1, 1};
    if (width <= 1024) return {1, 2};
    if (width <= 2048) return {4, 1};
    if (width <= 4096) return {4, 2};
    return {4, width <= 8192 ? 4 : 0};
}
constexpr int64_t kMostGroups = 2048;   // workgroups of the forward call: eight on a CU
constexpr int64_t kMostGradGroups = 512;   // of the gradient, each with a row of sums of dw
// Of the gradient without dw, which every turn of rows can have a workgroup for (16 rows of 1,024: 3.9 us, 8.5 in one workgroup) and
// which has no sums.  In bf16, inputs not in the caches, 16,384 x 2,048 takes 40 us so and 59 with 512, 60,000 x 448 31 and 47, but
// 16,384 x 1,024 25.4 and 25.1, 8,000 x 8,192 126 and 121 (138 with 2,048).
constexpr int64_t kMostStreamGroups = 1024;

// Turns of rows of a gradient's workgroup.
int64_t grad_groups(int64_t rows, int64_t width) {
    const int64_t per = kWaves / way_of(width).waves;
    return (rows + per - 1) / per;
}

int done() { return hipGetLastError() == hipSuccess ? BDLM_OK : BDLM_E_LAUNCH; }

template <bool X16, int RES>
int norm_of(const AddNormArgs &a, hipStream_t s) {
    const Way y = way_of(a.width);
    const int64_t per = kWaves / y.waves, groups = (a.rows + per - 1) / per;
    const dim3 g(static_cast<unsigned>(groups < kMostGroups ? groups : kMostGroups)), b(64 * kWaves);
    if (y.waves == 1 && y.pieces == 1) hipLaunchKernelGGL((bdlm_add_rmsnorm_kernel<1, 1, X16, RES>), g, b, 0, s, a);
    else if (y.waves == 1) hipLaunchKernelGGL((bdlm_add_rmsnorm_kernel<1, 2, X16, RES>), g, b, 0, s, a);
    else if (y.pieces == 1) hipLaunchKernelGGL((bdlm_add_rmsnorm_kernel<4, 1, X16, RES>), g, b, 0, s, a);
    else if (y.pieces == 2) hipLaunchKernelGGL((bdlm_add_rmsnorm_kernel<4, 2, X16, RES>), g, b, 0, s, a);
    else if (y.pieces == 4) hipLaunchKernelGGL((bdlm_add_rmsnorm_kernel<4, 4, X16, RES>), g, b, 0, s, a);
    else hipLaunchKernelGGL((bdlm_add_rmsnorm_kernel<4, 0, X16, RES>), g, b, 0, s, a);
    return done();
}
template <bool Y16, bool S16>
int grad_of(const AddNormGradArgs &a, hipStream_t s) {
    const Way y = way_of(a.width);
    const int64_t groups = a.part ? add_norm_grad_blocks(a.rows, a.width) : std::min(grad_groups(a.rows, a.width), kMostStreamGroups);
    const dim3 g(static_cast<unsigned>(groups)), b(64 * kWaves);
    if (y.waves == 1 && y.pieces == 1) hipLaunchKernelGGL((bdlm_add_rmsnorm_grad_kernel<1, 1, Y16, S16>), g, b, 0, s, a);
    else if (y.waves == 1) hipLaunchKernelGGL((bdlm_add_rmsnorm_grad_kernel<1, 2, Y16, S16>), g, b, 0, s, a);
    else if (y.pieces == 1) hipLaunchKernelGGL((bdlm_add_rmsnorm_grad_kernel<4, 1, Y16, S16>), g, b, 0, s, a);
    else if (y.pieces == 2) hipLaunchKernelGGL((bdlm_add_rmsnorm_grad_kernel<4, 2, Y16, S16>), g, b, 0, s, a);
    else if (y.pieces == 4) hipLaunchKernelGGL((bdlm_add_rmsnorm_grad_kernel<4, 4, Y16, S16>), g, b, 0, s, a);
    else hipLaunchKernelGGL((bdlm_add_rmsnorm_grad_kernel<4, 0, Y16, S16>), g, b, 0, s, a);
    return done();
}

}  // namespace

int32_t add_norm_grad_blocks(int64_t rows, int64_t width) {
    // (Times of rows that the caches hold.)
    // Two turns of rows of up to 4,096 columns are one workgroup's, whose dw needs no second launch: 8 rows of 448 columns take 4.1 us
    // so and 5.1 in two launches, 8 of 1,024 5.8 and 6.2, 2 of 4,096 6.0 and 6.4.  Past that the turns one after the other cost more
    // than the launch: 2 rows of 8,192 take 9.5 and 8.7, three turns 12 of 1,024 7.4 and 6.2, 4 rows of 32,768 93 and 26.
    const int64_t groups = grad_groups(rows, width);
    return static_cast<int32_t>(groups <= (width <= 4096 ? 2 : 1) ? (groups > 0 ? 1 : 0) : std::min(groups, kMostGradGroups));
}

int launch_add_norm(const AddNormArgs &a, void *stream) {
    if (a.rows <= 0) return BDLM_OK;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int res = !a.residual ? Types::kNone : a.res_bf16 ? Types::kBf16 : Types::kF32;
    switch ((a.x_bf16 ? 3 : 0) + res) {
        case 0: return norm_of<false, Types::kNone>(a, s);
        case 1: return norm_of<false, Types::kBf16>(a, s);
        case 2: return norm_of<false, Types::kF32>(a, s);
        case 3: return norm_of<true, Types::kNone>(a, s);
        case 4: return norm_of<true, Types::kBf16>(a, s);
        default: return norm_of<true, Types::kF32>(a, s);
    }
}

int launch_add_norm_grad(const AddNormGradArgs &a, void *stream) {
    if (a.rows <= 0) return BDLM_OK;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (a.dy_bf16) return a.s_bf16 ? grad_of<true, true>(a, s) : grad_of<true, false>(a, s);
    return a.s_bf16 ? grad_of<false, true>(a, s) : grad_of<false, false>(a, s);
}

}  // namespace bdlm
