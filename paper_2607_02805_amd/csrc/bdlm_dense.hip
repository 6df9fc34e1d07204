// bdlm_dense.hip -- gfx950 kernels around the products of the dense operators: operands laid out as
// bf16 terms, the gradient of a projection's activation with the bias gradient's column sums, the
// rows that count of a masked loss, and the merge of softmax records.  All are bound by the
// bytes they move or, of few bytes, by their launch: the gradient of a GELU over 16,384 x 4,096 in
// bf16 (402 MB) takes 80 to 95 us, 4.2 to 5.0 TB/s; the rows of 8,192 labels 7 us
// in the forward and 14 in the backward call (one workgroup in a loop, linear in the rows: 2^22 labels 3.4 ms); 8,192 rows
// of 197 records 12 us (a workgroup a row: 2^22 rows of one record 6.1 ms).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "bdlm.h"
#include "bdlm_dense.h"
#include "bdlm_dense_device.h"

namespace bdlm {
namespace {

template <int TERMS>
__device__ __forceinline__ void store_terms(uint16_t *dst, int64_t plane, const float (&v)[8]) {
    if constexpr (TERMS == 1) {
        *reinterpret_cast<uint4 *>(dst) = uint4{cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3]),
                                                cvt_pk_bf16(v[4], v[5]), cvt_pk_bf16(v[6], v[7])};
        return;
    }
    uint16_t h[8][3];
#pragma unroll
    for (int e = 0; e < 8; ++e) split_terms(v[e], h[e]);
#pragma unroll
    for (int k = 0; k < TERMS; ++k) {
        uint32_t u[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) u[e] = h[2 * e][k] | uint32_t(h[2 * e + 1][k]) << 16;
        *reinterpret_cast<uint4 *>(dst + k * plane) = uint4{u[0], u[1], u[2], u[3]};
    }
}

// Thread: eight columns of kPackBatch rows at a time, all asked for before any is used (with one row
// at a time, 1,003 x 1,934 fp32 took 33 us instead of 12); a workgroup takes kPackRows rows of 64 x 8
// columns with its four waves (row r of every four).  The column sums are of the fp32 values,
// before they are rounded.
constexpr int kPackBatch = 4;
static_assert(kPackRows % (4 * kPackBatch) == 0, "whole batches");
template <bool GRAD, bool BF16, bool PRE16, int TERMS>
__device__ __forceinline__ void pack_blocks(const PackArgs &a, int64_t first, int64_t step) {
    __shared__ float sums[4][GRAD ? 64 * 8 : 1];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t rows = a.rows_dev ? *a.rows_dev : a.rows, rows_up = (rows + 63) / 64 * 64;
    const bool slope = GRAD && a.act != BDLM_ACT_NONE;
    const int64_t across = (a.ld_dst + 511) / 512, blocks = across * pack_row_blocks(a.rows);
    for (int64_t block = first; block < blocks; block += step) {
        const int64_t down = block / across;
        const int c0 = static_cast<int>(block - down * across) * 512, c = c0 + lane * 8;
        const int64_t r0 = down * kPackRows;
        const int n = a.cols - c;
        float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (c < a.ld_dst) {
            for (int64_t q = r0 + wave; q < r0 + kPackRows && q < rows_up; q += 4 * kPackBatch) {
                Eight<BF16> v[kPackBatch];
                Eight<PRE16> z[kPackBatch];
#pragma unroll
                for (int k = 0; k < kPackBatch; ++k) {
                    const int64_t r = q + 4 * k;
                    const int64_t from = r >= rows ? 0 : a.row_of ? a.row_of[r] : r;
                    v[k].load(a.src, from * a.ld + c, r < rows ? n : 0, c);
                    if (slope) z[k].load(a.pre, from * a.ld_pre + c, r < rows ? n : 0, c);
                }
#pragma unroll
                for (int k = 0; k < kPackBatch; ++k) {
                    const int64_t r = q + 4 * k;
                    float f[8];
                    v[k].settle();
                    if (slope) z[k].settle();
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[e] = v[k].value(e);
                    if constexpr (!GRAD && BF16 && TERMS == 1) {
                        const float scale = a.scale && r < rows ? a.scale[r] : 1.f;
#pragma unroll
                        for (int e = 0; e < 8; ++e) f[e] *= scale;
                    }
                    if constexpr (GRAD) {
                        if (slope) {
#pragma unroll
                            for (int e = 0; e < 8; ++e) f[e] = r < rows && e < n ? f[e] * act_slope<!PRE16>(z[k].value(e), a.act) : 0.f;
                        }
#pragma unroll
                        for (int e = 0; e < 8; ++e) sum[e] += f[e];
                    }
                    if (a.dst && r < rows_up) store_terms<TERMS>(a.dst + r * a.ld_dst + c, a.plane, f);
                }
            }
        }
        if constexpr (GRAD) {
            if (!a.colsum) continue;
#pragma unroll
            for (int e = 0; e < 8; ++e) sums[wave][lane * 8 + e] = sum[e];
            __syncthreads();
            for (int x = threadIdx.x; x < 512; x += 256)
                if (c0 + x < a.cols)
                    a.colsum[down * a.cols + c0 + x] = (sums[0][x] + sums[1][x]) + (sums[2][x] + sums[3][x]);
            __syncthreads();
        }
    }
}
template <bool GRAD, bool BF16, bool PRE16, int TERMS>
__global__ void __launch_bounds__(256) bdlm_pack_kernel(const PackArgs a) {
    pack_blocks<GRAD, BF16, PRE16, TERMS>(a, blockIdx.x, gridDim.x);
}
// Several operands in one launch: operand i has the workgroups from first[i] on.
struct PackSome {
    PackArgs a[kPackMost];
    uint32_t first[kPackMost + 1];
};
template <bool BF16, int TERMS>
__global__ void __launch_bounds__(256) bdlm_pack_some_kernel(const PackSome p) {
    int i = 0;
    for (int j = 1; j < kPackMost; ++j) i = blockIdx.x >= p.first[j] ? j : i;
    pack_blocks<false, BF16, BF16, TERMS>(p.a[i], blockIdx.x - p.first[i], p.first[i + 1] - p.first[i]);
}

// The gradients of a gated product by its factors, as bdlm_pack_kernel lays out the one of a projection: a workgroup takes
// kPackRows rows of 64 x 8 columns, a thread eight columns of two rows at a time, and writes both parts.  With eight waves each
// waits for memory once: with four, which take two turns, 768 x 832 takes 10 us instead of 7.5; where there are workgroups
// for more than a round of the chip four are better, 113 us for 16,384 x 4,096 instead of 124 (kPackWide).  (Four rows a thread at
// a time leave too few waves: 179.)  WHOLE: widths of whole eights, which need fewer registers (16,384 x 1,024 x 4,096 with its products
// 614 us, 631 without the distinction).
constexpr int64_t kPackWide = 2048;   // workgroups
template <int WAVES, bool DH16, bool PRE16, int TERMS, bool WHOLE>
__global__ void __launch_bounds__(64 * WAVES, TERMS == 1 ? 4 : 1) bdlm_gated_pack_kernel(const GatedPackArgs a) {
    constexpr int kBatch = 2;
    __shared__ float sums[2][WAVES][64 * 8];
    static_assert(kPackRows % (kBatch * WAVES) == 0, "whole turns");
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t rows_up = (int64_t(a.rows) + 63) / 64 * 64;
    const int64_t across = (a.ldz + 511) / 512, blocks = across * pack_row_blocks(a.rows);
    for (int64_t block = blockIdx.x; block < blocks; block += gridDim.x) {
        const int64_t down = block / across;
        const int c0 = static_cast<int>(block - down * across) * 512, c = c0 + lane * 8;
        const int64_t r0 = down * kPackRows;
        const int n = a.n - c;
        float sum[2][8] = {};
        if (c < a.ldz) {
            for (int64_t q = r0 + wave; q < r0 + kPackRows && q < rows_up; q += WAVES * kBatch) {
                Eight<DH16, WHOLE> dh[kBatch];
                Eight<PRE16, WHOLE> gate[kBatch], up[kBatch];
#pragma unroll
                for (int k = 0; k < kBatch; ++k) {
                    const int64_t r = q + WAVES * k;
                    if (r >= a.rows) continue;
                    dh[k].load(a.dh, r * a.ld_dh + c, n, c);
                    gate[k].load(a.gate, r * a.ld_pre + c, n, c);
                    up[k].load(a.up, r * a.ld_pre + c, n, c);
                }
#pragma unroll
                for (int k = 0; k < kBatch; ++k) {
                    const int64_t r = q + WAVES * k;
                    if (r >= a.rows) {   // up to a multiple of 64
                        const float zero[8] = {};
                        if (a.dst && r < rows_up) {
                            store_terms<TERMS>(a.dst + r * 2 * a.ldz + c, a.plane, zero);
                            store_terms<TERMS>(a.dst + r * 2 * a.ldz + a.ldz + c, a.plane, zero);
                        }
                        continue;
                    }
                    float f[2][8];
                    dh[k].settle();
                    gate[k].settle();
                    up[k].settle();
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        float value, slope;
                        act_both<!PRE16>(gate[k].value(e), a.act, value, slope);
                        const bool here = WHOLE ? n > 0 : e < n;   // (a slope of no column is not 0)
                        f[0][e] = here ? dh[k].value(e) * up[k].value(e) * slope : 0.f;
                        f[1][e] = here ? dh[k].value(e) * value : 0.f;
                        sum[0][e] += f[0][e];
                        sum[1][e] += f[1][e];
                    }
                    if (a.dst) {
                        store_terms<TERMS>(a.dst + r * 2 * a.ldz + c, a.plane, f[0]);
                        store_terms<TERMS>(a.dst + r * 2 * a.ldz + a.ldz + c, a.plane, f[1]);
                    }
                    __builtin_amdgcn_sched_barrier(0);   // (one row's values in registers at a time)
                }
            }
        }
        if (!a.sum_gate && !a.sum_up) continue;
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int e = 0; e < 8; ++e) sums[p][wave][lane * 8 + e] = sum[p][e];
        __syncthreads();
        for (int x = threadIdx.x; x < 1024; x += 64 * WAVES) {
            const int p = x >> 9, y = x & 511;
            float *to = p ? a.sum_up : a.sum_gate;
            float t = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) t += sums[p][w][y];
            if (to && c0 + y < a.n) to[down * a.n + c0 + y] = t;
        }
        __syncthreads();
    }
}

// Column sums of the blocks' partial sums, of one matrix or two: 64 columns a workgroup, sixteen waves over the blocks,
// eight loads in flight in each.
__global__ void __launch_bounds__(1024) bdlm_colsum_kernel(const float *part, const float *part2, int blocks, int cols, float *out,
                                                          float *out2) {
    __shared__ float sums[16][64];
    if (blockIdx.y) part = part2, out = out2;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int c = blockIdx.x * 64 + lane;
    float s = 0.f;
    if (c < cols) {
        for (int b = wave; b < blocks; b += 128) {
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = b + 16 * k < blocks ? part[int64_t(b + 16 * k) * cols + c] : 0.f;
            s += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
        }
    }
    sums[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && c < cols) {
        s = 0.f;
#pragma unroll
        for (int w = 0; w < 16; ++w) s += sums[w][lane];
        out[c] = s;
    }
}

__device__ __forceinline__ bool counts(int64_t label, int64_t exclude, int vocab) {
    return label >= 0 && label < vocab && label != exclude;
}

// One workgroup lists the rows that count, in order.
__global__ void __launch_bounds__(1024) bdlm_rows_kernel(const RowsArgs a) {
    __shared__ int wave_sum[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int base = 0;
    for (int64_t r0 = 0; r0 < a.rows; r0 += 1024) {
        const int64_t r = r0 + threadIdx.x;
        const int64_t label = r < a.rows ? a.labels[r] : -1;
        const bool ok = counts(label, a.exclude, a.vocab);
        const uint64_t mask = __ballot(ok);
        if (lane == 0) wave_sum[wave] = __popcll(mask);
        __syncthreads();
        int before = base, all = 0;
        for (int w = 0; w < 16; ++w) {
            if (w < wave) before += wave_sum[w];
            all += wave_sum[w];
        }
        if (ok) {
            const int to = before + __popcll(mask & ((uint64_t(1) << lane) - 1));
            a.row_of[to] = static_cast<int32_t>(r);
            a.label[to] = static_cast<int32_t>(label);
            if (a.dloss) {
                a.weight_c[to] = a.dloss[r];
                a.loss_c[to] = a.loss[r];
                a.lse_c[to] = a.lse[r];
                // the label's probability less one is exp(-loss) - 1, without cancellation
                a.scale_c[to] = a.dloss[r] * expm1f(-a.loss[r]);
            }
        }
        base += all;
        __syncthreads();
    }
    if (threadIdx.x == 0) *a.count = base;
}

// One workgroup per row merges its records, four to a lane at a time.
__global__ void __launch_bounds__(256) bdlm_finish_kernel(const FinishArgs a) {
    __shared__ Best waves[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t i = blockIdx.x;
    const int n = a.count ? *a.count : a.rows;
    if (a.labels && threadIdx.x == 0 && !counts(a.labels[i], a.exclude, a.vocab)) {
        a.loss[i] = 0.f;
        a.lse[i] = 0.f;
    }
    if (i >= n) return;
    Best m{-INFINITY, 0.f, kNoColumn};
    for (int t = threadIdx.x; t < a.ntile; t += 1024) {
        Best o[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int64_t at = i * a.ntile + t + 256 * k;
            const bool here = t + 256 * k < a.ntile;
            o[k] = here ? Best{a.top[at], a.others[at], a.at[at]} : Best{-INFINITY, 0.f, kNoColumn};
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) m = merge(m, o[k]);
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const Best o{__shfl_xor(m.top, d, 64), __shfl_xor(m.others, d, 64), __shfl_xor(m.at, d, 64)};
        m = merge(m, o);
    }
    if (lane == 0) waves[wave] = m;
    __syncthreads();
    if (threadIdx.x != 0) return;
#pragma unroll
    for (int w = 1; w < 4; ++w) m = merge(m, waves[w]);
    const float rest = m.top == -INFINITY ? NAN : log1pf(m.others);
    if (a.labels) {
        const int64_t r = a.row_of[i];
        a.loss[r] = rest + (m.top - a.label_logit[i]);
        a.lse[r] = m.top + rest;
    } else {
        a.token[i] = m.top == -INFINITY ? (a.exclude == 0 ? 1 : 0) : m.at;
        a.logprob[i] = -rest;
    }
}

__global__ void __launch_bounds__(256) bdlm_zero_rows_kernel(const int64_t *labels, int64_t exclude, int vocab,
                                                             int rows, char *dx, int64_t ld, int cols, int esz) {
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        if (counts(labels[r], exclude, vocab)) continue;
        for (int c = threadIdx.x; c < cols; c += 256) {
            if (esz == 2) reinterpret_cast<uint16_t *>(dx)[r * ld + c] = 0;
            else reinterpret_cast<float *>(dx)[r * ld + c] = 0.f;
        }
    }
}

int done() { return hipGetLastError() == hipSuccess ? BDLM_OK : BDLM_E_LAUNCH; }

}  // namespace

int launch_pack(const PackArgs &a, void *stream) {
    if (a.rows <= 0) return BDLM_OK;
    const int64_t blocks = (a.ld_dst + 511) / 512 * pack_row_blocks(a.rows);
    const dim3 g(static_cast<unsigned>(blocks < (int64_t(1) << 22) ? blocks : int64_t(1) << 22));
    hipStream_t s = static_cast<hipStream_t>(stream);
    const dim3 b(256);
    const bool grad = a.act != BDLM_ACT_NONE || a.colsum;
    // (dy may be fp32 where the projection's inputs, and pre, are bf16; not the other way round
    // for a plain copy)
    const int kind = (a.terms - 1) * 4 + (a.src_bf16 ? 2 : 0) + (grad ? 1 : 0);
    switch (kind) {
        case 3: hipLaunchKernelGGL((bdlm_pack_kernel<true, true, true, 1>), g, b, 0, s, a); break;
        case 1: hipLaunchKernelGGL((bdlm_pack_kernel<true, false, true, 1>), g, b, 0, s, a); break;
        case 7: hipLaunchKernelGGL((bdlm_pack_kernel<true, true, true, 2>), g, b, 0, s, a); break;
        case 5: hipLaunchKernelGGL((bdlm_pack_kernel<true, false, true, 2>), g, b, 0, s, a); break;
        case 4: hipLaunchKernelGGL((bdlm_pack_kernel<false, false, true, 2>), g, b, 0, s, a); break;
        case 11: hipLaunchKernelGGL((bdlm_pack_kernel<true, true, false, 3>), g, b, 0, s, a); break;
        case 9: hipLaunchKernelGGL((bdlm_pack_kernel<true, false, false, 3>), g, b, 0, s, a); break;
        case 2: hipLaunchKernelGGL((bdlm_pack_kernel<false, true, true, 1>), g, b, 0, s, a); break;
        case 0: hipLaunchKernelGGL((bdlm_pack_kernel<false, false, true, 1>), g, b, 0, s, a); break;
        case 8: hipLaunchKernelGGL((bdlm_pack_kernel<false, false, false, 3>), g, b, 0, s, a); break;
        case 10: hipLaunchKernelGGL((bdlm_pack_kernel<false, true, false, 3>), g, b, 0, s, a); break;
        default: return BDLM_E_LAUNCH;
    }
    return done();
}

template <bool DH16, bool PRE16, int TERMS, bool WHOLE>
int gated_pack_as(const GatedPackArgs &a, hipStream_t s) {
    const int64_t blocks = (a.ldz + 511) / 512 * pack_row_blocks(a.rows);
    const dim3 g(static_cast<unsigned>(blocks < (int64_t(1) << 22) ? blocks : int64_t(1) << 22));
    if (blocks > kPackWide) hipLaunchKernelGGL((bdlm_gated_pack_kernel<4, DH16, PRE16, TERMS, WHOLE>), g, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((bdlm_gated_pack_kernel<8, DH16, PRE16, TERMS, WHOLE>), g, dim3(512), 0, s, a);
    return done();
}

template <bool DH16, bool PRE16, int TERMS>
int gated_pack_of(const GatedPackArgs &a, hipStream_t s) {
    return a.n % 8 == 0 ? gated_pack_as<DH16, PRE16, TERMS, true>(a, s) : gated_pack_as<DH16, PRE16, TERMS, false>(a, s);
}

int launch_gated_pack(const GatedPackArgs &a, void *stream) {
    if (a.rows <= 0) return BDLM_OK;
    hipStream_t s = static_cast<hipStream_t>(stream);
    // (bf16 inputs: one or two terms; fp32: three)
    if (a.terms == 1) return a.dh_bf16 ? gated_pack_of<true, true, 1>(a, s) : gated_pack_of<false, true, 1>(a, s);
    if (a.terms == 2) return a.dh_bf16 ? gated_pack_of<true, true, 2>(a, s) : gated_pack_of<false, true, 2>(a, s);
    return a.dh_bf16 ? gated_pack_of<true, false, 3>(a, s) : gated_pack_of<false, false, 3>(a, s);
}

int launch_pack_some(const PackArgs *a, int32_t n, void *stream) {
    if (n <= 0) return BDLM_OK;
    if (n == 1) return launch_pack(a[0], stream);
    if (n > kPackMost) return BDLM_E_LAUNCH;
    PackSome p{};
    uint32_t at = 0;
    for (int i = 0; i < kPackMost; ++i) {
        p.first[i] = at;
        if (i < n) {
            p.a[i] = a[i];
            const int64_t blocks = a[i].rows > 0 ? (a[i].ld_dst + 511) / 512 * pack_row_blocks(a[i].rows) : 0;
            at += static_cast<uint32_t>(blocks < (int64_t(1) << 22) ? blocks : int64_t(1) << 22);
        }
        p.first[i + 1] = at;
    }
    if (at == 0) return BDLM_OK;
    const dim3 g(at), b(256);
    hipStream_t s = static_cast<hipStream_t>(stream);
    // (as PackArgs of Operand::pack: bf16 in one term, fp32 in three)
    if (a[0].src_bf16) hipLaunchKernelGGL((bdlm_pack_some_kernel<true, 1>), g, b, 0, s, p);
    else hipLaunchKernelGGL((bdlm_pack_some_kernel<false, 3>), g, b, 0, s, p);
    return done();
}

int launch_colsum2(const float *part, const float *part2, int32_t blocks, int32_t cols, float *out, float *out2, void *stream) {
    if (!out || !out2) return out || out2 ? launch_colsum(out ? part : part2, blocks, cols, out ? out : out2, stream) : BDLM_OK;
    hipLaunchKernelGGL(bdlm_colsum_kernel, dim3((cols + 63) / 64, 2), dim3(1024), 0, static_cast<hipStream_t>(stream), part,
                       part2, blocks, cols, out, out2);
    return done();
}

int launch_colsum(const float *part, int32_t blocks, int32_t cols, float *out, void *stream) {
    hipLaunchKernelGGL(bdlm_colsum_kernel, dim3((cols + 63) / 64), dim3(1024), 0, static_cast<hipStream_t>(stream),
                       part, part, blocks, cols, out, out);
    return done();
}

int launch_rows(const RowsArgs &a, void *stream) {
    hipLaunchKernelGGL(bdlm_rows_kernel, dim3(1), dim3(1024), 0, static_cast<hipStream_t>(stream), a);
    return done();
}

int launch_finish(const FinishArgs &a, void *stream) {
    if (a.rows <= 0) return BDLM_OK;
    hipLaunchKernelGGL(bdlm_finish_kernel, dim3(a.rows), dim3(256), 0, static_cast<hipStream_t>(stream), a);
    return done();
}

int launch_zero_rows(const int64_t *labels, int64_t exclude, int32_t vocab, int32_t rows, void *dx, int64_t ld,
                     int32_t cols, int32_t bf16, void *stream) {
    if (rows <= 0) return BDLM_OK;
    hipLaunchKernelGGL(bdlm_zero_rows_kernel, dim3(rows < 4096 ? rows : 4096), dim3(256), 0,
                       static_cast<hipStream_t>(stream), labels, exclude, vocab, rows, static_cast<char *>(dx), ld,
                       cols, bf16 ? 2 : 4);
    return done();
}

}  // namespace bdlm
