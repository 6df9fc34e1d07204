// bdlm_logprobs.hip -- gfx950 kernel that makes a row's log-probability, entropy and most probable tokens of the records and
// values that the products of the head leave (TopArgs in bdlm_dense.h).
//
// One workgroup per row.  With M the largest value, o and l a group's sums of exp(d) and exp(d) d over all but one of its
// columns, and f = exp(top - M), D = top - M:
//     Z = 1 + others,  others = sum (1 + o) f less the largest one's own 1,  slope = sum f (l + D (1 + o)),
//     lse = M + log Z,  entropy = log Z - slope / Z   (both terms positive).
// The k largest values: of 16 or 64 parts of the groups, the k-th largest part's maximum is a bound that at least k values
// reach.  Values that reach it, mostly a few more than k, are gathered and each counts the ones before it, in the order of
// values and then columns: a count below k is its place.  (Listing them one after the other took 18 us for one row of
// 1,024 groups.)  Where too many reach the bound, as where all are equal, the first wave lists them one after the other.
//
// Bound by latency: the records, the values, three meetings of the waves.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "bdlm.h"
#include "bdlm_dense.h"
#include "bdlm_dense_device.h"
#include "bdlm_store.h"

namespace bdlm {
namespace {

template <int V>
struct Number {
    static constexpr int value = V;
};

// Largest value of LANES consecutive lanes (1 or 4: in each of them, 16: in the last, 64: in every lane).
template <int LANES>
__device__ __forceinline__ float largest(float v) {
    auto step = [&](auto ctrl, auto mask) {
        const int o = __builtin_amdgcn_update_dpp(__float_as_int(v), __float_as_int(v), decltype(ctrl)::value,
                                                  decltype(mask)::value, 0xf, false);
        v = fmaxf(v, __int_as_float(o));
    };
    if constexpr (LANES == 1) return v;
    if constexpr (LANES == 4) {
        step(Number<0xb1>{}, Number<0xf>{});    // quad_perm [1,0,3,2], [2,3,0,1]
        step(Number<0x4e>{}, Number<0xf>{});
        return v;
    }
    step(Number<0x111>{}, Number<0xf>{});   // row_shr:1, 2, 4, 8
    step(Number<0x112>{}, Number<0xf>{});
    step(Number<0x114>{}, Number<0xf>{});
    step(Number<0x118>{}, Number<0xf>{});
    if constexpr (LANES == 64) {
        step(Number<0x142>{}, Number<0xa>{});   // row_bcast:15 into rows 1 and 3
        step(Number<0x143>{}, Number<0xc>{});   // row_bcast:31 into rows 2 and 3
        v = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
    }
    return v;
}
__device__ __forceinline__ float wave_total(float v) {
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(wave_inclusive_sum(v)), 63));
}
__device__ __forceinline__ bool before(float v, int at, float u, int n) { return v > u || (v == u && at < n); }

// A wave's list of the k largest values seen, in order, entry j in lane j: of equal ones the lowest number first.  An empty
// entry is (-infinity, kNoColumn).
struct TopList {
    float v;
    int at;
    __device__ __forceinline__ TopList() : v(-INFINITY), at(kNoColumn) {}
    // One value a lane.  Every turn lists the first of those that come before the last entry.
    __device__ __forceinline__ void add(float u, int n, int k, int lane) {
        if (!(u > -INFINITY)) n = kNoColumn;   // (NaN as well)
        for (;;) {
            const float last = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), k - 1));
            const int last_at = __builtin_amdgcn_readlane(at, k - 1);
            const bool can = n != kNoColumn && before(u, n, last, last_at);
            if (!__ballot(can)) return;
            const float m = largest<64>(can ? u : -INFINITY);
            uint64_t eq = __ballot(can && u == m);
            int src = __ffsll(static_cast<unsigned long long>(eq)) - 1;
            int number = __builtin_amdgcn_readlane(n, src);
            for (eq &= eq - 1; eq; eq &= eq - 1) {   // equal values: the lowest number
                const int other = __ffsll(static_cast<unsigned long long>(eq)) - 1, t = __builtin_amdgcn_readlane(n, other);
                if (t < number) number = t, src = other;
            }
            if (lane == src) n = kNoColumn;
            const int place = __popcll(__ballot(lane < k && before(v, at, m, number)));
            const float up_v = __shfl_up(v, 1, 64);
            const int up_at = __shfl_up(at, 1, 64);
            if (lane > place) v = up_v, at = up_at;
            if (lane == place) v = m, at = number;
        }
    }
};

// f over the 16 lanes of a row, in each of them.
template <class F>
__device__ __forceinline__ float over_row(float v, F f) {
    auto step = [&](auto ctrl) {
        v = f(v, __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(v), __float_as_int(v), decltype(ctrl)::value, 0xf, 0xf, false)));
    };
    step(Number<0x121>{});   // row_ror:1, 2, 4, 8
    step(Number<0x122>{});
    step(Number<0x124>{});
    step(Number<0x128>{});
    return v;
}

// A lane has four columns of a row, 16 lanes a group.
__global__ void __launch_bounds__(256) bdlm_join_top_kernel(const float *part, int splits, int nrow, int ncol, const TopArgs t) {
    static_assert(kJoinGroup == 64, "16 lanes of four columns");
    const int across = (ncol + 1023) / 1024;
    const int64_t slice = int64_t(nrow) * ncol, all = int64_t(nrow) * across;
    for (int64_t block = blockIdx.x; block < all; block += gridDim.x) {
        const int64_t r = block / across;
        const int c = static_cast<int>(block - r * across) * 1024 + threadIdx.x * 4, group = c / kJoinGroup;
        const float *p = part + r * ncol + c;
        f32x4 v = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        if (c + 4 <= ncol) {
            v = sum_slices(p, slice, splits);
        } else {
            for (int e = 0; e < 4; ++e)
                if (c + e < ncol) {
                    v[e] = 0.f;
                    for (int k = 0; k < splits; ++k) v[e] += p[k * slice + e];
                }
        }
        const int64_t token = t.token ? t.token[r] : -1;
        float top = -INFINITY;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (c + e == t.exclude) v[e] = -INFINITY;
            if (c + e == token && c + e < ncol) t.token_logit[r] = v[e];
            top = fmaxf(top, v[e]);
        }
        if (t.list > 0 && group < t.ngroup)
            *reinterpret_cast<f32x4 *>(t.value + r * t.ngroup * kJoinGroup + c) = v;
        const float m = over_row(top, [](float x, float y) { return fmaxf(x, y); });
        // the first of the 64 columns that holds it (a number that is exact as a float) stays out of the sums
        float at = 64.f;
#pragma unroll
        for (int e = 3; e >= 0; --e) at = v[e] == m ? static_cast<float>(4 * (threadIdx.x & 15) + e) : at;
        at = over_row(at, [](float x, float y) { return fminf(x, y); });
        const float ref = m == -INFINITY ? 0.f : m;
        float others = 0.f, slope = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (at == static_cast<float>(4 * (threadIdx.x & 15) + e)) continue;
            const float s = __builtin_amdgcn_exp2f((v[e] - ref) * kLog2e);
            others += s;
            slope += slope_of(s, v[e] - ref);
        }
        auto sum = [](float x, float y) { return x + y; };
        others = over_row(others, sum);
        slope = over_row(slope, sum);
        if ((threadIdx.x & 15) == 0 && group < t.ngroup) {
            const int64_t o = r * t.ngroup + group;
            t.top[o] = m;
            t.others[o] = others;
            t.slope[o] = slope;
        }
    }
}

constexpr int kParts = 64;         // of the groups
static_assert(BDLM_MAX_TOP <= kParts, "as many parts as values");
constexpr int kRoom = 256;         // gathered groups, and values

// A gathered value.
struct alignas(8) Entry {
    float v;
    int at;
};

constexpr int32_t kWaveRows = 256;

template <int T>   // threads
__global__ void __launch_bounds__(T) bdlm_logprobs_kernel(const LogprobsArgs a) {
    constexpr int kWaves = T / 64, kLanes = T / kParts, kKeep = 4;   // lanes of a part
    static_assert(kLanes == 1 || kLanes == 4 || kLanes == 16, "a lane, a quad or a row of lanes");
    __shared__ float parts[kParts], sums[2][kWaves];
    __shared__ float firsts[kWaves];
    __shared__ int ngathered, nvalues;
    __shared__ int group[kRoom];
    __shared__ Entry entry[kRoom];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t i = blockIdx.x;
    const int k = a.list;
    const float *top = a.top + i * a.ngroup, *others = a.others + i * a.ngroup, *slopes = a.slope + i * a.ngroup;
    // Groups go to the parts in turn, so that few of them do not lie in few parts (34 groups for each of 4,032 rows, in the
    // lanes' order: 26 us instead of 9).  The first kKeep * T groups stay in registers.
    const int own = (tid & (kLanes - 1)) * kParts + tid / kLanes;
    Spread g[kKeep];
    float most = -INFINITY;
#pragma unroll
    for (int j = 0; j < kKeep; ++j) {
        const int x = own + T * j;
        g[j] = x < a.ngroup ? Spread{top[x], others[x], slopes[x]} : Spread{-INFINITY, 0.f, 0.f};
    }
    const int64_t token = a.token ? a.token[i] : -1;
    const bool given = token >= 0 && token < a.vocab;
    const float token_logit = given ? a.token_logit[i] : 0.f;
#pragma unroll
    for (int j = 0; j < kKeep; ++j) most = fmaxf(most, g[j].top);
    for (int x = own + T * kKeep; x < a.ngroup; x += T) most = fmaxf(most, top[x]);
    most = largest<kLanes>(most);
    if ((tid & (kLanes - 1)) == kLanes - 1) parts[tid / kLanes] = most;
    if (tid == 0) ngathered = nvalues = 0;
    static_assert(kRoom % 16 == 0, "whole turns of the count");
    for (int x = tid; x < kRoom; x += T) entry[x] = Entry{-INFINITY, kNoColumn};   // (before none)
    __syncthreads();
    float mine = parts[lane];
    const float m = largest<64>(mine);
    // The k-th largest of the parts' maxima.  Of 64 parts a few more than k groups reach it; 16 of them, each of four, are
    // enough up to k = 8 (11 groups), not for 16 (54).
    float bound = -INFINITY;
    if (k > 0) {
        int rank = 0;
        auto count = [&](auto step_) {
            constexpr int step = decltype(step_)::value;
#pragma unroll
            for (int j = 0; j < kParts; j += step) {
                const float v = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(mine), j));
                rank += before(v, j, mine, lane);
            }
            return __ballot(rank == k - 1 && lane % step == 0);
        };
        uint64_t at;
        if (k > 8) {
            at = count(Number<1>{});
        } else {
            mine = largest<4>(mine);
            at = count(Number<4>{});
        }
        bound = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(mine), __ffsll(static_cast<unsigned long long>(at)) - 1));
    }
    float s_others = 0.f, s_slope = 0.f;
    float largest_ones = 0.f;
    auto take = [&](const Spread &s, int x) {
        const float f = share(s.top, m);
        if (s.top == m && m > -INFINITY) {
            largest_ones += 1.f;
            s_others += s.others;
            s_slope += s.slope;
        } else if (f != 0.f) {
            s_others = fmaf(1.f + s.others, f, s_others);
            s_slope = fmaf(fmaf(s.top - m, 1.f + s.others, s.slope), f, s_slope);
        } else if (s.others != s.others) {   // a NaN stays one
            s_others = s_slope = s.others;
        }
        if (k > 0 && s.top >= bound && s.top > -INFINITY) {
            const int n = atomicAdd(&ngathered, 1);   // (whatever the order: the places are counted below)
            if (n < kRoom) group[n] = x;
        }
    };
#pragma unroll
    for (int j = 0; j < kKeep; ++j) take(g[j], own + T * j);
    for (int x = own + T * kKeep; x < a.ngroup; x += T) take(Spread{top[x], others[x], slopes[x]}, x);
    s_others = wave_total(s_others);
    s_slope = wave_total(s_slope);
    largest_ones = wave_total(largest_ones);
    if (lane == 0) sums[0][wave] = s_others, sums[1][wave] = s_slope, firsts[wave] = largest_ones;
    __syncthreads();
    float z = 0.f, slope = 0.f;
    float ones = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) z += sums[0][w], slope += sums[1][w], ones += firsts[w];
    z += fmaxf(ones - 1.f, 0.f);   // the largest one's own 1 stays out
    const float rest = fabsf(m) < INFINITY ? log1pf(z) : NAN;
    if (tid == 0) {
        if (a.entropy) a.entropy[i] = rest - slope / (1.f + z);
        if (a.token) a.logprob[i] = given ? (token_logit - m) - rest : 0.f;
    }
    if (k == 0) return;
    auto put = [&](int place, float v, int at) {
        const bool here = at != kNoColumn;
        a.top_token[i * k + place] = here ? at : -1;
        a.top_logprob[i * k + place] = here ? (v - m) - rest : -INFINITY;
    };
    const int ng = ngathered;
    if (ng <= kRoom) {
        // Four values of a thread are asked for at a time, with their columns.  (x / width by a product: x is below 2^16.)
        const uint32_t inverse = (0xffffffffu / static_cast<uint32_t>(a.width)) + 1u;
        const int all = ng * a.width;
        for (int x0 = tid; x0 < all; x0 += 4 * T) {
            float v[4];
            int c[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int x = x0 + T * q;
                const bool here = x < all;
                const int which = here ? (a.width > 1 ? static_cast<int>(__umulhi(x, inverse)) : x) : 0, j = x - which * a.width;
                const int from = group[which];
                const int64_t at = (i * a.ngroup + from) * a.width + j;
                v[q] = here ? a.value[at] : -INFINITY;
                c[q] = !here ? kNoColumn : a.column ? a.column[at] : from * a.width + j;
            }
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (v[q] >= bound && v[q] > -INFINITY) {
                    const int n = atomicAdd(&nvalues, 1);
                    if (n < kRoom) entry[n] = Entry{v[q], c[q]};
                }
        }
    }
    __syncthreads();
    const int nv = nvalues;
    if (ng <= kRoom && nv <= kRoom) {
        // four lanes count for an entry
        for (int x = tid >> 2; x < nv; x += T / 4) {
            const Entry e = entry[x];
            int place = 0;
            for (int j = tid & 3; j < nv; j += 16) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const Entry o = entry[j + 4 * q];
                    place += before(o.v, o.at, e.v, e.at);
                }
            }
            place += __builtin_amdgcn_update_dpp(0, place, 0xb1, 0xf, 0xf, true);
            place += __builtin_amdgcn_update_dpp(0, place, 0x4e, 0xf, 0xf, true);
            if ((tid & 3) == 0 && place < k) put(place, e.v, e.at);
        }
        if (tid >= nv && tid < k) put(tid, 0.f, kNoColumn);   // fewer than k: the rest of the list is empty
        return;
    }
    // The k largest lie in the k groups whose largest values (then the lower columns) come first: were one in another group, each of
    // those k would hold one before it.
    if (wave != 0) return;
    TopList list;
    for (int x = lane; x - lane < a.ngroup; x += 64) list.add(x < a.ngroup ? top[x] : -INFINITY, x, k, lane);
    const TopList groups = list;
    list = TopList();
    for (int x0 = 0; x0 < k * a.width; x0 += 64) {
        const int x = x0 + lane, which = x < k * a.width ? x / a.width : 0, j = x - which * a.width;
        const int from = __shfl(groups.at, which, 64);
        const int64_t at = (i * a.ngroup + from) * a.width + j;
        const bool here = x < k * a.width && from != kNoColumn;
        const float v = here ? a.value[at] : -INFINITY;
        list.add(v, !here ? kNoColumn : a.column ? a.column[at] : from * a.width + j, k, lane);
    }
    if (lane < k) put(lane, list.v, list.at);
}

}  // namespace

int launch_logprobs(const LogprobsArgs &a, void *stream) {
    if (a.rows <= 0) return BDLM_OK;
    hipStream_t s = static_cast<hipStream_t>(stream);
    // Few rows, or many groups: more threads hold them all.  Many rows of few groups: a wave each.
    if (a.ngroup <= 256 && a.rows > kWaveRows) hipLaunchKernelGGL(bdlm_logprobs_kernel<64>, dim3(a.rows), dim3(64), 0, s, a);
    else if (a.ngroup > 1024 || a.rows <= 256) hipLaunchKernelGGL(bdlm_logprobs_kernel<1024>, dim3(a.rows), dim3(1024), 0, s, a);
    else hipLaunchKernelGGL(bdlm_logprobs_kernel<256>, dim3(a.rows), dim3(256), 0, s, a);
    return hipGetLastError() == hipSuccess ? BDLM_OK : BDLM_E_LAUNCH;
}

int launch_join_top(const float *part, int32_t splits, int32_t nrow, int32_t ncol, const TopArgs &t, void *stream) {
    if (nrow <= 0 || ncol <= 0) return BDLM_OK;
    const int64_t blocks = int64_t(nrow) * ((ncol + 1023) / 1024);
    hipLaunchKernelGGL(bdlm_join_top_kernel, dim3(static_cast<unsigned>(blocks < (1 << 20) ? blocks : 1 << 20)), dim3(256), 0,
                       static_cast<hipStream_t>(stream), part, splits, nrow, ncol, t);
    return hipGetLastError() == hipSuccess ? BDLM_OK : BDLM_E_LAUNCH;
}

}  // namespace bdlm
