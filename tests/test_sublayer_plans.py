"""The plans of a sublayer's operators and of the head's log-probabilities, asked on the CPU of the entry points' own sources:
every kind of launch that tests/test_gpu_sublayer_chain.py means to reach is reached by its sizes, and operands and workspaces
hold what the kernels read and write."""
import ctypes
import os
import subprocess

import pytest

import paper_2607_02805_amd as bd

# The entry points' sources with launches that only take down what they are given.
SHIM = r"""
#include <vector>
#include "bdlm_sublayer_api.cpp"
#include "bdlm_logprobs_api.cpp"
static std::vector<int64_t> seen;
namespace bdlm {
int launch_tile(const TileArgs &a, void *) {
    const int64_t e = tile_edge(a.big), tiles = ((a.nrow + e - 1) / e) * ((a.ncol + e - 1) / e);
    for (int64_t v : {int64_t(a.out), e, int64_t(a.big || tiles * a.splits > kChip ? 2 : 4), int64_t(a.splits),
                      int64_t(2 * a.row_t + a.col_t), int64_t(a.npair), int64_t(a.half)}) seen.push_back(v);
    return BDLM_OK;
}
int launch_join(const float *, int32_t, int32_t, int32_t, int32_t, const int32_t *, const float *, const StoreArgs &,
                void *) { return BDLM_OK; }
int launch_join_two(const float *, int32_t, int32_t, int32_t, void *, int32_t, int32_t, const StoreArgs &, void *) { return BDLM_OK; }
int launch_join_gated(const float *, int32_t, int32_t, const GatedArgs &, void *) { return BDLM_OK; }
int launch_skinny(const SkinnyArgs &a, void *) {
    for (int64_t v : {int64_t(a.out), int64_t(0), int64_t(0), int64_t(0), int64_t(0), int64_t(0), int64_t(0)}) seen.push_back(v);
    return BDLM_OK;
}
int launch_pack(const PackArgs &, void *) { return BDLM_OK; }
int launch_pack_some(const PackArgs *, int32_t, void *) { return BDLM_OK; }
int launch_gated_pack(const GatedPackArgs &, void *) { return BDLM_OK; }
int launch_colsum(const float *, int32_t, int32_t, float *, void *) { return BDLM_OK; }
int launch_colsum2(const float *, const float *, int32_t, int32_t, float *, float *, void *) { return BDLM_OK; }
int launch_logprobs(const LogprobsArgs &, void *) { return BDLM_OK; }
int launch_join_top(const float *, int32_t, int32_t, int32_t, const TopArgs &, void *) { return BDLM_OK; }
int launch_add_norm(const AddNormArgs &, void *) { return BDLM_OK; }
int launch_add_norm_grad(const AddNormGradArgs &, void *) { return BDLM_OK; }
int32_t add_norm_grad_blocks(int64_t rows, int64_t) { return rows > 0; }
}
// Seven numbers a launch, up to `most` of them; how many, or the (negative) status.
extern "C" int launches(int op, int64_t m, int64_t k, int64_t n, int32_t dt, int64_t top, int64_t *out, int most) {
    const bdlm_dense_desc_t d{m, k, n, k, k, dt, 0};
    auto at = [](int i) { return reinterpret_cast<void *>(int64_t(i) << 42); };   // made-up addresses
    auto f = [&](int i) { return static_cast<float *>(at(i)); };
    auto l = [&](int i) { return static_cast<int64_t *>(at(i)); };
    const int64_t room = int64_t(1) << 41;
    seen.clear();
    int rc = BDLM_OK;
    if (op == 0) rc = bdlm_gated_projection(&d, 1, dt, at(1), at(2), at(3), nullptr, nullptr, at(4), n, nullptr, nullptr, 0, at(5), room, nullptr);
    else if (op == 1)
        rc = bdlm_gated_projection_backward(&d, 1, dt, at(1), n, at(2), at(3), at(4), at(5), at(6), n, at(7), k, at(8), at(9), k,
                                            f(10), f(11), at(12), room, nullptr);
    else rc = bdlm_head_logprobs(&d, l(1), -1, top, at(2), at(3), f(4), f(5), l(6), f(7), at(8), room, nullptr);
    if (rc != BDLM_OK) return rc;
    const int n_out = std::min<int>(most, seen.size());
    std::copy_n(seen.begin(), n_out, out);
    return n_out;
}
// Bytes between the parts of the weights that one product reads, and from a part's rows to its copy's end.
extern "C" int64_t between_copies(int64_t m, int64_t k, int64_t n, int32_t dt, int64_t *one) {
    const bdlm_dense_desc_t d{m, k, n, k, k, dt, 0};
    char *base = reinterpret_cast<char *>(int64_t(1) << 42);
    const GatedBackwardPlan p(d, base, base, base, base);
    *one = terms_of(dt) * p.wg.mat.plane;
    return between(p.wg.mat, p.wu.mat);
}
"""

PARTIAL, GATED, GATED_PART, TWO, TOP = 1, 4, 5, 6, 7
F32, BF = bd.DTYPE_F32, bd.DTYPE_BF16


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    d = tmp_path_factory.mktemp("plans")
    src, so = d / "shim.cpp", d / "shim.so"
    src.write_text(SHIM)
    csrc = os.path.join(os.path.dirname(bd.LIB_PATH), "csrc")
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", f"-I{csrc}", f"-I{os.path.dirname(bd.HEADER_PATH)}",
                    str(src), "-o", str(so)], check=True)
    lib = ctypes.CDLL(str(so))
    lib.between_copies.restype = ctypes.c_int64
    return lib


def launches(plans, op, m, k, n, dt, top=0):
    out = (ctypes.c_int64 * 70)()
    i64 = ctypes.c_int64
    got = plans.launches(op, i64(m), i64(k), i64(n), dt, i64(top), out, 70)
    assert got >= 0, got
    return [tuple(out[i:i + 7]) for i in range(0, got, 7)]


# The sizes of tests/test_gpu_sublayer_chain.py, and what each is there for: (kind, tile edge, buffers, whether split, which
# operands are read across their rows: 0 none, 1 the weights, for dx, 3 both, for dw)
GATED_SIZES = {
    (20, 64, 70): {(GATED, 0, 0, False, 0)},
    (40, 64, 30000): {(GATED, 128, 2, False, 0)},
    (40, 64, 70): {(GATED, 128, 4, False, 0)},
    (300, 64, 12000): {(GATED, 256, 2, False, 0)},
    (4096, 128, 2048): {(GATED, 256, 2, False, 0)},        # rows of a multiple of 512, which are stored one matrix after the other
    (40, 1600, 70): {(GATED_PART, 128, 4, True, 0)},
    (20000, 4096, 70): {(GATED_PART, 256, 2, True, 0)},
}
GRAD_SIZES = {
    (20, 64, 30000): {(TWO, 128, 2, False, 3)},
    (20, 64, 70): {(TWO, 128, 4, False, 3), (TWO, 128, 4, False, 1)},
    (20, 512, 4100): {(TWO, 256, 2, False, 3)},
    (1000, 64, 70): {(PARTIAL, 128, 4, True, 3)},
    (20, 64, 260): {(PARTIAL, 128, 4, True, 1)},
    (20000, 64, 4100): {(PARTIAL, 128, 2, True, 3)},
    (4500, 192, 4100): {(PARTIAL, 256, 2, True, 3), (PARTIAL, 256, 2, True, 1)},
    (4500, 1600, 70): {(TWO, 128, 2, False, 1)},
    (20000, 192, 70): {(TWO, 256, 2, False, 1)},
    (20, 4096, 5300): {(PARTIAL, 128, 2, True, 1)},
}
TOP_SIZES = {(20, 64, 70): {(TOP, 0, 0, False, 0)}, (40, 64, 70): {(TOP, 128, 4, False, 0)}, (300, 64, 12000): {(TOP, 128, 2, False, 0)},
             (2000, 64, 4100): {(TOP, 256, 2, False, 0)},
             (40, 1600, 1100): {(PARTIAL, 128, 4, True, 0)}, (1000, 4096, 4101): {(PARTIAL, 256, 2, True, 0)}}


def kinds(got):
    return {(g[0], g[1], g[2], g[3] > 1, g[4]) for g in got}


def test_the_gpu_tests_reach_every_kind_of_launch(plans):
    for op, sizes in ((0, GATED_SIZES), (1, GRAD_SIZES), (2, TOP_SIZES)):
        for (m, k, n), want in sizes.items():
            got = kinds(launches(plans, op, m, k, n, BF, top=3))
            assert want <= got, (op, m, k, n, got)


@pytest.mark.parametrize("dt", [F32, BF])
def test_pairs_of_planes(plans, dt):
    """dx is one product over both parts: twice the pairs of dw, the second half from `half` on."""
    for m in (8, 64, 65, 300):
        dx, dw = launches(plans, 1, m, 128, 96, dt)
        pairs = 6 if dt == F32 else 2 if m <= 64 else 1
        assert (dx[5], dx[6]) == (2 * pairs, pairs) and (dw[5], dw[6]) == (pairs, pairs)
        assert dx[4] == 1 and dw[4] == 3                   # the weights, and both of dw's, are read across their rows


@pytest.mark.parametrize("size", [(100, 100, 50), (100, 64, 64), (5, 33, 7), (1000, 130, 4097)])
def test_copies_of_both_weights_lie_one_behind_the_other(plans, size):
    one = ctypes.c_int64(0)
    for dt in (F32, BF):
        i64 = ctypes.c_int64
        if dt == BF and size[1] % 64 == 0:
            continue                                       # read as they lie
        assert plans.between_copies(i64(size[0]), i64(size[1]), i64(size[2]), dt, ctypes.byref(one)) == one.value > 0


def test_every_size_has_a_plan_or_is_refused(plans):
    """The largest rows and features: either what a launch holds, or BDLM_E_SHAPE, never more."""
    i64 = ctypes.c_int64
    out = (ctypes.c_int64 * 70)()
    big = 1 << 22
    for op in (0, 1, 2):
        for m, k, n in ((big, 64, 64), (64, big, 64), (64, 64, big), (big, big, big), (1, big, big), (big, 1, big)):
            got = plans.launches(op, i64(m), i64(k), i64(n), BF, i64(2), out, 70)
            assert got in (bd.E_SHAPE, bd.E_WORKSPACE) or got > 0, (op, m, k, n, got)
            for i in range(0, max(got, 0), 7):
                assert out[i + 1] in (0, 128, 256)
