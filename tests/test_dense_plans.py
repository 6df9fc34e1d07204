"""The plans of the dense operators, asked on the CPU of the entry points' own source: tiles, splits, pieces of the
vocabulary, and what fits a launch."""
import ctypes
import math
import os
import subprocess

import pytest

import paper_2607_02805_amd as bd

# The entry points' source with launches that only take down what they are given.
SHIM = r"""
#include <vector>
#include "bdlm_dense_api.cpp"
static std::vector<int64_t> seen;
namespace bdlm {
int launch_tile(const TileArgs &a, void *) {
    const int64_t e = tile_edge(a.big), tiles = ((a.nrow + e - 1) / e) * ((a.ncol + e - 1) / e);
    // (splits of 0: the device chooses them; this many if every row counts)
    const int64_t splits = a.splits ? a.splits : split_count(tiles);
    const int64_t groups = a.splits ? tiles * splits : std::max<int64_t>(tiles, kChip);
    for (int64_t v : {e, int64_t(a.big || groups > kChip ? 2 : 4), int64_t(2 * a.row_t + a.col_t), int64_t(a.out),
                      int64_t(a.npair), steps_of(a.k, a.npair) / splits, int64_t(a.ncol % e || a.nrow % e)})
        seen.push_back(v);
    return BDLM_OK;
}
int launch_join(const float *, int32_t, int32_t, int32_t, int32_t, const int32_t *, const float *, const StoreArgs &,
                void *) { return BDLM_OK; }
int launch_skinny(const SkinnyArgs &, void *) { return BDLM_OK; }
int launch_pack(const PackArgs &, void *) { return BDLM_OK; }
int launch_colsum(const float *, int32_t, int32_t, float *, void *) { return BDLM_OK; }
int launch_rows(const RowsArgs &, void *) { return BDLM_OK; }
int launch_finish(const FinishArgs &, void *) { return BDLM_OK; }
int launch_zero_rows(const int64_t *, int64_t, int32_t, int32_t, void *, int64_t, int32_t, int32_t, void *) { return BDLM_OK; }
}
extern "C" int fits(int64_t tiles) { return launch_fits(tiles); }
extern "C" int64_t piece(int64_t m, int64_t k, int64_t n, int32_t dt) {
    bdlm_dense_desc_t d;
    bdlm_dense_desc_init(&d, m, k, n, dt);
    return LossBackwardPlan(d, nullptr, nullptr, nullptr).piece;
}
// Seven numbers a launch, up to `most` of them; how many, or the (negative) status.
extern "C" int launches(int op, int64_t m, int64_t k, int64_t n, int32_t dt, int64_t *out, int most) {
    bdlm_dense_desc_t d;
    bdlm_dense_desc_init(&d, m, k, n, dt);
    auto at = [](int i) { return reinterpret_cast<void *>(int64_t(i) << 42); };   // made-up addresses
    auto f = [&](int i) { return static_cast<float *>(at(i)); };
    auto l = [&](int i) { return static_cast<int64_t *>(at(i)); };
    const int64_t room = int64_t(1) << 41;
    seen.clear();
    int rc = BDLM_OK;
    switch (op) {
        case 0: rc = bdlm_projection(&d, 0, dt, at(1), at(2), nullptr, nullptr, 0, at(3), n, nullptr, 0, at(4), room, nullptr); break;
        case 1: rc = bdlm_projection_backward(&d, 1, dt, at(1), n, at(2), at(3), at(4), n, at(5), k, at(6), k, f(7), at(8), room, nullptr); break;
        case 2: rc = bdlm_head_loss(&d, l(1), -1, at(2), at(3), f(4), f(5), at(6), room, nullptr); break;
        case 3: rc = bdlm_head_loss_backward(&d, l(1), -1, at(2), at(3), f(4), f(5), f(6), at(7), k, at(8), k, at(9), room, nullptr); break;
        default: rc = bdlm_head_select(&d, -1, at(1), at(2), l(3), f(4), at(5), room, nullptr);
    }
    if (rc != BDLM_OK) return rc;
    const int n_out = std::min<int>(most, seen.size());
    std::copy_n(seen.begin(), n_out, out);
    return n_out;
}
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    d = tmp_path_factory.mktemp("plans")
    src, so = d / "shim.cpp", d / "shim.so"
    src.write_text(SHIM)
    csrc = os.path.join(os.path.dirname(bd.LIB_PATH), "csrc")
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", f"-I{csrc}", f"-I{os.path.dirname(bd.HEADER_PATH)}",
                    str(src), "-o", str(so)], check=True)
    return ctypes.CDLL(str(so))


def test_a_launch_holds_fewer_than_2_to_the_32_threads(plans):
    """Workgroups of large and of small tiles have 512 threads."""
    for tiles in (1, 1 << 22, (1 << 23) - 1):
        assert plans.fits(ctypes.c_int64(tiles))
    for tiles in (1 << 23, (1 << 24) - 1, 1 << 24, 1 << 40):
        assert not plans.fits(ctypes.c_int64(tiles))


def launches(plans, op, m, k, n, dtype):
    """The tiled launches of a call: ((edge, buffers, layout, output, pairs of planes), steps of a workgroup, ragged)."""
    buf = (ctypes.c_int64 * 2800)()
    got = plans.launches(op, ctypes.c_int64(m), ctypes.c_int64(k), ctypes.c_int64(n), dtype, buf, len(buf))
    assert got >= 0, (op, m, k, n, dtype, got)
    return [(tuple(buf[i:i + 5]), buf[i + 5], bool(buf[i + 6])) for i in range(0, got, 7)]


def test_every_tile_kernel_is_run_by_a_test(plans):
    """What the plans of 20,000 drawn calls and of the timed cases choose, the GPU tests' sizes choose too: several
    stages deep (past the ring of buffers), with a tile that ends inside the matrix."""
    import random

    import torch

    import perf.operators
    from tests.test_gpu_dense_more import HEADS, PROJECTIONS
    code = {torch.float32: bd.DTYPE_F32, torch.bfloat16: bd.DTYPE_BF16}
    run = set()
    for sizes, ops in ((PROJECTIONS, (0, 1)), (HEADS, (2, 3, 4))):
        for m, k, n, dtype in sizes:
            for op in ops:
                for kernel, steps, ragged in launches(plans, op, m, k, n, code[dtype]):
                    # (two terms of up to 64 rows are one stage each)
                    deep = 2 if kernel[2:] == (3, 0, 2) else 5 if kernel[1] == 4 else 3
                    if steps >= deep and ragged:
                        run.add(kernel)
    rng = random.Random(7)

    def size(lo, hi):
        return round(math.exp(rng.uniform(math.log(lo), math.log(hi))))
    calls = [(op, size(1, 40000), size(1, 8000), size(1, 140000 if op > 1 else 20000), rng.randrange(2))
             for op in (rng.randrange(5) for _ in range(20000))]
    kinds = {"project": (0,), "project_grad": (1,), "select": (4,), "loss": (2,), "loss_grad": (2, 3)}
    for c in perf.operators.listed():
        calls += [(op, c["rows"], c["k"], c["n"], bd.DTYPE_F32 if c["dtype"] == "fp32" else bd.DTYPE_BF16)
                  for op in kinds[c["kind"]]]
    for call in calls:
        for kernel, _, _ in launches(plans, *call):
            assert kernel in run, (call, kernel)
    assert len(run) >= 54


def test_the_pieces_of_the_gpu_tests(plans):
    import torch

    from tests.test_gpu_dense_more import PIECES
    plans.piece.restype = ctypes.c_int64
    for m, k, n, dtype, _, piece in PIECES:
        code = bd.DTYPE_F32 if dtype == torch.float32 else bd.DTYPE_BF16
        got = plans.piece(ctypes.c_int64(m), ctypes.c_int64(k), ctypes.c_int64(n), code)
        assert got == piece and 2 * got < n < 3 * got
        # no piece takes more than 512 MB, as its floor of 4,096 columns is not reached
        assert m * got * (6 if dtype == torch.float32 else 2) <= 512 << 20
