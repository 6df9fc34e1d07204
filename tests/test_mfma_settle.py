"""The generated gfx950 code of the tiled products waits before it touches an accumulator.

The products of bdlm_tile.hip are written as inline assembly, so the compiler does not add the
wait states that a product's result needs before another instruction reads or writes it (at
most 19; another product on the same registers needs none).  This test follows
the generated code in program order: no instruction but a product may touch an accumulator of a
product issued fewer than 19 wait states before.
"""
import os
import re
import shutil
import subprocess
import tempfile

import pytest

from paper_2607_02805_amd import build

WAIT = 19


def _acc(text):
    """Numbers of the accumulation registers an instruction names."""
    got = set()
    for m in re.finditer(r"\ba\[(\d+):(\d+)\]|\ba(\d+)\b", text):
        lo = int(m.group(1) or m.group(3))
        got |= set(range(lo, int(m.group(2) or lo) + 1))
    return got


def early_touches(asm: str):
    """(function, product, instruction) for each accumulator touched too early."""
    found = []
    for block in re.split(r"\n(?=_Z\w+:)", asm):
        m = re.match(r"(_Z\w+):", block)
        if not m or "v_mfma" not in block:
            continue
        age, by = {}, {}           # register: wait states since its product, the product
        for line in block.splitlines()[1:]:
            line = line.split(";")[0].strip()
            if not line or line.startswith(".") or line.endswith(":"):
                continue
            op = line.split()[0]
            if op.startswith("v_mfma"):
                for r in age:
                    age[r] += 1
                for r in _acc(line.split(",")[0]):
                    age[r], by[r] = 0, line
                continue
            for r in _acc(line):
                if age.get(r, WAIT) < WAIT:
                    found.append((m.group(1)[:70], by[r], line))
            states = int(line.split()[1]) + 1 if op == "s_nop" else 1
            for r in age:
                age[r] += states
    return found


@pytest.fixture(scope="module")
def tile_asm():
    if not (os.path.exists(build.HIPCC) or shutil.which(build.HIPCC)):
        pytest.skip("hipcc not available")
    with tempfile.TemporaryDirectory() as d:
        out = os.path.join(d, "tile.s")
        cmd = [build.HIPCC, *build.HIP_FLAGS, f"-I{build.INCLUDE}", f"-I{build.CSRC}", "--cuda-device-only",
               "-S", os.path.join(build.CSRC, "bdlm_tile.hip"), "-o", out]
        r = subprocess.run(cmd, capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-2000:]
        yield open(out).read()


def test_accumulators_settle_before_they_are_touched(tile_asm):
    assert tile_asm.count("v_mfma") > 300
    assert early_touches(tile_asm) == []


def test_products_stay_in_place(tile_asm):
    """Every product adds onto its own registers and none lives in scratch memory."""
    for line in tile_asm.splitlines():
        if line.strip().startswith("v_mfma"):
            ops = line.replace(";", " ").split(None, 1)[1].replace(" ", "").split(",")
            assert ops[0] == ops[3], line
    sizes = re.findall(r"; ScratchSize: (\d+)", tile_asm)
    assert sizes and all(s == "0" for s in sizes)


def test_the_scan_finds_a_planted_touch():
    head = "_ZN4bdlm1fEv:\n"
    product = "\tv_mfma_f32_16x16x32_bf16 a[4:7], v[8:11], v[12:15], a[4:7]\n"
    assert len(early_touches(head + product + "\tv_accvgpr_read_b32 v2, a5\n")) == 1
    assert len(early_touches(head + product + "\ts_nop 8\n\tds_write_b128 v2, a[4:7]\n")) == 4
    assert early_touches(head + product + "\ts_nop 15\n\ts_nop 3\n\tv_accvgpr_read_b32 v2, a5\n") == []
    assert early_touches(head + product + "\tv_accvgpr_read_b32 v2, a8\n") == []
    assert early_touches(head + product + product) == []
