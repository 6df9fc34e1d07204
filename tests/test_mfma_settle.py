"""The generated gfx950 code of the tiled products waits before it touches an accumulator.

The products of bdlm_tile.hip are written as inline assembly, so the compiler does not add the
wait states that a product's result needs before another instruction reads or writes it (at
most 19; another product on the same registers needs none).  This test follows
the generated code along every path: no instruction but a product may touch an accumulator of a
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


def _blocks(lines):
    """Basic blocks [(instructions, successors)] of a function's lines, in order."""
    blocks, names = [[[], None]], {}
    for line in lines:
        line = line.split(";")[0].strip()
        label = re.match(r"(\.L\w+):$", line)
        if label:
            names[label.group(1)] = len(blocks)
            blocks.append([[], None])
        elif line and not line.startswith(".") and not line.endswith(":"):
            blocks[-1][0].append(line)
            if re.match(r"s_c?branch|s_endpgm", line):
                blocks[-1][1] = line
                blocks.append([[], None])
    out = []
    for n, (code, end) in enumerate(blocks):
        after = [n + 1] if n + 1 < len(blocks) and not (end or "").startswith(("s_branch", "s_endpgm")) else []
        target = re.search(r"\.L\w+", end or "")
        out.append((code, after + ([names[target.group(0)]] if target else [])))
    return out


def early_touches(asm: str):
    """(function, product, instruction) for each accumulator touched too early on any path."""
    found = set()
    for block in re.split(r"\n(?=_Z\w+:)", asm):
        m = re.match(r"(_Z\w+):", block)
        if not m or "v_mfma" not in block:
            continue
        blocks = _blocks(block.split(".Lfunc_end")[0].splitlines()[1:])
        entry = {0: {}}            # block: {register: (wait states since its product, the product)}
        todo = [0]
        while todo:
            n = todo.pop()
            age = dict(entry[n])
            for line in blocks[n][0]:
                op = line.split()[0]
                if op.startswith("v_mfma"):
                    age = {r: (a + 1, by) for r, (a, by) in age.items()}
                    age.update({r: (0, line) for r in _acc(line.split(",")[0])})
                    continue
                found |= {(m.group(1)[:70], age[r][1], line) + (r,) for r in _acc(line) if r in age}
                states = int(line.split()[1]) + 1 if op == "s_nop" else 1
                age = {r: (a + states, by) for r, (a, by) in age.items() if a + states < WAIT}
            for to in blocks[n][1]:
                known = entry.get(to)
                merged = dict(known or {})
                for r, v in age.items():
                    if r not in merged or v[0] < merged[r][0]:
                        merged[r] = v
                if known is None or {r: a for r, (a, _) in merged.items()} != {r: a for r, (a, _) in known.items()}:
                    entry[to] = merged
                    todo.append(to)
    return sorted(found)


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


def test_the_scan_follows_branches():
    head = "_ZN4bdlm1fEv:\n"
    product = "\tv_mfma_f32_16x16x32_bf16 a[4:7], v[8:11], v[12:15], a[4:7]\n"
    settle, touch = "\ts_nop 15\n\ts_nop 3\n", "\tv_accvgpr_read_b32 v2, a5\n"
    # what follows an unconditional branch in the text does not follow the product
    away = head + product + "\ts_branch .LBB0_2\n.LBB0_1:\n" + touch + "\ts_endpgm\n.LBB0_2:\n"
    assert early_touches(away + settle + touch + "\ts_endpgm\n") == []
    assert len(early_touches(away + touch + "\ts_endpgm\n")) == 1
    # a loop's first instruction follows its last, and a conditional branch goes both ways
    loop = head + ".LBB0_1:\n" + touch + settle + product + "\ts_cbranch_scc1 .LBB0_1\n" + settle + "\ts_endpgm\n"
    assert len(early_touches(loop)) == 1
    assert early_touches(loop.replace(touch, settle + touch)) == []
