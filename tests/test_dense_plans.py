"""The plans of the dense operators, asked on the CPU of the entry points' own source: tiles, splits, pieces of the
vocabulary, and what fits a launch."""
import ctypes
import os
import subprocess

import pytest

import paper_2607_02805_amd as bd

SHIM = r"""
#include "bdlm_dense_api.cpp"
extern "C" int fits(int64_t tiles) { return launch_fits(tiles); }
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    bd.lib()
    d = tmp_path_factory.mktemp("plans")
    src, so = d / "shim.cpp", d / "shim.so"
    src.write_text(SHIM)
    package = os.path.dirname(bd.LIB_PATH)
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", f"-I{os.path.join(package, 'csrc')}",
                    f"-I{os.path.dirname(bd.HEADER_PATH)}", str(src), "-o", str(so), f"-L{package}", "-l:libbdlm.so",
                    f"-Wl,-rpath,{package}"], check=True)
    return ctypes.CDLL(str(so))


def test_a_launch_holds_fewer_than_2_to_the_32_threads(plans):
    """Workgroups of large and of small tiles have 512 threads."""
    for tiles in (1, 1 << 22, (1 << 23) - 1):
        assert plans.fits(ctypes.c_int64(tiles))
    for tiles in (1 << 23, (1 << 24) - 1, 1 << 24, 1 << 40):
        assert not plans.fits(ctypes.c_int64(tiles))
