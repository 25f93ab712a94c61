"""The workgroups of sp_cache_append, cut as sp_append_grid.h does it, walked on the CPU: every call that is taken can be launched."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

from paper_2502_02789_amd import binding as sp
from tests.test_cache_args import ROOT

SHIM = r"""
#include "sp_append_grid.h"
extern "C" void grid_of(int64_t T, int rows, int d, int dtype, int64_t* out) {
  const sp::AppendGrid g = sp::append_grid(T, rows, d, dtype);
  out[0] = g.tokens; out[1] = g.blocks; out[2] = g.parts;
}
extern "C" int64_t most_tokens() { return sp::kMostTokens; }
"""
KINDS = (sp.SP_K_BF16, sp.SP_K_FP8_E4M3, sp.SP_K_MXFP4)


@pytest.fixture(scope="module")
def shim(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("c++") or shutil.which("clang++") or "/opt/rocm/llvm/bin/clang++"
    where = tmp_path_factory.mktemp("grid")
    (where / "shim.cpp").write_text(SHIM)
    subprocess.run([cxx, "-std=c++17", "-O1", "-Wall", "-shared", "-fPIC", "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2502_02789_amd", "csrc"), "shim.cpp", "-o", "shim.so"], cwd=where, check=True)
    lib = C.CDLL(str(where / "shim.so"))
    lib.grid_of.argtypes = [C.c_int64, C.c_int, C.c_int, C.c_int, C.c_void_p]
    lib.most_tokens.restype = C.c_int64
    return lib


def _grid(shim, T, rows, d, dtype):
    out = (C.c_int64 * 3)()
    shim.grid_of(T, rows, d, dtype, out)
    return tuple(out)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", KINDS)
def test_every_call_fits_a_launch(shim, dtype, d):
    """Fewer than 2^32 threads, at most 65535 parts, a workgroup for every token, and no more tokens to one than its tables hold."""
    assert shim.most_tokens() == 1 << 25
    sizes = [1, 2, 511, 512, 513, 1024, 6592, 100000, (1 << 23) + 1, (1 << 24) - 1, 1 << 24, (1 << 24) + 1, (1 << 25) - 2, (1 << 25) - 1, 1 << 25]
    for T in sizes:
        for rows in (2, 3, 12, 48, 49, 50, 80, 96, 98, 128, 192, 193, 300, 1000, 3000):
            tokens, blocks, parts = _grid(shim, T, rows, d, dtype)
            assert 1 <= tokens <= 4 and (blocks - 1) * tokens < T <= blocks * tokens, (T, rows)
            assert blocks * parts * 256 < 1 << 32 and 1 <= parts <= 512, (T, rows)


def test_ordinary_calls_are_cut_as_measured(shim):
    for T, rows, d, want in ((6592, 80, 128, (1, 6592, 1)), (8192, 10, 128, (4, 2048, 1)), (8192, 48, 128, (2, 4096, 1)), (100000, 48, 64, (4, 25000, 1)),
                             (1, 48, 128, (1, 1, 2)), (100, 80, 128, (1, 100, 3))):
        assert _grid(shim, T, rows, d, sp.SP_K_MXFP4) == want
    for dtype in KINDS[:2]:
        assert _grid(shim, 6592, 80, 128, dtype) == (4, 1648, 1) and _grid(shim, 1000, 48, 128, dtype) == (1, 1000, 1)
