"""The cut of an attention call as sp_attend_plan.h makes it, walked on the CPU: which form a batch takes, which of its groups share their
prefix, which blocks are cut."""
import ctypes as C
import os
import shutil
import subprocess

import numpy as np
import pytest

from tests import test_attend_plan as plan

MORE = r"""
extern "C" int pays(int rows, int members, int prefix, int d, int fp8) { return prefix_pays(rows, members, prefix, d, fp8 != 0); }
extern "C" int few_rows() { return kFewRows; }
extern "C" int waves_of(int d) { return attend_waves(d); }
"""


def build(where):
    cxx = shutil.which("g++") or shutil.which("c++") or shutil.which("clang++") or "/opt/rocm/llvm/bin/clang++"
    (where / "walk.cpp").write_text(plan.SHIM + MORE)
    subprocess.run([cxx, "-std=c++17", "-O1", "-Wall", "-shared", "-fPIC", "-I", os.path.join(plan.ROOT, "include"),
                    "-I", os.path.join(plan.ROOT, "paper_2502_02789_amd", "csrc"), "walk.cpp", "-o", "walk.so"], cwd=where, check=True)
    lib = C.CDLL(str(where / "walk.so"))
    lib.by_stretches_of.argtypes = [C.c_int64, C.c_int64, C.c_int, C.c_int]
    lib.print_of.restype = C.c_uint64
    return lib


@pytest.fixture(scope="session")
def walk(tmp_path_factory):
    return build(tmp_path_factory.mktemp("walk"))


def walk_batch(lib, new, length, groups, H, H_kv, d, fp8):
    """blocks and pieces as test_attend_plan has them, with what the batch comes to."""
    G, B = H // H_kv, len(new)
    shared, segs, sharing = [0] * B, [], []
    for lo, hi, prefix in groups:
        live = [b for b in range(lo, hi) if new[b] > 0]
        p = min([prefix] + [max(0, length[b] - new[b]) for b in live] + ([length[lo]] if hi > lo else []))
        rows = sum(new[lo:hi]) * G
        pays = bool(lib.pays(rows, len(live), p, d, int(fp8)))
        sharing.append(pays)
        if pays:
            segs.append((rows, 0, 0, p))
            shared[lo:hi] = [p] * (hi - lo)
    n_prefix = len(segs)
    segs += [(n * G, n, m, s) for n, m, s in zip(new, length, shared)]
    blocks, pieces, n_stretches = plan._cut(lib, segs, G, H_kv, d, int(fp8))
    rows = np.array([s[0] for s in segs])
    nr = np.minimum(blocks[:, 5], rows[blocks[:, 0]] - blocks[:, 1] * blocks[:, 5])
    large = nr > lib.few_rows()
    return dict(segs=segs, n_prefix=n_prefix, sharing=sharing, shared=shared, blocks=blocks, pieces=pieces, n_stretches=n_stretches, nr=nr, large=large,
                stretched=bool(lib.by_stretches_of(len(blocks), int(large.sum()), d, H_kv)))
