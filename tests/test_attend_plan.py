"""How sp_attend cuts a call into pieces (sp_attend_plan.h), walked on the CPU with the functions that the device walks it
with: every row and key is met once, and nothing is written beyond the room that the host side reserved from the shape fields alone."""
import ctypes as C
import os
import random
import shutil
import subprocess

import numpy as np
import pytest

from paper_2502_02789_amd import binding as sp

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SHIM = r"""
#include "sp_attend_plan.h"
#include <algorithm>
#include <vector>
using namespace sp;
extern "C" void caps(const sp_attend_args* a, int64_t* out) {
  const AttendCaps c = attend_caps(a);
  const AttendPlanLayout l = attend_plan_layout(a);
  out[0] = c.blocks; out[1] = c.units; out[2] = c.joins; out[3] = c.slots; out[4] = (int64_t)l.bytes; out[5] = (int64_t)l.units;
  out[6] = (int64_t)l.joins; out[7] = (int64_t)l.seg_start; out[8] = (int64_t)l.seqs; out[9] = (int64_t)l.groups;
  out[10] = sizeof(AttendUnit); out[11] = sizeof(AttendJoin); out[12] = (int64_t)attend_workspace(a); out[13] = (int64_t)attend_sums_bytes(a); out[14] = c.rows; out[15] = sizeof(AttendRow); out[16] = (int64_t)l.rows;
}
extern "C" uint64_t print_of(const sp_attend_args* a) { return attend_print(a); }
extern "C" int share(int64_t rows, int members) { return shares(rows, members); }
// segments: rows, n (0: a prefix), len, shared; blocks out: segment, i, keys, pieces, rows of a block; pieces out: block, first key, end
extern "C" int cut_up(int n_seg, const int64_t* rows, const int* n, const int* len, const int* shared, int G, int H_kv, int* blocks, int* pieces, int* n_pieces) {
  int64_t total = 0;
  int nb = 0;
  for (int pass = 0; pass < 2; ++pass) {
    const int cut = make_cut(total, H_kv);
    nb = 0; *n_pieces = 0;
    for (int s = 0; s < n_seg; ++s)
      for (int i = 0; rows[s] > 0 && i < segment_blocks(rows[s]); ++i, ++nb) {
        const int keys = n[s] ? own_block_keys(rows[s], i, G, n[s], len[s], shared[s]) : shared[s];
        if (pass == 0) { total += keys; continue; }
        const int p = pieces_of(keys, cut);
        int* b = blocks + 5 * nb;
        b[0] = s; b[1] = i; b[2] = keys; b[3] = p; b[4] = block_rows(rows[s]);
        for (int q = 0; q < p; ++q, ++*n_pieces) {
          int* x = pieces + 3 * *n_pieces;
          x[0] = nb; x[1] = piece_start(shared[s] * (n[s] != 0), keys, p, q); x[2] = piece_start(shared[s] * (n[s] != 0), keys, p, q + 1);
        }
      }
  }
  return nb;
}
"""


@pytest.fixture(scope="module")
def shim(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("c++") or shutil.which("clang++") or "/opt/rocm/llvm/bin/clang++"
    where = tmp_path_factory.mktemp("plan")
    (where / "shim.cpp").write_text(SHIM)
    subprocess.run([cxx, "-std=c++17", "-O1", "-Wall", "-shared", "-fPIC", "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2502_02789_amd", "csrc"), "shim.cpp", "-o", "shim.so"], cwd=where, check=True)
    lib = C.CDLL(str(where / "shim.so"))
    lib.print_of.restype = C.c_uint64
    lib.share.argtypes = [C.c_int64, C.c_int]
    return lib


def _args(**kw):
    a = sp.AttendArgs()
    for k, v in dict(dict(B=1, H=32, H_kv=8, d=128, T_new=1, n_groups=0, n_rows=4096, page_size=16, blocks_per_seq=64, d_block_table=64), **kw).items():
        setattr(a, k, v)
    return a


def _caps(shim, a):
    out = (C.c_int64 * 17)()
    shim.caps(C.byref(a), out)
    return dict(zip("blocks units joins slots bytes at_units at_joins at_seg at_seqs at_groups unit join workspace sums rows row at_rows".split(), out))


def _batches():
    rng = random.Random(11)
    fixed = [([1], [1], []), ([1], [131072], []), ([0, 0, 1], [0, 5, 9], []), ([5000], [5000], []), ([3] * 64, [900] * 64, [(0, 64, 700)]),
             ([1] * 64, [33000] * 64, [(0, 64, 32768)]), ([1] * 16, [40] * 16, [(0, 16, 39)]), ([200, 1, 0, 7], [300, 300, 300, 300], [(0, 4, 100)]),
             ([40, 40, 40], [50, 0, 10], [(0, 3, 10)]), ([1, 300, 2, 1], [20000, 300, 7, 131072], [])]
    for _ in range(300):
        B = rng.randint(1, 40)
        new = [rng.choice([0, 1, 1, 1, 2, 4, 5, 17, rng.randint(0, 700)]) for _ in range(B)]
        length = [max(0, n + rng.choice([-3, 0, 0, rng.randint(0, 100), rng.randint(0, 30000)])) for n in new]
        groups, b = [], 0
        while rng.random() < 0.7 and b < B:
            e = rng.randint(b, B)
            groups.append((b, e, rng.choice([0, 1, 63, 64, 1000, rng.randint(0, 20000)])))
            b = e
        fixed.append((new, length, groups if groups and groups[0][0] == 0 else []))
    return fixed


@pytest.mark.parametrize("heads", [(32, 8), (8, 8), (128, 8), (24, 8), (7, 1), (1024, 1024)])
def test_pieces_cover_every_block_within_the_reserved_room(shim, heads):
    H, H_kv = heads
    G = H // H_kv
    for new, length, groups in _batches():
        B = len(new)
        shared = [0] * B
        segs = []
        for lo, hi, prefix in groups:
            live = [b for b in range(lo, hi) if new[b] > 0]
            p = min([prefix] + [max(0, length[b] - new[b]) for b in live] + ([length[lo]] if hi > lo else []))
            rows = sum(new[lo:hi]) * G
            p = p if shim.share(rows, len(live)) else 0
            if p > 0:
                for b in range(lo, hi):
                    shared[b] = p
                segs.append((rows, 0, 0, p))
        n_prefix = len(segs)
        segs += [(n * G, n, m, s) for n, m, s in zip(new, length, shared)]
        arr = lambda i, t: np.array([s[i] for s in segs], dtype=t)  # noqa: E731
        rows, n, ln, sh = arr(0, np.int64), arr(1, np.int32), arr(2, np.int32), arr(3, np.int32)
        blocks, pieces = np.zeros(5 * 40000, np.int32), np.zeros(3 * 40000, np.int32)
        n_pieces = C.c_int()
        ptr = lambda x: x.ctypes.data_as(C.c_void_p)  # noqa: E731
        nb = shim.cut_up(len(segs), ptr(rows), ptr(n), ptr(ln), ptr(sh), G, H_kv, ptr(blocks), ptr(pieces), C.byref(n_pieces))
        blocks, pieces = blocks[:5 * nb].reshape(-1, 5), pieces[:3 * n_pieces.value].reshape(-1, 3)
        caps = _caps(shim, _args(B=B, H=H, H_kv=H_kv, T_new=sum(new), n_groups=len(groups)))
        # the keys of a block, in order and without gaps; whole steps of 64 apart from the end
        for i, (s, k, keys, p, m) in enumerate(blocks):
            mine = pieces[pieces[:, 0] == i]
            first_key = sh[s] if n[s] else 0
            assert len(mine) == p and mine[0, 1] == first_key and mine[-1, 2] == first_key + keys
            assert (mine[1:, 1] == mine[:-1, 2]).all() and (mine[1:, 1] % 64 == 0).all()
            assert p == 1 or (mine[:, 2] > mine[:, 1]).all()
            if n[s]:   # no row of the block sees a key beyond the last row's
                last = min((k + 1) * m, rows[s]) - 1
                want = min(ln[s], max(0, ln[s] - n[s] + last // G + 1)) - sh[s]
                assert keys == max(0, want)
                first = ln[s] - n[s] + (k * m) // G + 1
                assert sh[s] == 0 or first > sh[s]    # every row sees the whole prefix and a key behind it
        # room
        leaves = [bool(p > 1 or s < n_prefix or sh[s] > 0) for s, _, _, p, _ in blocks]
        assert nb <= caps["blocks"] and len(pieces) <= caps["units"]
        assert sum(1 for x, b in zip(leaves, blocks) if x and b[0] >= n_prefix) <= caps["joins"]
        slots = sum(int(b[3]) * int(b[4]) // 16 for x, b in zip(leaves, blocks) if x)
        assert slots <= caps["slots"], (new, length, groups)
        assert caps["at_units"] + caps["units"] * caps["unit"] <= caps["at_joins"]
        assert caps["at_joins"] + caps["joins"] * caps["join"] <= caps["at_rows"]
        assert sum(min(int(b[4]), int(rows[b[0]] - b[1] * b[4])) for x, b in zip(leaves, blocks) if x and b[0] >= n_prefix) <= caps["rows"]
        assert caps["at_rows"] + caps["rows"] * caps["row"] <= caps["at_seg"]
        assert caps["at_seg"] + 4 * (B + len(groups) + 1) <= caps["at_seqs"] and caps["at_seqs"] + 16 * B <= caps["at_groups"]
        assert caps["at_groups"] + 32 * len(groups) <= caps["bytes"]
        assert caps["sums"] >= caps["slots"] * H_kv * 16 * 128 * 4 and caps["workspace"] >= caps["sums"] + caps["slots"] * H_kv * 16 * 8


def test_equal_work_is_spread_over_the_device(shim):
    """One long sequence: about a thousand workgroups of equal pieces; short ones: pieces of 128 keys; many blocks: no cuts."""
    def pieces_of(rows, n, ln):
        arrays = [np.array([rows], np.int64), np.array([n], np.int32), np.array([ln], np.int32), np.zeros(1, np.int32)]
        blocks, pieces, count = np.zeros(5 * 4000, np.int32), np.zeros(3 * 8000, np.int32), C.c_int()
        shim.cut_up(1, *[x.ctypes.data_as(C.c_void_p) for x in arrays], 4, 8, blocks.ctypes.data_as(C.c_void_p), pieces.ctypes.data_as(C.c_void_p), C.byref(count))
        p = pieces[:3 * count.value].reshape(-1, 3)
        return p[:, 2] - p[:, 1]
    long = pieces_of(4, 1, 131072)
    assert 100 <= len(long) <= 128 and long.max() <= 1.1 * long.mean() + 64
    assert pieces_of(4, 1, 1000).max() <= 128
    assert len(pieces_of(4 * 20000, 20000, 20000)) == 4 * 20000 // 128


def test_a_plan_knows_the_shape_it_was_made_for(shim):
    base = _args()
    seen = {shim.print_of(C.byref(base))}
    for k, v in dict(B=2, H=16, H_kv=4, d=64, T_new=2, n_groups=1, page_size=32, blocks_per_seq=65, n_rows=4112, cache_dtype=1, d_block_table=None).items():
        p = shim.print_of(C.byref(_args(**{k: v})))
        assert p != 0 and p not in seen, k
        seen.add(p)
    a = _args(d_q=7, d_kv_len=9, scale=0.5, cache_token_stride=1)
    assert shim.print_of(C.byref(a)) == shim.print_of(C.byref(base))
