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
#include <utility>
#include <vector>
using namespace sp;
extern "C" void caps(const sp_attend_args* a, int64_t* out) {
  const AttendCaps c = attend_caps(a);
  const AttendPlanLayout l = attend_plan_layout(a);
  out[0] = c.blocks; out[1] = c.units; out[2] = c.joins; out[3] = c.slots; out[4] = (int64_t)l.bytes; out[5] = (int64_t)l.units;
  out[6] = (int64_t)l.joins; out[7] = (int64_t)l.seg_start; out[8] = (int64_t)l.seqs; out[9] = (int64_t)l.groups;
  out[10] = sizeof(AttendUnit); out[11] = sizeof(AttendJoin); out[12] = (int64_t)attend_workspace(a); out[13] = (int64_t)attend_sums_bytes(a); out[14] = c.rows; out[15] = sizeof(AttendRow); out[16] = (int64_t)l.rows; out[17] = (int64_t)l.stretches; out[18] = sizeof(AttendStretch); out[19] = most_stretches(a);
}
extern "C" uint64_t print_of(const sp_attend_args* a) { return attend_print(a); }
extern "C" int by_stretches_of(int64_t blocks, int64_t many, int d, int H_kv) { return by_stretches(blocks, many, d, H_kv); }
extern "C" int share(int rows, int members) { return shares(rows, members); }
// segments (prefixes first): rows, n (0: a prefix), len, shared.  blocks out, in the order that they are laid out in: segment, i,
// first key, keys, pieces, rows of a block, cost of a step, steps; pieces out: block, first key, end, stretch.  Returns the number of blocks.
extern "C" int cut_up(int n_seg, const int* rows, const int* n, const int* len, const int* shared, int G, int H_kv, int d, int fp8, int* blocks,
                      int* pieces, int* n_pieces, int* n_stretches) {
  int nb = 0;
  int64_t keys_all = 0, cost_all = 0, many = 0;
  std::vector<int64_t> start;
  auto add = [&](int s, int i) {
    int* b = blocks + 9 * nb++;
    b[0] = s; b[1] = i; b[2] = n[s] ? shared[s] : 0;
    b[3] = n[s] ? own_block_keys(rows[s], i, block_rows(rows[s], d), G, n[s], len[s], shared[s]) : shared[s];
    b[4] = 0; b[5] = block_rows(rows[s], d); b[6] = step_cost(std::min(b[5], rows[s] - i * b[5]), d, fp8); b[7] = block_steps(b[2], b[3]);
    const int nr = std::min(b[5], rows[s] - i * b[5]);
    b[8] = piece_cost(nr, b[3], d);
    many += nr > kFewRows;
    start.push_back(cost_all);
    keys_all += b[3]; cost_all += (int64_t)b[7] * b[6] + b[8];
  };
  for (int s = 0; s < n_seg; ++s) if (!n[s]) for (int i = 0; rows[s] > 0 && i < segment_blocks(rows[s], d); ++i) add(s, i);
  for (int s = n_seg - 1; s >= 0; --s) if (n[s]) for (int i = segment_blocks(rows[s], d) - 1; i >= 0; --i) add(s, i);
  *n_pieces = 0;
  auto piece = [&](int b, int k0, int k1, int s) { int* x = pieces + 4 * (*n_pieces)++; x[0] = b; x[1] = k0; x[2] = k1; x[3] = s; ++blocks[9 * b + 4]; };
  if (!by_stretches(nb, many, d, H_kv)) {
    const int cut = make_cut(keys_all, d, H_kv);
    for (int b = 0; b < nb; ++b) {
      const int* k = blocks + 9 * b;
      const int p = pieces_of(k[3], cut);
      for (int q = 0; q < p; ++q) piece(b, piece_start(k[2], k[3], p, q), piece_start(k[2], k[3], p, q + 1), *n_pieces);
    }
    *n_stretches = *n_pieces;
    return nb;
  }
  const int ns = stretch_count(cost_all, d, H_kv);
  *n_stretches = ns;
  std::vector<std::pair<int, int>> cuts;
  for (int s = 0; s <= ns; ++s) {
    if (s == 0 || s == ns) { cuts.push_back({s == 0 ? 0 : nb, 0}); continue; }
    const int64_t x = stretch_start(cost_all, ns, s);
    int b = (int)(std::upper_bound(start.begin(), start.end(), x) - start.begin()) - 1;
    int j = step_at(x, start[b], blocks[9 * b + 7], blocks[9 * b + 6], blocks[9 * b + 8]);
    if (j > 0 && j >= blocks[9 * b + 7]) { ++b; j = 0; }
    cuts.push_back({b, j});
  }
  for (int s = 0; s < ns; ++s)
    for (int b = cuts[s].first; b < cuts[s + 1].first + (cuts[s + 1].second > 0); ++b) {
      const int* k = blocks + 9 * b;
      const int j0 = b == cuts[s].first ? cuts[s].second : 0, j1 = b == cuts[s + 1].first ? cuts[s + 1].second : k[7];
      piece(b, step_key(k[2], k[3], k[7], j0), step_key(k[2], k[3], k[7], j1), s);
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
    lib.share.argtypes = [C.c_int, C.c_int]
    lib.by_stretches_of.argtypes = [C.c_int64, C.c_int64, C.c_int, C.c_int]
    return lib


def _args(**kw):
    a = sp.AttendArgs()
    for k, v in dict(dict(B=1, H=32, H_kv=8, d=128, T_new=1, n_groups=0, n_rows=4096, page_size=16, blocks_per_seq=64, d_block_table=64), **kw).items():
        setattr(a, k, v)
    return a


def _caps(shim, a):
    out = (C.c_int64 * 20)()
    shim.caps(C.byref(a), out)
    return dict(zip("blocks units joins slots bytes at_units at_joins at_seg at_seqs at_groups unit join workspace sums rows row at_rows at_stretches stretch most_stretches".split(), out))


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


def _cut(shim, segs, G, H_kv, d=128, fp8=0):
    arr = lambda i, t: np.array([s[i] for s in segs], dtype=t)  # noqa: E731
    arrays = [arr(0, np.int32), arr(1, np.int32), arr(2, np.int32), arr(3, np.int32)]
    blocks, pieces = np.zeros(9 * 80000, np.int32), np.zeros(4 * 80000, np.int32)
    n_pieces, n_stretches = C.c_int(), C.c_int()
    ptr = lambda x: x.ctypes.data_as(C.c_void_p)  # noqa: E731
    nb = shim.cut_up(len(segs), *[ptr(x) for x in arrays], G, H_kv, d, fp8, ptr(blocks), ptr(pieces), C.byref(n_pieces), C.byref(n_stretches))
    return blocks[:9 * nb].reshape(-1, 9), pieces[:4 * n_pieces.value].reshape(-1, 4), n_stretches.value


@pytest.mark.parametrize("heads", [(32, 8), (8, 8), (128, 8), (24, 8), (7, 1), (1024, 1024), (64, 2)])
@pytest.mark.parametrize("kind", [(128, 0), (128, 1), (64, 0)])
def test_pieces_cover_every_block_within_the_reserved_room(shim, heads, kind):
    H, H_kv = heads
    G, (d, fp8) = H // H_kv, kind
    many = 128 if d == 64 else 256
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
        rows, n, ln, sh = ([s[i] for s in segs] for i in range(4))
        blocks, pieces, n_stretches = _cut(shim, segs, G, H_kv, d, fp8)
        caps = _caps(shim, _args(B=B, H=H, H_kv=H_kv, d=d, T_new=sum(new), n_groups=len(groups), cache_dtype=fp8, page_size=8, blocks_per_seq=-(-max(length) // 8)))
        # the keys of a block, in order and without gaps; whole steps of 64 of the sequence apart from the ends
        for i, (s, k, first_key, keys, p, m, cost, steps, extra) in enumerate(blocks):
            mine = pieces[pieces[:, 0] == i]
            assert len(mine) == p and mine[0, 1] == first_key and mine[-1, 2] == first_key + keys
            assert (mine[1:, 1] == mine[:-1, 2]).all() and (mine[1:, 1] % 64 == 0).all()
            assert p == 1 or (mine[:, 2] > mine[:, 1]).all()
            if n[s]:   # no row of the block sees a key beyond the last row's
                last = min((k + 1) * m, rows[s]) - 1
                want = min(ln[s], max(0, ln[s] - n[s] + last // G + 1)) - sh[s]
                assert keys == max(0, want)
                first = ln[s] - n[s] + (k * m) // G + 1
                assert sh[s] == 0 or first > sh[s]    # every row sees the whole prefix and a key behind it
        assert sorted(set(zip(blocks[:, 0], blocks[:, 1]))) == sorted((s, i) for s in range(len(segs)) for i in range(-(-rows[s] // (16 if rows[s] <= 16 else many))))
        # every stretch is a run of pieces; none has much more than its share
        assert (np.diff(pieces[:, 3]) >= 0).all() and (len(pieces) == 0 or pieces[-1, 3] < n_stretches)
        large = sum(min(int(b[5]), int(rows[b[0]] - b[1] * b[5])) > 16 for b in blocks)
        if shim.by_stretches_of(len(blocks), large, d, H_kv) and len(pieces):
            cost = [int(blocks[x[0], 8]) + -(-(int(x[2]) - (int(x[1]) & ~63)) // 64) * int(blocks[x[0], 6]) for x in pieces]
            per = np.bincount(pieces[:, 3], weights=cost, minlength=n_stretches)
            share = (blocks[:, 7] * blocks[:, 6] + blocks[:, 8]).sum() / n_stretches
            assert per.max() <= share + 2 * 12 + 4 * 8 + 1     # a snapped end on either side, a cut block's cost again
        # room
        leaves = [bool(b[4] > 1 or b[0] < n_prefix or sh[b[0]] > 0) for b in blocks]
        assert len(blocks) <= caps["blocks"] and len(pieces) <= caps["units"] and n_stretches <= max(caps["units"], 1)
        assert n_stretches <= max(caps["most_stretches"], 1) and caps["most_stretches"] <= max(caps["units"], 1)
        assert sum(1 for x, b in zip(leaves, blocks) if x and b[0] >= n_prefix) <= caps["joins"]
        slots = sum(int(b[4]) * int(b[5]) // 16 for x, b in zip(leaves, blocks) if x)
        assert slots <= caps["slots"], (new, length, groups)
        assert caps["at_units"] + caps["units"] * caps["unit"] <= caps["at_stretches"]
        assert caps["at_stretches"] + caps["stretch"] * caps["units"] <= caps["at_joins"]
        assert caps["at_joins"] + caps["joins"] * caps["join"] <= caps["at_rows"]
        assert sum(min(int(b[5]), int(rows[b[0]] - b[1] * b[5])) for x, b in zip(leaves, blocks) if x and b[0] >= n_prefix) <= caps["rows"]
        assert caps["at_rows"] + caps["rows"] * caps["row"] <= caps["at_seg"]
        assert caps["at_seg"] + 4 * (B + len(groups) + 1) <= caps["at_seqs"] and caps["at_seqs"] + 16 * B <= caps["at_groups"]
        assert caps["at_groups"] + 32 * len(groups) <= caps["bytes"]
        assert caps["sums"] >= caps["slots"] * H_kv * 16 * d * 4 and caps["workspace"] >= caps["sums"] + caps["slots"] * H_kv * 16 * 8


def test_equal_work_is_spread_over_the_device(shim):
    """One long sequence: 32 stretches for each of 8 KV heads; a short one: pieces of two or three steps; many blocks: no cuts."""
    blocks, pieces, n = _cut(shim, [(4, 1, 131072, 0)], 4, 8)
    size = pieces[:, 2] - pieces[:, 1]
    assert n == len(pieces) == 32 and size.max() <= 1.1 * size.mean() + 64
    assert (lambda p: (p[:, 2] - p[:, 1]).max())(_cut(shim, [(4, 1, 1000, 0)], 4, 8)[1]) <= 192
    blocks, pieces, n = _cut(shim, [(4 * 20000, 20000, 20000, 0)], 4, 8)
    assert n == len(pieces) == len(blocks) == -(-4 * 20000 // 256)
    assert (np.diff(pieces[:, 2]) <= 0).all()          # the longest first
    blocks, pieces, n = _cut(shim, [(4, 1, 1000 + 37 * i, 0) for i in range(64)], 4, 8)
    assert n == 32 and len(pieces) <= 64 + 31


def test_a_plan_knows_the_shape_it_was_made_for(shim):
    base = _args()
    seen = {shim.print_of(C.byref(base))}
    for k, v in dict(B=2, H=16, H_kv=4, d=64, T_new=2, n_groups=1, page_size=32, blocks_per_seq=65, n_rows=4112, cache_dtype=1, d_block_table=None).items():
        p = shim.print_of(C.byref(_args(**{k: v})))
        assert p != 0 and p not in seen, k
        seen.add(p)
    a = _args(d_q=7, d_kv_len=9, scale=0.5, cache_token_stride=1)
    assert shim.print_of(C.byref(a)) == shim.print_of(C.byref(base))
