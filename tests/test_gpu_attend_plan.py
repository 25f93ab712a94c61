"""GPU: the lists that sp_attend_plan leaves on the device, read back: every row meets every key that it sees in one piece, pieces lie in slots of
their own, the rows to join name all of their pieces; and they are the lists that the walk on the CPU makes."""
import ctypes as C

import numpy as np
import pytest

from tests import attend_batches as ab
from tests import cache_cases as cc
from tests import test_attend_plan as host
from tests.attend_walk import walk, walk_batch  # noqa: F401

pytestmark = pytest.mark.gpu

NO_LIMIT, BAD = 0x7FFFFFFF, -1


def _plan(walk, new, length, groups, H, H_kv, d, fp8, page=8):  # noqa: F811
    """(plan's parts read back, the sizes of its lists)."""
    import torch
    from paper_2502_02789_amd import device as dev
    B, blocks = len(new), max(1, -(-max(length) // page))
    cache = torch.empty((1, 1, 1, d), dtype=torch.uint8 if fp8 else torch.bfloat16, device="cuda").expand(blocks + 3, page, H_kv, d)   # (never read)
    group = {}
    if groups:
        group = dict(cu_group=cc.cuda_ints([g[0] for g in groups] + [groups[-1][1]]), prefix_len=cc.cuda_ints([g[2] for g in groups]))
    p = dev.AttendPlan(cc.cuda_ints(cc.offsets(new)), cc.cuda_ints(length), cache, H=H, total_new=sum(new), block_table=cc.cuda_ints(np.zeros((B, blocks))), **group)
    p.run()
    torch.cuda.synchronize()
    caps = host._caps(walk, p.args)
    raw = p.plan.cpu().numpy()
    head = raw[:24]
    ints = lambda at, n, width: raw[at:at + 4 * n * width].view(np.int32).reshape(n, width)  # noqa: E731
    assert head[:8].view(np.uint64)[0] == walk.print_of(C.byref(p.args))
    n_stretches, n_rows, most = head[8:20].view(np.int32).tolist()
    stretches = ints(caps["at_stretches"], n_stretches, 12)
    n_units = int(stretches[:, 1].max(initial=0))
    assert n_units <= caps["units"] and n_rows <= caps["rows"] and n_stretches <= caps["most_stretches"]
    return stretches, ints(caps["at_units"], n_units, 8), ints(caps["at_rows"], n_rows, 8), most, caps


def _verify(walk, new, length, groups, H, H_kv, d, fp8):  # noqa: F811
    stretches, units, rows, most, caps = _plan(walk, new, length, groups, H, H_kv, d, fp8)
    w = walk_batch(walk, new, length, groups, H, H_kv, d, fp8)
    G, T = H // H_kv, sum(new)
    t0 = np.concatenate([[0], np.cumsum(new)])
    # the walk's pieces
    starts = [t0[lo] for (lo, hi, _), pays in zip(groups, w["sharing"]) if pays] + t0[:-1].tolist()
    first = [lo for (lo, hi, _), pays in zip(groups, w["sharing"]) if pays] + list(range(len(new)))
    assert len(stretches) == w["n_stretches"] and len(units) == len(w["pieces"])
    for u, (b, k0, k1, s) in zip(units, w["pieces"]):
        seg, i, m = int(w["blocks"][b, 0]), int(w["blocks"][b, 1]), int(w["blocks"][b, 5])
        prefix = seg < w["n_prefix"]
        q = seg - w["n_prefix"]
        want = (starts[seg] * G + i * m, w["nr"][b], first[seg], k0, k1, NO_LIMIT if prefix else length[q] - new[q] + 1 - t0[q])
        assert tuple(u[:6]) == want
        assert stretches[s, 0] <= stretches[s, 1] and s < len(stretches)
    # stretches: runs of units, one behind the other, the first unit's copy
    at = 0
    for a, b, _, _, *copy in stretches.tolist():
        if a == b:
            continue
        assert a == at and (units[a] == copy).all()
        at = b
    assert at == len(units)
    # pieces side by side lie in one stretch
    end = np.zeros(len(units), np.int64)
    for a, b in stretches[:, :2]:
        end[a:b] = b
    side = units[:, 7]
    assert (side >= 0).all() and (side <= walk.waves_of(d)).all() and (np.arange(len(units)) + np.maximum(side, 1) <= end).all()
    # every row and key once
    token = np.arange(T * G) // G
    seq = np.repeat(np.arange(len(new)), new)[token] if T else token
    limit = np.clip(np.array(length)[seq] - np.array(new)[seq] + (token - t0[seq]) + 1, 0, np.array(length)[seq]) if T else token
    met, pieces = np.zeros(T * G, np.int64), [[] for _ in range(T * G)]
    used = np.zeros(caps["slots"], bool)
    kept = np.zeros(T * G, bool)
    # (the prefixes' pieces lie in front of all others, a block's in the order of their keys)
    order = np.lexsort((np.arange(len(units)), units[:, 3]))
    for x in order:
        r0, nr, _, k0, k1, off, slot, _ = units[x].tolist()
        r = np.arange(r0, r0 + nr)
        stop = np.minimum(k1, limit[r]) if off != NO_LIMIT else np.full(nr, k1)
        assert (met[r] == np.minimum(k0, limit[r])).all()
        met[r] = np.maximum(met[r], stop)
        if slot < 0:
            kept[r] = True
            continue
        n = -(-nr // 16)
        assert 0 <= slot and slot + n <= caps["slots"] and not used[slot:slot + n].any()
        used[slot:slot + n] = True
        for y in r:
            pieces[y].append((off == NO_LIMIT, 16 * slot + y - r0))
    assert (met == limit).all()
    # rows to join: those whose pieces are in slots, each with all of them; no row has pieces of both kinds
    assert sorted(rows[:, 0].tolist()) == [y for y in range(T * G) if pieces[y]]
    assert not any(kept[y] for y in rows[:, 0])
    for y, own_at, own_n, own_step, pre_at, pre_n, pre_step, _ in rows.tolist():
        assert sorted([own_at + q * own_step for q in range(own_n)]) == sorted(at for prefix, at in pieces[y] if not prefix)
        assert sorted([pre_at + q * pre_step for q in range(pre_n)]) == sorted(at for prefix, at in pieces[y] if prefix)
    assert most == max((r[2] + r[5] for r in rows.tolist()), default=0)


@pytest.mark.parametrize("batch", ab.SHARED + ab.BLOCKS, ids=lambda b: b["name"])
def test_lists_of_batches_that_are_run(walk, batch):  # noqa: F811
    _verify(walk, *ab.shape(batch))


@pytest.mark.parametrize("kind", [(32, 8, 128, 0), (16, 16, 128, 1), (24, 8, 64, 0), (7, 1, 64, 1), (300, 300, 128, 0)])
def test_lists_of_batches_of_all_sorts(walk, kind):  # noqa: F811
    batches = host._batches()
    some = batches[:10] + batches[10::12]
    for new, length, groups in some:
        if sum(new) * kind[0] // kind[1] < 40000 and len(groups) <= len(new):       # (more groups than sequences are refused)
            _verify(walk, new, length, groups, *kind)


@pytest.mark.parametrize("cu_group", [[0, 40], [0, 9, 33, 40], [0, 0, 40], [-7, 40], [-7, -2, 40], [5, 3, 40], [0, 30, 10, 40], [40, 0], [12, 50], [0, 2**31 - 1], [39, 90]])
@pytest.mark.parametrize("prefix", [2000, 2**31 - 1])
def test_no_piece_reaches_beyond_the_table(walk, cu_group, prefix):  # noqa: F811
    """Offsets of groups that do not ascend, or lie outside: what the rows get is not defined, but every piece's keys lie in the room of the sequence whose
    pages it reads, and its rows among the call's."""
    import torch
    from paper_2502_02789_amd import device as dev
    rng, B, page, blocks = np.random.default_rng(8), 40, 16, 200
    new = rng.integers(0, 3, B)
    new[[0, 5, 39]] = 0             # (the sequence whose table is read may have no query, and fewer tokens than the others)
    length = rng.integers(2000, 3200, B)
    length[[0, 5, 39]] = 30
    cache = torch.empty((1, 1, 1, 128), dtype=torch.bfloat16, device="cuda").expand(blocks, page, 2, 128)
    p = dev.AttendPlan(cc.cuda_ints(cc.offsets(new)), cc.cuda_ints(length), cache, H=8, total_new=int(new.sum()) + 3, block_table=cc.cuda_ints(np.zeros((B, blocks))),
                       cu_group=cc.cuda_ints(cu_group), prefix_len=cc.cuda_ints([prefix] * (len(cu_group) - 1)))
    p.run()
    torch.cuda.synchronize()
    raw, caps = p.plan.cpu().numpy(), host._caps(walk, p.args)
    if raw[:8].view(np.uint64)[0] == 0:
        return                      # no plan: NaN everywhere
    n_stretches, n_rows, _ = raw[8:20].view(np.int32).tolist()
    stretches = raw[caps["at_stretches"]:][:48 * n_stretches].view(np.int32).reshape(-1, 12)
    units = raw[caps["at_units"]:][:32 * int(stretches[:, 1].max())].view(np.int32).reshape(-1, 8)
    assert ((0 <= units[:, 2]) & (units[:, 2] < B)).all()
    assert ((0 <= units[:, 3]) & (units[:, 3] <= units[:, 4])).all()
    # (a piece without keys reads none)
    assert ((units[:, 4] <= length[units[:, 2]]) | (units[:, 3] == units[:, 4])).all()
    assert ((0 <= units[:, 0]) & (units[:, 0] + units[:, 1] <= 4 * p.total_new)).all()
    assert ((units[:, 6] == -1) | ((0 <= units[:, 6]) & (units[:, 6] < caps["slots"]))).all()
    rows = raw[caps["at_rows"]:][:32 * n_rows].view(np.int32).reshape(-1, 8)
    assert ((0 <= rows[:, 0]) & (rows[:, 0] < 4 * p.total_new)).all()
    for at, n, step in ((1, 2, 3), (4, 5, 6)):
        assert ((rows[:, n] == 0) | ((rows[:, at] >= 0) & (rows[:, at] + (rows[:, n] - 1) * rows[:, step] < 16 * caps["slots"]))).all()
