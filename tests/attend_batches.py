"""Batches of sp_attend by the way that they take through its plan: groups that share their prefix, blocks laid end to end or a workgroup each.
A test on the CPU holds them to that way, tests on the GPU run them."""
import numpy as np


def _batch(name, new, own, H, H_kv, d, *, groups=(), sharing=(), bits=16, page=16, **kw):
    """own: keys of a sequence behind what its group shares; groups: (first, end, tokens shared); sharing: which of them are read once."""
    length = [o + next((p for lo, hi, p in groups if lo <= b < hi), 0) for b, o in enumerate(own)]
    return dict(name=name, new=[int(n) for n in new], length=[int(m) for m in length], groups=tuple(groups), sharing=list(sharing), H=H, H_kv=H_kv, d=d,
                bits=bits, page=page, **kw)


def shape(b):
    return b["new"], b["length"], b["groups"], b["H"], b["H_kv"], b["d"], b["bits"] == 8


def _ints(seed, lo, hi, n):
    return np.random.default_rng(seed).integers(lo, hi + 1, n).tolist()


def _some(seed, lo, hi, new, least=0):
    """Keys of each sequence: its new ones and lo .. hi more."""
    return [max(n, least) + x for n, x in zip(new, _ints(seed, lo, hi, len(new)))]


def _shared():
    out = []
    for bits, d, page in ((16, 128, 16), (8, 128, 64), (16, 64, 8), (8, 64, 16)):
        at = f"{bits} bits d {d}"
        kw = dict(d=d, bits=bits, page=page)
        out += [
            _batch(f"prefix of 12 rows, {at}", [1] * 4, [3, 90, 17, 1], 3, 1, groups=[(0, 4, 1333)], sharing=[True], **kw),
            _batch(f"prefix of 32 rows, {at}", [1] * 8, _ints(1, 1, 200, 8), 4, 1, groups=[(0, 8, 1333)], sharing=[True], **kw),
            _batch(f"prefix of 192 rows, {at}", [1, 2, 3] * 8, _some(2, 0, 300, [1, 2, 3] * 8), 8, 2, groups=[(0, 24, 2111)], sharing=[True], **kw),
            _batch(f"prefix of 320 rows, {at}", [2] * 40, _some(3, 0, 90, [2] * 40), 8, 2, groups=[(0, 40, 2047)], sharing=[True], **kw),
            _batch(f"members of two tiles, {at}", [5, 6, 7, 8] * 3, _some(4, 0, 130, [5, 6, 7, 8] * 3), 8, 2, groups=[(0, 12, 4100)], sharing=[True], **kw),
            _batch(f"members of a large block, {at}", [10, 12] * 6, _some(5, 0, 500, [10, 12] * 6), 4, 1, groups=[(0, 12, 9001)], sharing=[True], **kw),
            # one group behind the other, with members of no token, a group of one, one that is too short to be read once
            _batch(f"five groups, {at}", [1, 0, 2, 1, 3, 1, 0, 1, 1, 1, 1, 2, 1, 1, 0, 1, 1], [9, 4, 70, 1, 33, 5, 8, 64, 65, 2, 128, 2, 7, 31, 3, 1, 250], 8, 2,
                   groups=[(0, 6, 1500), (6, 8, 99), (8, 9, 400), (9, 12, 20), (12, 17, 1811)], sharing=[True, False, False, False, True], **kw),
        ]
    new = _ints(6, 0, 3, 700)
    groups = [(7 * i, 7 * i + 7, 390 + i) for i in range(100)]
    out.append(_batch("more sequences than the plan keeps in LDS", new, _some(7, 0, 20, new, 1), 2, 1, 64, groups=groups, sharing=[True] * 100, page=8))
    return out


SHARED = _shared()
BLOCKS = []
