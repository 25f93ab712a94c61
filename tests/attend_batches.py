"""Batches of sp_attend by the way that they take through its plan: groups that share their prefix, blocks laid end to end or a workgroup each.
A test on the CPU holds them to that way, tests on the GPU run them."""
import numpy as np


def _batch(name, new, own, H, H_kv, d, *, groups=(), sharing=(), bits=16, page=16, **kw):
    """own: keys of a sequence behind what its group shares; groups: (first, end, tokens shared); sharing: which of them are read once."""
    length = [o + next((p for lo, hi, p in groups if lo <= b < hi), 0) for b, o in enumerate(own)]
    return dict(name=name, new=[int(n) for n in new], length=[int(m) for m in length], groups=tuple(groups), sharing=list(sharing or ()), H=H, H_kv=H_kv, d=d,
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


def _blocks():
    """So many large blocks that a workgroup takes one at a time: 768 (d = 128) or 2304 (d = 64) and more of them, KV heads counted.  cut: of a sequence's
    large blocks some are longer than a workgroup's share and cut, cut_prefix: of a group's."""
    out = []
    for H, H_kv, d, n, page, bits in ((16, 16, 128, 50, 8, 16), (16, 16, 128, 50, 16, 8), (32, 8, 128, 100, 16, 16), (64, 64, 64, 40, 8, 16), (64, 16, 64, 150, 16, 8)):
        G = H // H_kv
        at = f"H {H}, {H_kv} of d {d}, {bits} bits"
        kw = dict(d=d, bits=bits, page=page)
        new = _ints(41, 32 // G + 1, 40 // G + 2, n)
        own = _some(42, 0, 30, new)
        # large blocks, small ones between them, sequences of none; a block that is cut, several blocks of which the last are
        few = [1, 0, 2, 1, 16 // G, 32 // G, 3, 1]
        new2 = new[:20] + few + new[20:] + [60, 300 // G + 5]
        own2 = own[:20] + [5, 9, 700, 1, 40, 300, 3, 2500] + own[20:] + [1500, 2000 + 300 // G]
        out.append(_batch(f"blocks that are cut, {at}", new2, own2, H, H_kv, cut=True, cut_prefix=False, **kw))
        # groups: a prefix of single tokens that is cut, one of large blocks, one that each member reads; then sequences without a group
        m = 40 // G + 1
        new3 = [1] * m + [34 // G + 1] * 6 + [1, 0, 2] + new
        own3 = _some(43, 0, 60, new3)
        groups = [(0, m, 1801), (m, m + 6, 2600), (m + 6, m + 9, 30)] + [(b, b + 1, 0) for b in range(m + 9, len(new3))]
        out.append(_batch(f"prefixes that are cut, {at}", new3, own3, H, H_kv, groups=groups, sharing=[True, True, False] + [False] * (len(new3) - m - 9), cut=False,
                          cut_prefix=True, **kw))
    for d, n, bits in ((128, 3000, 16), (64, 4600, 16), (128, 2900, 8)):
        out.append(_batch(f"a whole prompt of {n} tokens, d {d}, {bits} bits", [n], [n], 64, 64, d, bits=bits, page=0, cut=False, cut_prefix=False))
    return out


def drawn(seed):
    """A batch of any kind: heads, pages and lengths over the whole ranges; some sequences of no token, or with more new tokens than keys."""
    r = np.random.default_rng(seed)
    H, H_kv = [(8, 2), (5, 5), (12, 1), (16, 1), (24, 2), (14, 2), (1, 1), (32, 8)][r.integers(8)]
    d, bits, page = [64, 128][r.integers(2)], [16, 8][r.integers(2)], [0, 8, 16, 64, 1024][r.integers(5)]
    B = int(np.exp(r.uniform(0, np.log(60))))
    most = int(np.exp(r.uniform(0, np.log(max(2, 900 // B)))))
    new = [int(n) for n in r.integers(0 if most > 1 else 1, most + 1, B)]
    new[0] = max(new[0], 1)
    far = int(np.exp(r.uniform(0, np.log(min(20000, 60000 // B)))))
    own = [max(0, n + int(r.integers(-3 if far > 3 else 0, far + 1))) for n in new]
    groups = []
    if page and r.random() < 0.6:
        b = 0
        while b < B:
            e = int(min(B, b + r.integers(1, B + 1)))
            groups.append((b, e, int(np.exp(r.uniform(0, np.log(8000 if e - b > 1 else 50))))))
            b = e
    return _batch(f"drawn {seed}", new, own, H, H_kv, d, groups=groups, sharing=None, bits=bits, page=page)


SHARED = _shared()
BLOCKS = _blocks()
