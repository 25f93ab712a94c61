"""The sizes that sp_verify takes are the ones that its header names.  No GPU needed: only sizes are asked for."""
import itertools

import pytest

from paper_2502_02789_amd import binding as sp


def _taken(B, V, T):
    a = sp.VerifyArgs()
    a.B, a.V, a.T, a.logits_dtype = B, V, T, sp.SP_LOGITS_BF16
    return sp.sp_verify_workspace_bytes(a) > 0


def _named(B, V, T):
    return 1 <= B and 1 <= V < 1 << 24 and 0 <= T and (2 * T + B) * -(-V // 8192) < 1 << 24 and B * -(-V // 4096) < 1 << 24


@pytest.mark.parametrize("V", [1, 2048, 4096, 4097, 8192, 8193, 9 * 8192, 128256, (1 << 24) - 1, 1 << 24])
def test_limits(V):
    slices, parts = -(-V // 8192), -(-V // 4096)
    sizes = {1, 2, 511, 512, 513, *(((1 << 24) - 1) // n + k for n in (slices, parts) for k in (-1, 0, 1))}
    for B, T in itertools.product([b for b in sizes if 0 < b < 1 << 31], sorted({0, 1, *sizes, *(s // 2 for s in sizes)})):
        assert _taken(B, V, T) == _named(B, V, T), (B, T)
