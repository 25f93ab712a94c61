"""Layouts in which rows that are written lie in one another are refused on the host: which of two values would be left is anyone's guess.
No GPU needed: device pointers are made up and never used."""
import ctypes as C

import pytest

from paper_2502_02789_amd import binding as sp
from tests.test_cache_args import FP8, P, _append, _attend

CONTIGUOUS = dict(d_block_table=None, d_cu_cache=P + 512)


@pytest.mark.parametrize("change", [
    dict(cache_head_stride=0), dict(cache_head_stride=56), dict(cache_token_stride=0), dict(cache_token_stride=56), dict(cache_page_stride=0),
    dict(cache_page_stride=32), dict(d_v_cache=P + 65536), dict(cache_head_stride=48, cache_token_stride=96, cache_page_stride=1536, **FP8),
    dict(cache_token_stride=0, **CONTIGUOUS), dict(cache_head_stride=0, **CONTIGUOUS),
])
def test_append_refuses_caches_whose_rows_overlap(change):
    assert sp.load_library().sp_cache_append(C.byref(_append(**change)), None) == sp.SP_EINVAL


@pytest.mark.parametrize("change", [
    dict(H_kv=1, H=8, cache_head_stride=0), dict(n_rows=1, cache_token_stride=0, **CONTIGUOUS), dict(n_rows=16, blocks_per_seq=1, cache_page_stride=0),
    dict(cache_page_stride=0, **CONTIGUOUS),
    dict(cache_head_stride=1024, cache_token_stride=64),       # [pages, H_kv, page_size, d]
])
def test_append_takes_strides_that_are_never_used_and_other_orders(change):
    assert sp.load_library().sp_cache_append(C.byref(_append(T_new=0, **change)), None) == sp.SP_OK


@pytest.mark.parametrize("change", [dict(out_head_stride=0), dict(out_head_stride=56), dict(out_token_stride=0), dict(out_token_stride=8)])
def test_attend_refuses_outputs_whose_rows_overlap(change):
    assert sp.load_library().sp_attend(C.byref(_attend(**change)), None) == sp.SP_EINVAL


@pytest.mark.parametrize("change", [
    dict(out_head_stride=640, out_token_stride=64), dict(H=1, H_kv=1, out_head_stride=0),
    dict(q_token_stride=0, q_head_stride=0), dict(cache_head_stride=0), dict(d_v_cache=P + 65536),     # what is only read may be shared
])
def test_attend_takes_other_orders_and_shared_inputs(change):
    assert sp.load_library().sp_attend(C.byref(_attend(T_new=0, **change)), None) == sp.SP_OK
