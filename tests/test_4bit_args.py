"""What the calls refuse of a 4-bit cache, what sp_cache_read refuses, and the format's oracle against its literal values.  No GPU
needed: device pointers are made up and never used."""
import ctypes as C
import os
import re

import numpy as np
import pytest
import torch

from oracle import mxfp4_oracle as mx
from paper_2502_02789_amd import binding as sp
from tests.test_cache_args import P, ROOT, _append, _attend

FOUR = dict(cache_dtype=sp.SP_K_MXFP4, d_k_block_scale=P + 0x300000, d_v_block_scale=P + 0x310000)


def _read(**kw):
    a = sp.CacheReadArgs()
    base = dict(B=2, H_kv=2, d=64, T_rows=10, d_cu_rows=P, d_first=P + 64, d_index=P + 128, d_k_cache=P + 65536, d_v_cache=P + 131072,
                cache_token_stride=128, cache_head_stride=64, cache_page_stride=2048, d_block_table=P + 512, page_size=16, blocks_per_seq=4,
                n_rows=160, d_k_out=P + 4096, k_out_token_stride=128, k_out_head_stride=64, d_v_out=P + 16384, v_out_token_stride=128,
                v_out_head_stride=64)
    for k, v in dict(base, **kw).items():
        setattr(a, k, v)
    return a


BOTH_BAD = [
    (sp.SP_ENULL, dict(FOUR, d_k_block_scale=None)), (sp.SP_ENULL, dict(FOUR, d_v_block_scale=None)), (sp.SP_EINVAL, dict(FOUR, d_k_scale=P)),
    (sp.SP_EINVAL, dict(FOUR, d_v_scale=P)), (sp.SP_EINVAL, dict(d_k_block_scale=P)), (sp.SP_EINVAL, dict(d_v_block_scale=P)),
    (sp.SP_EINVAL, dict(d_k_block_scale=P, cache_dtype=sp.SP_K_FP8_E4M3)), (sp.SP_EALIGN, dict(FOUR, cache_token_stride=144)),
    (sp.SP_EALIGN, dict(FOUR, cache_head_stride=80)), (sp.SP_EALIGN, dict(FOUR, cache_page_stride=2064)), (sp.SP_EALIGN, dict(FOUR, d_k_cache=P + 65544)),
    (sp.SP_EALIGN, dict(FOUR, cache_token_stride=160)), (sp.SP_EALIGN, dict(FOUR, d_k_block_scale=P + 0x300001)), (sp.SP_EALIGN, dict(FOUR, d_v_block_scale=P + 0x310001)),
    (sp.SP_EINVAL, dict(FOUR, cache_dtype=3)), (sp.SP_EINVAL, dict(FOUR, cache_dtype=5)),
]


@pytest.mark.parametrize("status,change", BOTH_BAD)
def test_4_bit_caches_are_checked(status, change):
    lib = sp.load_library()
    assert lib.sp_cache_append(C.byref(_append(**change)), None) == status
    assert lib.sp_attend(C.byref(_attend(**change)), None) == status
    assert lib.sp_cache_read(C.byref(_read(**change)), None) == status


def test_append_refuses_scales_over_scales_and_scoring_a_4_bit_cache():
    lib = sp.load_library()
    assert lib.sp_cache_append(C.byref(_append(**dict(FOUR, d_v_block_scale=FOUR["d_k_block_scale"]))), None) == sp.SP_EINVAL
    assert lib.sp_cache_append(C.byref(_append(**dict(FOUR, T_new=0))), None) == sp.SP_OK
    assert lib.sp_attend(C.byref(_attend(**dict(FOUR, T_new=0))), None) == sp.SP_OK
    from tests.test_abi import _fake_score_args
    a = _fake_score_args()
    a.k_dtype = sp.SP_K_MXFP4
    assert lib.sp_score(C.byref(a), None) == sp.SP_EINVAL and lib.sp_score_workspace_bytes(C.byref(a)) == 0


READ_BAD = [
    (sp.SP_EINVAL, dict(B=0)), (sp.SP_EINVAL, dict(d=96)), (sp.SP_EINVAL, dict(H_kv=0)), (sp.SP_EINVAL, dict(H_kv=1025)), (sp.SP_EINVAL, dict(T_rows=-1)),
    (sp.SP_EINVAL, dict(T_rows=(1 << 25) + 1)), (sp.SP_EINVAL, dict(n_rows=0)), (sp.SP_EINVAL, dict(n_rows=1 << 31)), (sp.SP_EINVAL, dict(n_rows=161)),
    (sp.SP_EINVAL, dict(cache_dtype=2)), (sp.SP_EINVAL, dict(d_k_scale=P)), (sp.SP_ENULL, dict(d_cu_rows=None)), (sp.SP_ENULL, dict(d_k_cache=None)),
    (sp.SP_ENULL, dict(d_v_cache=None)), (sp.SP_ENULL, dict(d_k_out=None)), (sp.SP_ENULL, dict(d_v_out=None)), (sp.SP_ENULL, dict(d_block_table=None)),
    (sp.SP_EINVAL, dict(d_cu_cache=P)), (sp.SP_EINVAL, dict(page_size=4)), (sp.SP_EINVAL, dict(page_size=24)), (sp.SP_EINVAL, dict(blocks_per_seq=0)),
    (sp.SP_EINVAL, dict(cache_token_stride=-32)), (sp.SP_EINVAL, dict(k_out_token_stride=-8)), (sp.SP_EINVAL, dict(k_out_token_stride=56)),
    (sp.SP_EINVAL, dict(v_out_head_stride=32)), (sp.SP_EINVAL, dict(d_v_out=P + 4096)), (sp.SP_EALIGN, dict(v_out_token_stride=132)),
    (sp.SP_EALIGN, dict(d_k_out=P + 8)), (sp.SP_EALIGN, dict(cache_head_stride=68)), (sp.SP_EALIGN, dict(d_v_cache=P + 4)),
    (sp.SP_EINVAL, dict(d_v_cache=None, d_v_out=None, d_v_scale=P, cache_dtype=sp.SP_K_FP8_E4M3)),
    (sp.SP_EINVAL, dict(FOUR, d_v_cache=None, d_v_out=None)),
]


@pytest.mark.parametrize("status,change", READ_BAD)
def test_read_refuses(status, change):
    assert sp.load_library().sp_cache_read(C.byref(_read(**change)), None) == status


def test_read_of_nothing():
    lib = sp.load_library()
    assert lib.sp_cache_read(None, None) == sp.SP_ENULL
    assert lib.sp_cache_read(C.byref(_read(T_rows=0, d_k_out=None, d_v_out=None)), None) == sp.SP_OK
    assert lib.sp_cache_read(C.byref(_read(T_rows=0, d_v_cache=None, d_k_out=None, d_v_out=None)), None) == sp.SP_OK


def test_struct_layouts_match_the_header():
    text = open(os.path.join(ROOT, "include", "specprefill.h")).read()
    kinds = {C.c_int32: "int32_t ", C.c_int64: "int64_t ", C.c_float: "float ", C.c_size_t: "size_t "}
    for cname, cls in (("sp_cache_read_args", sp.CacheReadArgs), ("sp_verify_args", sp.VerifyArgs)):
        body = re.search(r"typedef struct \{([^}]*)\}\s*" + cname + ";", text).group(1)
        decls = [d.strip() for d in re.sub(r"/\*.*?\*/", "", body, flags=re.S).split(";") if d.strip()]
        assert [re.search(r"(\w+)\s*$", d).group(1) for d in decls] == [f[0] for f in cls._fields_], cname
        for d, (_, t) in zip(decls, cls._fields_):
            assert "*" in d if t is C.c_void_p else d.startswith(kinds[t]) and "*" not in d, d


def test_device_classes_tell_4_bit_caches_from_8_bit_ones():
    from paper_2502_02789_amd import device as dev
    codes = torch.zeros((4, 16, 2, 64), dtype=torch.uint8)
    four = codes.view(torch.float4_e2m1fn_x2)
    scales = torch.zeros((4, 16, 2, 4), dtype=torch.uint8)
    dev._check_block_scales(four, scales, "s")
    dev._check_block_scales(four, scales.view(torch.float8_e8m0fnu), "s")
    dev._check_block_scales(codes, None, "s")
    for cache, s in ((four, None), (codes, scales), (four, scales[:, :, :, :3]), (four, scales.int()), (four, scales[:, :8]),
                     (four, scales.transpose(1, 2).contiguous().transpose(1, 2))):
        with pytest.raises(ValueError):
            dev._check_block_scales(cache, s, "s")
    assert dev._head_dim(four) == 128 and dev._head_dim(codes) == 64
    with pytest.raises(ValueError):
        dev._check_cache(four, four, None, None, 1)
    table = torch.zeros((1, 4), dtype=torch.int32)
    with pytest.raises(ValueError):  # fp32 scales are of 8-bit caches
        dev._check_cache(four, four, table, None, 1, (torch.ones(2),))
    a = sp.make_attend_plan_args(torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), four, H=4, total_new=1, block_table=table)
    assert (a.d, a.cache_dtype, a.cache_token_stride, a.cache_head_stride, a.cache_page_stride) == (128, sp.SP_K_MXFP4, 256, 128, 4096)


def test_cache_helper_lays_heads_outermost():
    from paper_2502_02789_amd import device as dev
    for rows, lead in (((5, 16), (5, 16)), (7, (7,))):
        codes, scales = dev.mxfp4_cache(rows, 3, 128, device="cpu")
        assert codes.shape == (*lead, 3, 64) and scales.shape == (*lead, 3, 4)
        assert codes.stride(-3) == 64 and scales.stride(-3) == 4
        dev._check_block_scales(codes, scales, "s")


def test_oracle_values_and_rounding():
    """The format's 16 values; every value and every number half-way between two, with the scales that they get."""
    codes = np.arange(16, dtype=np.uint8).repeat(2)[None]
    want = np.array([0, .5, 1, 1.5, 2, 3, 4, 6, -0.0, -.5, -1, -1.5, -2, -3, -4, -6]).repeat(2)
    for s, f in ((127, 1.0), (130, 8.0), (1, 2.0 ** -126), (0, 2.0 ** -127), (254, 2.0 ** 127)):
        assert (mx.values(codes, np.array([[s]], np.uint8))[0] == want * f).all()
    assert np.isnan(mx.values(codes, np.array([[255]], np.uint8))).all()
    x = np.zeros((1, 32), np.float32)
    x[0, :16] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5, 7]
    x[0, 16:20] = [0.2500001, 0.7499999, 5.0000005, -0.0]
    c, s = mx.quantise(x)
    assert s[0, 0] == 127
    assert mx.values(c, s)[0, :20].tolist() == [6, 0, 1, 1, 2, 2, 4, 4, 0, -1, -1, -2, -2, -4, -4, 6, 0.5, 0.5, 6, 0]
    for top, want in ((7.0, 127), (np.nextafter(np.float32(7), np.float32(8)), 128), (3.5, 126), (np.nextafter(np.float32(3.5), np.float32(8)), 127), (0.0, 2),
                      (2.0 ** -130, 2), (7 * 2.0 ** -125, 2), (7.01 * 2.0 ** -125, 3), (np.nan, 255), (np.inf, 255)):
        x = np.zeros((1, 32), np.float32)
        x[0, 5] = -top
        assert mx.quantise(x)[1][0, 0] == want, top
    assert (mx.unpack(mx.pack(codes)) == codes).all()


def test_scoring_takes_no_4_bit_tensor():
    """A tensor of 4-bit codes has elements of one byte, as an 8-bit cache has, but half as many."""
    q, cu = torch.zeros(1, 1, 1, 8, 128, dtype=torch.bfloat16), torch.tensor([0, 16], dtype=torch.int32)
    codes = torch.zeros(16, 2, 64, dtype=torch.uint8).view(torch.float4_e2m1fn_x2)
    with pytest.raises(ValueError, match="4-bit"):
        sp.make_score_args(q, [codes], cu, torch.zeros(16), H_kv=2, scale=1.0)
