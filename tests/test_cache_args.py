"""What sp_cache_append, sp_attend_plan and sp_attend refuse on the host, before anything is launched; and the oracle's own
pieces against the formats' literal values.  No GPU needed: device pointers are made up and never used."""
import ctypes as C
import os
import re

import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from oracle import specprefill_oracle as orc
from paper_2502_02789_amd import binding as sp

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x7000_0000_0000


def _append(**kw):
    a = sp.CacheAppendArgs()
    base = dict(B=2, H=8, H_kv=2, d=64, T_new=10, d_q=P, q_token_stride=768, q_head_stride=64, d_k=P + 4096, k_token_stride=768, k_head_stride=64,
                d_v=P + 8192, v_token_stride=768, v_head_stride=64, d_cu_new=P + 64, d_cache_len=P + 128, d_pos=P + 256, rope_theta=5e5,
                d_q_out=P + 16384, d_k_cache=P + 65536, d_v_cache=P + 131072, cache_token_stride=128, cache_head_stride=64,
                cache_page_stride=2048, d_block_table=P + 512, page_size=16, blocks_per_seq=4, n_rows=160)
    for k, v in dict(base, **kw).items():
        setattr(a, k, v)
    return a


def _attend(**kw):
    a = sp.AttendArgs()
    base = dict(B=2, H=8, H_kv=2, d=64, T_new=10, d_cu_new=P, d_kv_len=P + 64, d_block_table=P + 512, page_size=16, blocks_per_seq=4, n_rows=160,
                d_q=P + 4096, q_token_stride=512, q_head_stride=64, d_k_cache=P + 65536, d_v_cache=P + 131072, cache_token_stride=128,
                cache_head_stride=64, cache_page_stride=2048, scale=0.125, d_out=P + 16384, out_token_stride=512, out_head_stride=64,
                d_plan=P + 0x100000, plan_bytes=1 << 30, d_workspace=P + 0x200000, workspace_bytes=1 << 40)
    for k, v in dict(base, **kw).items():
        setattr(a, k, v)
    return a


FP8 = dict(cache_dtype=sp.SP_K_FP8_E4M3)
APPEND_BAD = [
    (sp.SP_EINVAL, dict(B=0)), (sp.SP_EINVAL, dict(d=96)), (sp.SP_EINVAL, dict(H=7)), (sp.SP_EINVAL, dict(H=34)), (sp.SP_EINVAL, dict(H=0)),
    (sp.SP_EINVAL, dict(H_kv=0)), (sp.SP_EINVAL, dict(H=2048, H_kv=256)), (sp.SP_EINVAL, dict(T_new=-1)), (sp.SP_EINVAL, dict(T_new=1 << 28)),
    (sp.SP_EINVAL, dict(n_rows=0)), (sp.SP_EINVAL, dict(n_rows=1 << 31)), (sp.SP_EINVAL, dict(n_rows=161)), (sp.SP_EINVAL, dict(cache_dtype=2)),
    (sp.SP_EINVAL, dict(d_k_scale=P)), (sp.SP_EINVAL, dict(rope_theta=-1.0)), (sp.SP_EINVAL, dict(rope_theta=float("nan"))),
    (sp.SP_EINVAL, dict(rope_theta=float("inf"))), (sp.SP_EINVAL, dict(d_inv_freq=P)), (sp.SP_EINVAL, dict(rope_theta=0.0)),
    (sp.SP_ENULL, dict(d_k=None)), (sp.SP_ENULL, dict(d_v=None)), (sp.SP_ENULL, dict(d_cu_new=None)), (sp.SP_ENULL, dict(d_k_cache=None)),
    (sp.SP_ENULL, dict(d_v_cache=None)), (sp.SP_ENULL, dict(d_q_out=None)), (sp.SP_ENULL, dict(d_q=None)), (sp.SP_ENULL, dict(d_block_table=None)),
    (sp.SP_EINVAL, dict(d_cu_cache=P)), (sp.SP_EINVAL, dict(page_size=4)), (sp.SP_EINVAL, dict(page_size=24)), (sp.SP_EINVAL, dict(blocks_per_seq=0)),
    (sp.SP_EINVAL, dict(blocks_per_seq=1 << 27)), (sp.SP_EINVAL, dict(k_token_stride=-8)), (sp.SP_EINVAL, dict(cache_page_stride=-16)),
    (sp.SP_EALIGN, dict(k_token_stride=772)), (sp.SP_EALIGN, dict(v_head_stride=4)), (sp.SP_EALIGN, dict(q_head_stride=4)),
    (sp.SP_EALIGN, dict(cache_token_stride=132)), (sp.SP_EALIGN, dict(cache_token_stride=136, **FP8)), (sp.SP_EALIGN, dict(cache_page_stride=2056, **FP8)),
    (sp.SP_EALIGN, dict(d_k=P + 2)), (sp.SP_EALIGN, dict(d_q=P + 8)), (sp.SP_EALIGN, dict(d_q_out=P + 8)), (sp.SP_EALIGN, dict(d_v_cache=P + 8)),
    (sp.SP_EINVAL, dict(d_q=None, d_q_out=None, T_new=(1 << 25) + 1)),
]
PLAN_BAD = [
    (sp.SP_EINVAL, dict(B=0)), (sp.SP_EINVAL, dict(d=32)), (sp.SP_EINVAL, dict(H=9)), (sp.SP_EINVAL, dict(H=34)), (sp.SP_EINVAL, dict(H=2048, H_kv=256)),
    (sp.SP_EINVAL, dict(T_new=-1)), (sp.SP_EINVAL, dict(T_new=1 << 28)), (sp.SP_EINVAL, dict(n_groups=-1)), (sp.SP_EINVAL, dict(n_groups=3, d_cu_group=P, d_prefix_len=P)),
    (sp.SP_EINVAL, dict(n_rows=0)), (sp.SP_EINVAL, dict(n_rows=1 << 31)), (sp.SP_EINVAL, dict(n_rows=161)), (sp.SP_EINVAL, dict(cache_dtype=-1)), (sp.SP_EINVAL, dict(page_size=12)),
    (sp.SP_EINVAL, dict(page_size=4)), (sp.SP_EINVAL, dict(blocks_per_seq=0)), (sp.SP_ENULL, dict(d_cu_new=None)), (sp.SP_ENULL, dict(d_kv_len=None)),
    (sp.SP_ENULL, dict(d_block_table=None)), (sp.SP_EINVAL, dict(d_cu_cache=P)), (sp.SP_ENULL, dict(n_groups=1, d_cu_group=P)),
    (sp.SP_ENULL, dict(n_groups=1, d_prefix_len=P)), (sp.SP_EINVAL, dict(d_cu_group=P)), (sp.SP_EINVAL, dict(d_prefix_len=P)),
    (sp.SP_EUNSUPPORTED, dict(n_groups=1, d_cu_group=P, d_prefix_len=P, d_block_table=None, d_cu_cache=P)), (sp.SP_ENULL, dict(d_plan=None)),
    (sp.SP_EALIGN, dict(d_plan=P + 16)), (sp.SP_EWORKSPACE, dict(plan_bytes=64)),
    (sp.SP_EINVAL, dict(n_rows=0x7fff0010)), (sp.SP_EINVAL, dict(blocks_per_seq=0x7fff001)),
    (sp.SP_EINVAL, dict(B=1 << 22, T_new=1 << 22, H=8, H_kv=8)), (sp.SP_EINVAL, dict(T_new=(1 << 31) // 64 - 1, H=64, H_kv=4, d=128)),  # threads of a launch
]
ATTEND_BAD = PLAN_BAD + [
    (sp.SP_EINVAL, dict(scale=0.0)), (sp.SP_EINVAL, dict(scale=-1.0)), (sp.SP_EINVAL, dict(scale=float("nan"))), (sp.SP_EINVAL, dict(scale=float("inf"))),
    (sp.SP_EINVAL, dict(d_v_scale=P)), (sp.SP_ENULL, dict(d_q=None)), (sp.SP_ENULL, dict(d_k_cache=None)), (sp.SP_ENULL, dict(d_v_cache=None)),
    (sp.SP_ENULL, dict(d_out=None)), (sp.SP_EINVAL, dict(q_token_stride=-8)), (sp.SP_EINVAL, dict(cache_head_stride=-64)),
    (sp.SP_EALIGN, dict(q_token_stride=516)), (sp.SP_EALIGN, dict(out_head_stride=68)), (sp.SP_EALIGN, dict(cache_token_stride=132)),
    (sp.SP_EALIGN, dict(cache_token_stride=136, **FP8)), (sp.SP_EALIGN, dict(d_q=P + 8)), (sp.SP_EALIGN, dict(d_out=P + 8)),
    (sp.SP_EALIGN, dict(d_k_cache=P + 4)), (sp.SP_EWORKSPACE, dict(workspace_bytes=1024)), (sp.SP_EWORKSPACE, dict(d_workspace=None)),
    (sp.SP_EALIGN, dict(d_workspace=P + 16)), (sp.SP_EINVAL, dict(scale=3e38)), (sp.SP_EINVAL, dict(cache_token_stride=1 << 26)),
]


@pytest.mark.parametrize("status,change", APPEND_BAD)
def test_append_refuses(status, change):
    assert sp.load_library().sp_cache_append(C.byref(_append(**change)), None) == status


@pytest.mark.parametrize("status,change", PLAN_BAD)
def test_plan_refuses(status, change):
    assert sp.load_library().sp_attend_plan(C.byref(_attend(**change)), None) == status


@pytest.mark.parametrize("status,change", ATTEND_BAD)
def test_attend_refuses(status, change):
    assert sp.load_library().sp_attend(C.byref(_attend(**change)), None) == status


def test_null_structs_no_tokens_and_sizes():
    lib = sp.load_library()
    assert lib.sp_cache_append(None, None) == lib.sp_attend_plan(None, None) == lib.sp_attend(None, None) == sp.SP_ENULL
    assert lib.sp_attend_plan_bytes(None) == lib.sp_attend_workspace_bytes(None) == 0
    assert lib.sp_cache_append(C.byref(_append(T_new=0)), None) == sp.SP_OK      # nothing to do, nothing launched
    assert lib.sp_attend(C.byref(_attend(T_new=0)), None) == sp.SP_OK
    nothing = dict(T_new=0, d_q=None)                                            # (tensors without elements have no address)
    assert lib.sp_cache_append(C.byref(_append(d_k=None, d_v=None, d_q_out=None, **nothing)), None) == sp.SP_OK
    assert lib.sp_attend(C.byref(_attend(d_out=None, **nothing)), None) == sp.SP_OK
    for bad in (dict(B=0), dict(d=65), dict(H=9), dict(n_rows=0), dict(page_size=9)):
        assert sp.sp_attend_plan_bytes(_attend(**bad)) == sp.sp_attend_workspace_bytes(_attend(**bad)) == 0
    few, many = _attend(T_new=1, B=1), _attend(T_new=4000, B=64, n_groups=4)
    assert 0 < sp.sp_attend_plan_bytes(few) < sp.sp_attend_plan_bytes(many)
    assert 0 < sp.sp_attend_workspace_bytes(few) < sp.sp_attend_workspace_bytes(many)


def test_struct_layouts_match_the_header():
    text = open(os.path.join(ROOT, "include", "specprefill.h")).read()
    for cname, cls in (("sp_cache_append_args", sp.CacheAppendArgs), ("sp_attend_args", sp.AttendArgs)):
        body = re.search(r"typedef struct \{([^}]*)\}\s*" + cname + ";", text).group(1)
        body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
        decls = [d.strip() for d in body.split(";") if d.strip()]
        assert [re.search(r"(\w+)\s*$", d).group(1) for d in decls] == [f[0] for f in cls._fields_], cname
        kinds = {C.c_int32: "int32_t ", C.c_int64: "int64_t ", C.c_float: "float ", C.c_size_t: "size_t "}
        for d, (_, t) in zip(decls, cls._fields_):
            assert "*" in d if t is C.c_void_p else d.startswith(kinds[t]) and "*" not in d, d


def test_device_classes_refuse_tensors_off_the_gpu():
    from paper_2502_02789_amd import device as dev
    k = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    cu = torch.tensor([0, 4], dtype=torch.int32)
    with pytest.raises(ValueError):
        dev.CacheAppender(k, k, cu, k.clone(), k.clone(), cu_cache=cu)
    with pytest.raises(ValueError):
        dev.AttendPlan(cu, cu[1:].clone(), k, H=2, total_new=4, cu_cache=cu)


def test_oracle_e4m3_rounding_against_torch():
    x = np.concatenate([np.linspace(-470, 470, 20001), np.linspace(-0.02, 0.02, 20001), 2.0 ** np.arange(-14, 9)]).astype(np.float32)
    want = torch.from_numpy(np.clip(x, -448, 448)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert (co.f32_to_e4m3_codes(x) == want).all()
    assert co.f32_to_e4m3_codes(np.array([np.nan, np.inf, -np.inf], np.float32)).tolist() == [0x7F, 0x7E, 0xFE]
    y = np.random.default_rng(0).standard_normal(5000).astype(np.float32)
    assert (co.f32_to_bf16_bits(y) == torch.from_numpy(y).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)).all()


def test_oracle_rotation_is_the_scoring_oracle_s():
    rng = np.random.default_rng(1)
    x = co.f32_to_bf16_bits(rng.standard_normal((50, 2, 64)).astype(np.float32))
    pos = rng.integers(0, 131072, 50)
    got = co.f32_to_bf16_bits(co.rotate_f32(x, pos, co.rope_frequencies(5e5, 64)))
    assert (got == orc.rope_rotate_bits(x, pos, 5e5)).mean() > 0.9999


def test_oracle_attention_is_the_scoring_oracle_s_softmax():
    """One sequence, one query per head at the end: the weights are those that sp_score's definition gives the prompt's tokens."""
    rng = np.random.default_rng(2)
    m, H, H_kv, d = 40, 4, 2, 64
    q, k = rng.standard_normal((1, H, d)), rng.standard_normal((m, H_kv, d))
    eye = np.zeros((m, H_kv, d))
    eye[:, :, :] = np.eye(m, d)[:, None]
    cache = {"cu_cache": np.array([0, m]), "n_rows": m}
    out, lse, size, _ = co.attend(q, k, eye, [0, 1], [m], cache, 0.125)
    w, want_lse = orc.layer_attention(q.reshape(1, H, d), k, 0.125)
    np.testing.assert_allclose(out[0][:, :m], w[0].T, rtol=1e-12)
    np.testing.assert_allclose(lse[0], want_lse.reshape(H), rtol=1e-12)
    np.testing.assert_allclose(size, out)
    # causal: the second of two new tokens sees one token more; the first row of three new tokens over two sees nothing
    out2, lse2, _, _ = co.attend(np.repeat(q, 2, 0), k, eye, [0, 2], [m], cache, 0.125)
    np.testing.assert_allclose(out2[1], out[0])
    assert (out2[0][:, m - 1] == 0).all()
    _, lse3, _, _ = co.attend(np.repeat(q, 3, 0), k, eye, [0, 3], [2], cache, 0.125)
    assert np.isneginf(lse3[0]).all() and np.isfinite(lse3[1:]).all()
