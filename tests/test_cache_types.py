"""Which element types of a cache the checks take: bf16 and 8-bit caches need no torch that has a 4-bit type, and scoring takes no 4-bit one."""
import pytest
import torch

from paper_2502_02789_amd import binding as sp
from paper_2502_02789_amd import device as dev


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.uint8, torch.float8_e4m3fn])
def test_other_caches_without_a_4_bit_type(monkeypatch, dtype):
    monkeypatch.delattr(torch, "float4_e2m1fn_x2")
    cache, table = torch.zeros((4, 16, 2, 64), dtype=torch.uint8).to(dtype), torch.zeros((1, 4), dtype=torch.int32)
    dev._check_cache(cache, cache.clone(), table, None, 1, (torch.ones(2),) if cache.element_size() == 1 else ())
    dev._check_block_scales(cache, None, "s")
    assert dev._head_dim(cache) == 64 and not sp.is_4bit(cache)
    with pytest.raises(ValueError):
        dev._check_cache(cache.float(), cache, table, None, 1)


def test_4_bit_caches_are_taken_by_their_own_type_alone():
    codes, table = torch.zeros((4, 16, 2, 64), dtype=torch.uint8), torch.zeros((1, 4), dtype=torch.int32)
    dev._check_cache(codes.view(torch.float4_e2m1fn_x2), codes.view(torch.float4_e2m1fn_x2), table, None, 1)
    for dtype in (torch.float8_e5m2, torch.int8, torch.float16):
        with pytest.raises(ValueError):
            dev._check_cache(codes.to(dtype), codes.to(dtype), table, None, 1)


def test_scoring_takes_no_4_bit_tensor_in_any_layer():
    q, cu = torch.zeros(3, 1, 1, 8, 64, dtype=torch.bfloat16), torch.tensor([0, 16], dtype=torch.int32)
    codes = torch.zeros(16, 2, 64, dtype=torch.uint8)
    for at in range(3):
        layers = [codes] * 3
        layers[at] = codes[:, :, :32].contiguous().view(torch.float4_e2m1fn_x2)
        with pytest.raises(ValueError, match="4-bit"):
            sp.make_score_args(q, layers, cu, torch.zeros(16), H_kv=2, scale=1.0)
    assert sp.make_score_args(q, [codes] * 3, cu, torch.zeros(16), H_kv=2, scale=1.0).k_dtype == sp.SP_K_FP8_E4M3
