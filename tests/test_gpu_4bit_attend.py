"""GPU: sp_attend over a 4-bit cache against the fp64 oracle: every value within the bound that its roundings allow (the codes' values are exact, so
the bounds are those of a bf16 cache); the scales of what lies behind the sequences are NaN throughout."""
import math

import numpy as np
import pytest

from oracle import cache_oracle as co
from oracle import mxfp4_oracle as mx
from tests import cache_cases as cc
from tests import mxfp4_cases as mc
from tests import test_gpu_attend as checks

pytestmark = pytest.mark.gpu


def _case(rng, new, length, H, H_kv, d, *, page=16, groups=(), spare=2, head_major=False, scale=None, lo=122, hi=128, tweak=None):
    room = [max(m, 0) + (3 if page else 0) for m in length]
    cache = mc.FourBitCache(rng, room, H_kv, d, page, groups=groups, lo=lo, hi=hi)
    q = cc.normal_bits(rng, (sum(new) + spare, H, d))
    cache.share(groups)
    cache.spoil_unused([max(m, 0) for m in length])
    if tweak:
        tweak(cache, q)
    return dict(cache=cache, q=q, new=new, length=length, groups=groups, H=H, head_major=head_major, scale=scale or co.softmax_scale(d))


LAYOUTS = [dict(page=16), dict(page=8, head_major=True), dict(page=0), dict(page=0, head_major=True), dict(page=64, head_major=True), dict(page=1024)]
HEADS = [(8, 2, 128), (8, 2, 64), (3, 1, 128), (16, 1, 64), (5, 5, 64), (32, 2, 128)]


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("heads", HEADS)
def test_single_tokens(layout, heads):
    rng = np.random.default_rng(1)
    length = [1, 2, 15, 16, 17, 31, 33, 127, 129, 500, 1111]
    checks._run(_case(rng, [1] * len(length), length, *heads, **layout))


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("heads", HEADS)
def test_several_tokens_and_whole_prompts(layout, heads):
    rng = np.random.default_rng(2)
    checks._run(_case(rng, [1, 4, 0, 33, 64, 65, 130, 2], [1, 4, 9, 33, 300, 65, 140, 900], *heads, **layout))


@pytest.mark.parametrize("n", [1, 3, 7, 40])
@pytest.mark.parametrize("m", [1, 63, 64, 65, 128, 200, 2047, 5001])
def test_one_sequence_of_any_length(n, m):
    rng = np.random.default_rng(m + n)
    checks._run(_case(rng, [min(n, m)], [m], 8, 2, 128, head_major=True))
    checks._run(_case(rng, [min(n, m)], [m], 4, 2, 64))


@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 4, 64), (16, 1, 128), (3, 1, 64)])
@pytest.mark.parametrize("layout", [dict(page=16), dict(page=64, head_major=True), dict(page=8)])
def test_shared_prefixes(heads, layout):
    rng = np.random.default_rng(3)
    for new, own, groups in [([1] * 12, [3, 40, 1, 99, 8, 17, 64, 65, 5, 2, 31, 200], [(0, 12, 700)]),
                             ([1, 3, 0, 8, 1, 1, 2, 4], [10, 3, 5, 100, 1, 70, 2, 9], [(0, 4, 333), (4, 6, 1), (6, 8, 129)]),
                             ([60, 2, 1, 200, 1], [60, 80, 1, 210, 33], [(0, 3, 150), (3, 5, 90)])]:
        length = [o + next(p for lo, hi, p in groups if lo <= b < hi) for b, o in enumerate(own)]
        checks._run(_case(rng, new, length, *heads, groups=groups, **layout))


@pytest.mark.parametrize("layout", [dict(page=16), dict(page=8, head_major=True), dict(page=0)])
@pytest.mark.parametrize("heads", [(8, 2, 128), (8, 2, 64)])
def test_short_pieces_of_one_and_of_two_tiles_of_rows_side_by_side(heads, layout):
    rng = np.random.default_rng(4)
    new = [1, 5, 6, 8, 8, 4, 1, 1, 7, 5, 0, 5, 9, 8, 2, 6] * 6
    length = [n + int(x) for n, x in zip(new, rng.integers(0, 300, len(new)))]
    length[20], length[50] = 4000, 9000
    checks._run(_case(rng, new, length, *heads, **layout))


def test_more_sequences_than_the_plan_keeps_in_lds_and_more_kv_heads_than_workgroups():
    rng = np.random.default_rng(5)
    length = rng.integers(9, 40, 700).tolist()
    checks._run(_case(rng, [int(min(n, m - 8)) for n, m in zip(rng.integers(0, 4, 700), length)], length, 4, 2, 64, page=8))
    checks._run(_case(rng, [1, 20, 2], [300, 70, 9], 300, 300, 128, page=16))


def test_rows_that_see_nothing():
    c = _case(np.random.default_rng(6), [1, 10, 200, 3], [0, 4, 150, 3], 8, 2, 128)
    _, a = checks._run(c)
    assert (a.out[0] == 0).all() and a.lse[0].isneginf().all() and (a.out[1:7] == 0).all()


@pytest.mark.parametrize("heads", [(8, 2, 128), (8, 2, 64)])
@pytest.mark.parametrize("lo,hi", [(0, 4), (60, 70), (100, 140)])
def test_scales_far_from_one(lo, hi, heads):
    """Blocks whose scales differ by factors of up to 2^40 within a row, and the smallest of the format."""
    rng = np.random.default_rng(7)
    checks._run(_case(rng, [1, 3, 60], [300, 77, 60], *heads, lo=lo, hi=hi, scale=2.0 ** -14 if hi > 128 else None))


def test_each_key_and_each_element_counts():
    """A key among 700 that alone is aligned with the query, at every place in turn: its value comes out, every element in its place."""
    import torch
    from paper_2502_02789_amd import device as dev
    rng = np.random.default_rng(8)
    for d, page, head_major in ((128, 16, True), (64, 8, False), (128, 0, False)):
        m, H_kv = 700, 2
        cache = mc.FourBitCache(rng, [m], H_kv, d, page, lo=126, hi=129)
        rows = cache.rows(0, m)
        cache.k[rows] = 0
        q = np.zeros((1, H_kv, d), np.float32)
        q[0, :, :] = 4.0
        for i in list(range(0, 140)) + [511, 512, 513, 639, 640, 698, 699]:
            cache.k[rows[i]], cache.k_blocks[rows[i]] = 7, 130        # 48 in every element
            where, kc, vc, scales = cache.device(head_major)
            plan = dev.AttendPlan(cc.cuda_ints([0, 1]), cc.cuda_ints([m]), kc, H=H_kv, total_new=1, **where)
            plan.run()
            got = dev.Attender(plan, torch.from_numpy(q).cuda().bfloat16(), kc, vc, scale=1.0, **scales).run()
            assert (got[0].double().cpu().numpy() == cache.values()[1][rows[i]]).all(), (d, page, i)
            cache.k[rows[i]] = 0


def test_pages_outside_the_pool_and_lengths_that_are_none():
    import torch

    def bad(cache, q):
        cache.table[1, 2], cache.table[3, 0] = 1 << 28, -7
    for heads in ((8, 2, 128), (8, 2, 64)):
        c = _case(np.random.default_rng(9), [1, 1, 70, 3], [100, 90, 200, 60], *heads, tweak=bad)
        plan, a = checks._device(c)
        plan.run()
        a.run()
        torch.cuda.synchronize()
        assert a.out[1].isnan().all() and a.lse[1].isnan().all() and a.out[72:75].isnan().all() and a.lse[72:75].isnan().all()
        good = np.r_[0, 2:72]
        for b in (1, 3):
            c["cache"].table[b] = c["cache"].table[0]
        checks._check(c, a, rows=good)
        c = _case(np.random.default_rng(10), [1, 1, 40], [100, 64, 80], *heads)
        c["length"] = [100, 1 << 20, -1]
        plan, a = checks._device(c)
        plan.run()
        a.run()
        torch.cuda.synchronize()
        assert a.out[1:42].isnan().all() and a.lse[1:42].isnan().all() and a.out[0].isfinite().all()


def test_a_plan_of_another_type_gives_nan_and_the_class_refuses_it():
    import torch
    from paper_2502_02789_amd import binding as sp
    from paper_2502_02789_amd import device as dev
    rng = np.random.default_rng(11)
    c = _case(rng, [1], [50], 8, 2, 128)
    plan, a = checks._device(c)
    eight = cc.Cache(rng, [53], 2, 64, 16, 8)
    where, kc, vc, scales = eight.device()
    with pytest.raises(ValueError):
        dev.Attender(plan, torch.zeros((3, 8, 64), dtype=torch.bfloat16, device="cuda"), kc, vc, scale=1.0, **scales)
    args = type(a.args).from_buffer_copy(a.args)
    plan.args.cache_dtype = sp.SP_K_FP8_E4M3      # (the plan's size is the same)
    plan.run()
    sp.sp_attend(args)
    torch.cuda.synchronize()
    assert a.out.isnan().all() and a.lse.isnan().all()


def test_the_same_on_every_run_on_another_stream_and_in_a_graph():
    import torch
    rng = np.random.default_rng(12)
    c = _case(rng, [1, 2, 5, 90], [700, 1500, 130, 400], 8, 2, 128, head_major=True)
    plan, a = checks._run(c)
    want, want_lse = a.out.clone(), a.lse.clone()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        a.out.fill_(1.0)
        plan.run()
        a.run()
    torch.cuda.current_stream().wait_stream(stream)
    assert torch.equal(a.out[:98], want[:98])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.run()
        a.run()
    for _ in range(3):
        a.out.fill_(7.0)
        a.lse.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a.out, want) and torch.equal(a.lse, want_lse)


def test_agrees_with_the_bf16_cache_of_the_same_values():
    """The values read back into a bf16 cache: the same definition on the same numbers, so both lie within its bounds."""
    import torch
    from paper_2502_02789_amd import device as dev
    rng = np.random.default_rng(13)
    for heads in ((8, 2, 128), (4, 4, 64)):
        c = _case(rng, [1, 3, 100], [900, 64, 100], *heads, page=16, spare=0)
        _, a = checks._run(c)
        where, kc, vc, scales = c["cache"].device()
        pages = kc.shape[0]
        all_rows = cc.cuda_ints([0, pages * 16])
        flat = dict(block_table=torch.arange(pages, dtype=torch.int32, device="cuda").view(1, -1))
        wide = [torch.empty((pages * 16, heads[1], heads[2]), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        dev.CacheReader(kc, vc, all_rows, total=pages * 16, k_out=wide[0], v_out=wide[1], **flat, **scales).run()
        wide = [x.view(pages, 16, heads[1], heads[2]) for x in wide]
        plan = dev.AttendPlan(cc.cuda_ints(cc.offsets(c["new"])), cc.cuda_ints(c["length"]), wide[0], H=heads[0], total_new=len(c["q"]), **where)
        plan.run()
        b = dev.Attender(plan, dev.bf16_from_bits(c["q"]), *wide, scale=c["scale"], want_lse=True)
        b.run()
        torch.cuda.synchronize()
        out, lse, size, reach = checks._oracle(c)
        tol, tol_l = co.attend_bounds(out, lse, size, reach, heads[2], 900)
        assert (np.abs(a.out.double().cpu().numpy() - b.out.double().cpu().numpy()) <= 2 * tol).all()
        assert (np.abs(a.lse.double().cpu().numpy() - b.lse.double().cpu().numpy()) <= 2 * tol_l).all()
        assert math.isfinite(float(b.lse.sum()))


@pytest.mark.parametrize("paged", [False, True])
def test_beyond_offsets_of_2_to_the_32(paged):
    """More than 2^32 bytes of codes, token strides of 2^16 bytes: one key of all is aligned with the query, and its value comes out."""
    import torch
    from paper_2502_02789_amd import device as dev
    rows, H_kv, d, page = 70016, 2, 128, 16

    def wide(n):
        pool = torch.zeros((rows, n), dtype=torch.uint8, device="cuda")
        return pool, pool[:, :H_kv * d // (2 if n == 65536 else 32)].unflatten(1, (H_kv, d // (2 if n == 65536 else 32)))
    (kp, k), (_, v), (_, ks), (_, vs) = wide(65536), wide(65536), wide(4096), wide(4096)
    g = torch.Generator(device="cuda")
    g.manual_seed(14)
    v.copy_(torch.randint(0, 256, v.shape, generator=g, device="cuda").to(torch.uint8))
    ks.fill_(127)
    vs.copy_(torch.randint(125, 130, vs.shape, generator=g, device="cuda").to(torch.uint8))
    q = torch.full((1, 4, d), 4.0, dtype=torch.bfloat16, device="cuda")
    parts = [k, v, ks, vs]
    if paged:
        parts = [x.unflatten(0, (rows // page, page)) for x in parts]
        where = dict(block_table=torch.arange(rows // page, dtype=torch.int32, device="cuda").flip(0).view(1, -1).contiguous())
    else:
        where = dict(cu_cache=cc.cuda_ints([0, rows]))
    kc, vc = (x.view(torch.float4_e2m1fn_x2) for x in parts[:2])
    plan = dev.AttendPlan(cc.cuda_ints([0, 1]), cc.cuda_ints([rows - 5]), kc, H=4, total_new=1, **where)
    plan.run()
    a = dev.Attender(plan, q, kc, vc, scale=1.0, k_block_scale=parts[2], v_block_scale=parts[3])
    for i in (0, 17, 40000, 65535, 65536, 69999, rows - 6):
        row = (rows // page - 1 - i // page) * page + i % page if paged else i
        k[row] = 0x77
        got = a.run()
        torch.cuda.synchronize()
        kp[row] = 0
        codes = torch.stack([v[row] & 15, v[row] >> 4], dim=-1).flatten(-2).cpu().numpy()
        want = mx.values(codes, vs[row].cpu().numpy())
        assert (got[0].view(H_kv, 2, d).double().cpu().numpy() == want[:, None]).all(), i
