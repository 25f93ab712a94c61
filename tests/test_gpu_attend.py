"""GPU: sp_attend against the fp64 oracle: every value within the bound that its roundings allow (attend_bounds), on plans of every kind
of batch; what lies behind the sequences in the cache is NaN throughout."""
import math

import numpy as np
import pytest

from oracle import cache_oracle as co
from oracle.specprefill_oracle import bf16_bits_to_f64
from tests import cache_cases as cc

pytestmark = pytest.mark.gpu


def _case(rng, new, length, H, H_kv, d, *, page=16, bits=16, groups=(), spare=2, salient=0.4, head_major=False, scale=None, tweak=None):
    room = [max(m, 0) + (3 if page else 0) for m in length]
    cache = cc.Cache(rng, room, H_kv, d, page, bits, groups=groups)
    q = cc.normal_bits(rng, (sum(new) + spare, H, d))
    if salient and bits == 16:     # some keys aligned with queries: peaked rows, sums that are rescaled
        some = rng.permutation(cache.n_rows)[: cache.n_rows // 20]
        lead = bf16_bits_to_f64(q[rng.integers(0, len(q), len(some))][:, :: H // H_kv])
        cache.k[some] = co.f32_to_bf16_bits((bf16_bits_to_f64(cache.k[some]) + salient * lead).astype(np.float32))
    cache.share(groups)
    cache.spoil_unused([max(m, 0) for m in length])
    if tweak:
        tweak(cache, q)
    return dict(cache=cache, q=q, new=new, length=length, groups=groups, H=H, head_major=head_major, scale=scale or co.softmax_scale(d))


def _device(c, want_lse=True, strided=False):
    import torch
    from paper_2502_02789_amd import device as dev
    where, kc, vc, scales = c["cache"].device(c["head_major"])
    T, H, d = c["q"].shape
    q = dev.bf16_from_bits(c["q"])
    out = torch.full((T, H, d), 7.0, dtype=torch.bfloat16, device="cuda")
    if strided:      # head-major queries, outputs inside wider rows
        q = q.transpose(0, 1).contiguous().transpose(0, 1)
        out = torch.full((T, H + 3, d + 8), 7.0, dtype=torch.bfloat16, device="cuda")[:, 1:H + 1, :d]
    group = {}
    if len(c["groups"]):
        group = dict(cu_group=cc.cuda_ints([g[0] for g in c["groups"]] + [c["groups"][-1][1]]), prefix_len=cc.cuda_ints([g[2] for g in c["groups"]]))
    plan = dev.AttendPlan(cc.cuda_ints(cc.offsets(c["new"])), cc.cuda_ints(c["length"]), kc, H=H, total_new=T, **where, **group)
    a = dev.Attender(plan, q, kc, vc, scale=c["scale"], out=out, want_lse=want_lse, **scales)
    if want_lse:
        a.lse.fill_(7.0)
    return plan, a


def _check(c, a, rows=None, oracle=None):
    """rows: those that are compared (default: all of the sequences')."""
    n = int(sum(c["new"]))
    k, v = c["cache"].values()
    out, lse, size, reach = oracle or _oracle(c)
    tol_o, tol_l = co.attend_bounds(out, lse, size, reach, c["q"].shape[2], max(c["length"]))
    got, got_lse = a.out.float().cpu().numpy().astype(np.float64), a.lse.cpu().numpy().astype(np.float64)
    assert (got[n:] == 7).all() and (got_lse[n:] == 7).all(), "rows behind the last sequence"
    rows = np.arange(n) if rows is None else np.asarray(rows)
    if len(rows) == 0:
        return
    assert np.isfinite(got[rows]).all()
    off = np.abs(got - out)[rows] / tol_o[rows]
    assert off.max() <= 1, f"out: {off.max():.2f} of the bound at row {rows[np.unravel_index(off.argmax(), off.shape)[0]]}"
    empty = np.isinf(lse[rows])
    assert (np.isneginf(got_lse[rows]) == empty).all()
    with np.errstate(invalid="ignore"):
        off = np.where(empty, 0, np.abs(got_lse - lse)[rows] / tol_l[rows])
    assert off.max() <= 1, f"lse: {off.max():.2f} of the bound"


def _oracle(c):
    k, v = c["cache"].values()
    n = int(sum(c["new"]))
    return co.attend(bf16_bits_to_f64(c["q"]), k, v, cc.offsets(c["new"]), c["length"], c["cache"].where(), c["scale"])


def _run(c, **kw):
    import torch
    plan, a = _device(c, **kw)
    plan.run()
    a.run()
    torch.cuda.synchronize()
    _check(c, a)
    return plan, a


LAYOUTS = [dict(page=16), dict(page=8), dict(page=0), dict(page=64, head_major=True), dict(page=16, bits=8), dict(page=0, bits=8)]
HEADS = [(8, 2, 128), (8, 2, 64), (3, 1, 128), (16, 1, 64), (5, 5, 64), (32, 2, 128)]


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("heads", HEADS)
def test_single_tokens(layout, heads):
    rng = np.random.default_rng(1)
    length = [1, 2, 15, 16, 17, 31, 33, 127, 129, 500, 1111]
    _run(_case(rng, [1] * len(length), length, *heads, **layout))


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("heads", HEADS)
def test_several_tokens_and_whole_prompts(layout, heads):
    rng = np.random.default_rng(2)
    _run(_case(rng, [1, 4, 0, 33, 64, 65, 130, 2], [1, 4, 9, 33, 300, 65, 140, 900], *heads, **layout))


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("n", [1, 3, 40])
@pytest.mark.parametrize("m", [1, 63, 64, 65, 128, 200, 2047, 5001])
def test_one_sequence_of_any_length(n, m, bits):
    rng = np.random.default_rng(m + n)
    _run(_case(rng, [min(n, m)], [m], 8, 2, 128, bits=bits))


@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 4, 64), (16, 1, 128), (3, 1, 64)])
@pytest.mark.parametrize("layout", [dict(page=16), dict(page=64, bits=8), dict(page=8)])
def test_shared_prefixes(heads, layout):
    rng = np.random.default_rng(3)
    #  many short answers to one document; members of one and of no token; a prefix of one token; members with many tokens of their own
    for new, own, groups in [([1] * 12, [3, 40, 1, 99, 8, 17, 64, 65, 5, 2, 31, 200], [(0, 12, 700)]),
                             ([1, 3, 0, 8, 1, 1, 2, 4], [10, 3, 5, 100, 1, 70, 2, 9], [(0, 4, 333), (4, 6, 1), (6, 8, 129)]),
                             ([60, 2, 1, 200, 1], [60, 80, 1, 210, 33], [(0, 3, 150), (3, 5, 90)]),
                             ([1, 1], [1, 1], [(0, 1, 50), (1, 2, 60)])]:
        length = [o + next(p for lo, hi, p in groups if lo <= b < hi) for b, o in enumerate(own)]
        _run(_case(rng, new, length, *heads, groups=groups, **layout))


@pytest.mark.parametrize("groups", [False, True])
@pytest.mark.parametrize("bits", [16, 8])
def test_more_sequences_than_the_plan_keeps_in_lds(groups, bits):
    rng = np.random.default_rng(20)
    length = rng.integers(9, 40, 700).tolist()
    new = [int(min(n, m - 8)) for n, m in zip(rng.integers(0, 4, 700), length)]
    share = [(7 * i, 7 * i + 7, int(rng.integers(0, 9))) for i in range(100)] if groups else ()
    _run(_case(rng, new, length, 4, 2, 64, page=8, bits=bits, groups=share))


@pytest.mark.parametrize("groups", [False, True])
def test_more_blocks_than_are_laid_end_to_end(groups):
    """One block to a workgroup: more blocks in all than the stretches' table has room for, more large ones than three rounds of
    workgroups; of both kinds, some longer than a workgroup's share."""
    rng = np.random.default_rng(21)
    length = rng.integers(9, 24, 2500).tolist()
    length[1200] = 900
    _run(_case(rng, [1] * 2500, length, 1, 1, 64, page=8, groups=[(5 * i, 5 * i + 5, i % 9) for i in range(500)] if groups else ()))
    new = rng.integers(17, 21, 160).tolist()
    length = [n + int(x) for n, x in zip(new, rng.integers(8, 50, 160))]
    new[77], length[77] = 3, 2000
    _run(_case(rng, new, length, 16, 16, 64, page=8, groups=[(8 * i, 8 * i + 8, 3 + i % 6) for i in range(20)] if groups else ()))
    new, length = new[:100], length[:100]
    _run(_case(rng, new, length, 8, 8, 128, page=8, bits=8, groups=[(10 * i, 10 * i + 10, 3 + i % 6) for i in range(10)] if groups else ()))


@pytest.mark.parametrize("layout", [dict(page=16), dict(page=8, bits=8), dict(page=0)])
@pytest.mark.parametrize("heads", [(8, 2, 128), (8, 2, 64)])
def test_short_pieces_of_one_and_of_two_tiles_of_rows_side_by_side(heads, layout):
    rng = np.random.default_rng(23)
    new = [1, 5, 6, 8, 8, 4, 1, 1, 7, 5, 0, 5, 9, 8, 2, 6] * 6
    length = [n + int(x) for n, x in zip(new, rng.integers(0, 300, len(new)))]
    length[20], length[50] = 4000, 9000
    _run(_case(rng, new, length, *heads, **layout))
    if layout["page"]:
        _run(_case(rng, new, [m + 70 for m in length], *heads, groups=[(0, 16, 70), (16, 90, 33), (90, 96, 64)], **layout))


def test_more_kv_heads_than_workgroups_at_once():
    rng = np.random.default_rng(22)
    _run(_case(rng, [1, 20, 2], [300, 70, 9], 300, 300, 128, page=16))
    _run(_case(rng, [1, 20], [100, 70], 1000, 1000, 64, page=0))


def test_prefixes_that_not_every_query_sees():
    """Members whose own queries lie inside the stated prefix, shorter members, an empty one, a first member without queries."""
    rng = np.random.default_rng(4)
    _run(_case(rng, [1, 30, 1, 2], [200, 100, 90, 130], 8, 2, 64, groups=[(0, 4, 90)]))
    _run(_case(rng, [1, 1, 1], [200, 1, 220], 8, 2, 64, groups=[(0, 3, 1)]))
    _run(_case(rng, [0, 1, 1, 0], [64, 300, 280, 64], 8, 2, 64, groups=[(0, 4, 64)]))


def test_rows_that_see_nothing():
    """No tokens in the cache; more new tokens than the cache holds (the first see none)."""
    rng = np.random.default_rng(5)
    c = _case(rng, [1, 10, 200, 3], [0, 4, 150, 3], 8, 2, 128)
    _, a = _run(c)
    assert (a.out[0] == 0).all() and a.lse[0].isneginf().all() and (a.out[1:7] == 0).all() and (a.out[11:61] == 0).all()


def test_strides_of_queries_and_outputs():
    import torch
    rng = np.random.default_rng(6)
    for new, length in (([1, 1, 4], [50, 700, 9]), ([300], [300])):
        c = _case(rng, new, length, 8, 2, 128)
        _, a = _run(c)
        whole = torch.full((1,), 0)
        plan, b = _device(c, strided=True)
        plan.run()
        b.run()
        torch.cuda.synchronize()
        n = sum(new)
        assert torch.equal(a.out[:n], b.out[:n]) and torch.equal(a.lse[:n], b.lse[:n])
        base = b.out._base
        assert (base[:, 0] == 7).all() and (base[:, -2:] == 7).all() and (base[:, :, 128:] == 7).all() and (base[n:] == 7).all()


@pytest.mark.parametrize("sign", [1.0, -1.0, 0.0])
def test_scales_of_any_sign(sign):
    rng = np.random.default_rng(7)

    def tweak(cache, q):
        cache.k_scale *= np.float32(sign)
        cache.v_scale *= np.float32(-sign)
    _run(_case(rng, [1, 150], [600, 190], 8, 2, 128, bits=8, tweak=tweak))


@pytest.mark.parametrize("n", [1, 100])
def test_keys_whose_logits_overflow(n):
    """Finite queries and keys whose product does not fit fp32 (-infinity): such keys take nothing from the others; very large
    differences of logits; a row whose first tiles are all of that kind."""
    rng = np.random.default_rng(8)

    def tweak(cache, q):
        q[..., 0] = 0x6904                       # 1e25
        cache.k[..., 0] = 0
        rows = cache.rows(0, 900)
        cache.k[rows[:500], :, 0] = 0xE904       # -1e25
        cache.k[rows[700:710], :, 0] = 0xE904
    c = _case(rng, [n], [900], 4, 2, 64, tweak=tweak, salient=0)
    with np.errstate(over="ignore"):
        out, lse, size, reach = _oracle(c)
    import torch
    plan, a = _device(c)
    plan.run()
    a.run()
    torch.cuda.synchronize()
    # the magnitudes that count are those of the keys that have weight: column 0 adds nothing there
    c2 = dict(c, q=c["q"].copy())
    c2["q"][..., 0] = 0
    reach = _oracle(c2)[3]
    _check(c, a, oracle=(out, lse, size, reach))


def test_large_logits_and_tiny_scales():
    rng = np.random.default_rng(9)
    _run(_case(rng, [1, 90], [700, 600], 4, 2, 64, scale=20.0))
    _run(_case(rng, [1, 90], [700, 600], 4, 2, 64, scale=1e-6))


def test_what_cannot_be_answered_is_nan_and_nothing_else():
    import torch
    rng = np.random.default_rng(10)
    c = _case(rng, [1, 2, 1, 140, 1], [100, 60, 90, 150, 70], 8, 2, 128)
    oracle = _oracle(c)
    c["cache"].table[0, 2] = c["cache"].n_rows // 16           # one past the pool
    c["cache"].table[3, 0] = -5
    c["length"] = [100, 60, -1, 150, 16 * c["cache"].table.shape[1] + 1]     # lengths that are none
    plan, a = _device(c)
    plan.run()
    a.run()
    torch.cuda.synchronize()
    bad = [0] + [3] + list(range(4, 144)) + [144]
    assert a.out[bad].isnan().all() and a.lse[bad].isnan().all()
    c["length"] = [100, 60, 90, 150, 70]
    _check(c, a, rows=[1, 2], oracle=oracle)


def test_bad_pages_of_a_shared_prefix_reach_its_group_only():
    import torch
    rng = np.random.default_rng(11)
    c = _case(rng, [1] * 6, [300, 310, 320, 200, 210, 220], 8, 2, 64, groups=[(0, 3, 256), (3, 6, 150)])
    oracle = _oracle(c)
    c["cache"].table[0, 3] = 2**31 - 1
    plan, a = _device(c)
    plan.run()
    a.run()
    torch.cuda.synchronize()
    assert a.out[:3].isnan().all() and a.lse[:3].isnan().all()
    _check(c, a, rows=[3, 4, 5], oracle=oracle)


def test_contiguous_rows_outside_the_cache_are_not_read():
    import torch
    rng = np.random.default_rng(12)
    c = _case(rng, [1, 1, 1], [100, 50, 30], 8, 2, 64, page=0)
    oracle = _oracle(c)
    plan, a = _device(c)
    plan.cu_cache.copy_(torch.tensor([0, 100, 150, 190], dtype=torch.int32))
    plan.kv_len.copy_(torch.tensor([100, 50, 31], dtype=torch.int32))       # the third would end behind the cache
    plan.run()
    a.run()
    torch.cuda.synchronize()
    assert a.out[2].isnan().all()
    _check(c, a, rows=[0, 1], oracle=oracle)


def test_a_plan_for_another_shape_or_none_gives_nan():
    import torch
    from paper_2502_02789_amd import binding as sp
    rng = np.random.default_rng(13)
    c = _case(rng, [1, 1], [100, 50], 8, 2, 64)
    plan, a = _device(c)
    a.run()                                       # no plan yet
    torch.cuda.synchronize()
    assert a.out.isnan().all() and a.lse.isnan().all()
    plan.run()
    a.args.n_rows -= 16                           # another cache
    a.out.zero_()
    a.run()
    torch.cuda.synchronize()
    assert a.out.isnan().all()
    a.args.n_rows += 16
    a.out.fill_(7)
    a.lse.fill_(7)
    a.run()
    torch.cuda.synchronize()
    _check(c, a)


def test_same_result_on_every_run_and_without_lse():
    import torch
    rng = np.random.default_rng(14)
    c = _case(rng, [1] * 5 + [150], [900, 5000, 30, 777, 64, 2000], 8, 2, 128, groups=[(0, 6, 30)])
    _, a = _run(c)
    first = a.out.clone()
    for _ in range(5):
        a.run()
        torch.cuda.synchronize()
        assert torch.equal(first, a.out)
    plan, b = _device(c, want_lse=False)
    plan.run()
    b.run()
    torch.cuda.synchronize()
    assert torch.equal(first, b.out)


def test_captured_steps_follow_lengths_and_tables():
    """Plan and attention in one graph: replayed with other lengths, groups and caches, eager work in between."""
    import torch
    rng = np.random.default_rng(15)
    lens = [[300, 280, 500], [260, 300, 900], [1000, 999, 257], [256, 256, 256]]
    c = _case(rng, [1, 2, 1], [max(x) for x in zip(*lens)], 8, 2, 64, groups=[(0, 3, 256)])
    plan, a = _device(c)
    plan.run()
    a.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.run()
        a.run()
    k = plan.cu_new.clone()
    for step, x in enumerate(lens + lens[:2]):
        plan.kv_len.copy_(torch.tensor(x, dtype=torch.int32))
        plan.prefix_len.fill_([256, 0, 100, 255][step % 4])
        a.out.fill_(7)
        a.lse.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        d = dict(c, length=x)
        _check(d, a)
        k = (k * 3 + 1) % 7
        torch.cuda.synchronize()


def test_two_layers_at_once_on_streams_of_their_own():
    import torch
    from paper_2502_02789_amd import device as dev
    rng = np.random.default_rng(16)
    c = _case(rng, [1] * 8, [2000 + 37 * i for i in range(8)], 8, 2, 128)
    plan, a = _device(c)
    where, kc, vc, _ = c["cache"].device()
    b = dev.Attender(plan, a._held[0], vc, kc, scale=c["scale"], workspace=torch.empty_like(plan.workspace))   # keys and values swapped
    plan.run()
    a.run()
    b.run()
    torch.cuda.synchronize()
    wa, wb = a.out.clone(), b.out.clone()
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(10):
        a.out.zero_()
        b.out.zero_()
        torch.cuda.synchronize()
        a.run(stream=sa)
        b.run(stream=sb)
        torch.cuda.synchronize()
        assert torch.equal(a.out[:8], wa[:8]) and torch.equal(b.out[:8], wb[:8])


def test_long_caches_offsets_beyond_32_bits():
    """The last pages of a pool whose byte offsets pass 2^32; keys beyond 65536."""
    import torch
    from paper_2502_02789_amd import device as dev
    pages, page, H, H_kv, d, m = 140000, 16, 8, 8, 128, 70001
    g = torch.Generator(device="cuda").manual_seed(1)
    kc = torch.empty((pages, page, H_kv, d), dtype=torch.bfloat16, device="cuda")
    vc = torch.empty_like(kc)
    need = -(-m // page)
    first = pages - need
    for x in (kc, vc):
        x[:first] = float("nan")
        x[first:] = torch.randn((need, page, H_kv, d), generator=g, device="cuda", dtype=torch.bfloat16)
    table = torch.randperm(need, generator=g, device="cuda").to(torch.int32).add_(first).view(1, need)
    q = torch.randn((2, H, d), generator=g, device="cuda").to(torch.bfloat16)
    plan = dev.AttendPlan(cc.cuda_ints([0, 2]), cc.cuda_ints([m]), kc, H=H, total_new=2, block_table=table.contiguous())
    a = dev.Attender(plan, q, kc, vc, scale=1 / math.sqrt(d), want_lse=True)
    plan.run()
    a.run()
    rows = table[0].long()
    k, v = kc[rows].view(-1, H_kv, d)[:m].double(), vc[rows].view(-1, H_kv, d)[:m].double()
    for h in range(H):
        s = q[:, h].double() @ k[:, h].t().contiguous() / math.sqrt(d)
        s[0, m - 1] = -math.inf
        w = torch.softmax(s, -1)
        want, size = w @ v[:, h], w @ v[:, h].abs()
        tol = size * (2.0 ** -8 + 2 * m * 2.0 ** -24 + 1e-4) * 1.01 + want.abs() * 2.0 ** -8
        assert ((a.out[:, h].double() - want).abs() <= tol).all()
        assert (a.lse[:, h].double() - torch.logsumexp(s, -1)).abs().max() < 1e-4 + m * 2.0 ** -24
