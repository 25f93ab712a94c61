"""GPU: sp_attend with queries of zeros.  All weights are exactly one then, values are small whole numbers, so every sum is a whole number that fp32 holds:
the number of keys that a row met can be told from its lse, and a key that is met twice, missed or taken for another moves the sums."""
import numpy as np
import pytest

from oracle import cache_oracle as co
from tests import attend_batches as ab
from tests import cache_cases as cc

pytestmark = pytest.mark.gpu


def _counted(b, seed, values, head_major=False, wide=False):
    """The batch on the device: (plan, attender, sums that are wanted [T, H_kv, d], keys that a row sees [T])."""
    import torch
    from paper_2502_02789_amd import device as dev
    rng = np.random.default_rng(seed)
    cache = cc.Cache(rng, [m + (3 if b["page"] else 0) for m in b["length"]], b["H_kv"], b["d"], b["page"], b["bits"], groups=b["groups"])
    whole = values(rng, cache.v.shape).astype(np.float32)
    cache.v[:] = co.f32_to_e4m3_codes(whole) if b["bits"] == 8 else co.f32_to_bf16_bits(whole)
    if b["bits"] == 8:
        cache.v_scale[:] = 0.5       # (exact)
    cache.share(b["groups"])
    cache.spoil_unused(b["length"])
    v = cache.values()[1].astype(np.float32)      # (exact)
    T = sum(b["new"])
    sums, seen, t = np.zeros((T, b["H_kv"], b["d"]), np.float32), np.zeros(T, np.int64), 0
    for s, (n, m) in enumerate(zip(b["new"], b["length"])):
        if n == 0:
            continue
        seen[t:t + n] = np.clip(m - n + np.arange(n) + 1, 0, m)
        rows, before = cache.rows(s, m), max(0, m - n)
        first = v[rows[:before]].sum(0)
        sums[t + max(0, n - m):t + n] = first + np.cumsum(v[rows[before:]], axis=0)
        t += n
    where, kc, vc, scales = cache.device(head_major)
    group = {}
    if b["groups"]:
        group = dict(cu_group=cc.cuda_ints([g[0] for g in b["groups"]] + [b["groups"][-1][1]]), prefix_len=cc.cuda_ints([g[2] for g in b["groups"]]))
    plan = dev.AttendPlan(cc.cuda_ints(cc.offsets(b["new"])), cc.cuda_ints(b["length"]), kc, H=b["H"], total_new=T, **where, **group)
    q = torch.zeros((T, b["H"], b["d"]), dtype=torch.bfloat16, device="cuda")
    out = None
    if wide:        # queries of one row for all, outputs inside wider rows, head by head
        q = q[:1].expand(q.shape)
        out = torch.full((b["H"] + 1, T + 1, b["d"] + 8), 7.0, dtype=torch.bfloat16, device="cuda")[1:, 1:, 8:].transpose(0, 1)
    a = dev.Attender(plan, q, kc, vc, scale=co.softmax_scale(b["d"]), out=out, want_lse=True, **scales)
    a.out.fill_(7)
    a.lse.fill_(7)
    return plan, a, sums, seen


def _check(b, a, sums, seen):
    G = b["H"] // b["H_kv"]
    lse, out = a.lse.cpu().numpy().astype(np.float64), a.out.float().cpu().numpy().astype(np.float64)
    sums = np.repeat(sums, G, axis=1).astype(np.float64)
    assert seen.max() < 100000           # the lse of n and n + 1 keys differ by 1 / n, its own error is 2^-22 (1 + log n)
    some = seen > 0
    assert np.isneginf(lse[~some]).all() and (out[~some] == 0).all()
    met = np.rint(np.exp(lse[some]))
    wrong = np.argwhere(met != seen[some][:, None])
    assert len(wrong) == 0, f"row, head {wrong[0]}: {met[tuple(wrong[0])]:.0f} keys instead of {seen[some][wrong[0][0]]}"
    want = sums[some] / seen[some][:, None, None]
    # the quotient in fp32 (a reciprocal, a product: 2^-20 is ample), then rounded to bf16
    off = np.abs(out[some] - want) - np.abs(want) * (2.0 ** -8 + 2.0 ** -20)
    wrong = np.argwhere(off > 0)
    assert len(wrong) == 0, f"row, head, element {wrong[0]}: {out[some][tuple(wrong[0])]} instead of {want[tuple(wrong[0])]}"


@pytest.mark.parametrize("batch", ab.SHARED + ab.BLOCKS, ids=lambda b: b["name"])
def test_every_key_is_met_once(batch):
    import torch
    plan, a, sums, seen = _counted(batch, 5, lambda rng, shape: rng.integers(-8, 9, shape))
    plan.run()
    a.run()
    torch.cuda.synchronize()
    _check(batch, a, sums, seen)


@pytest.mark.parametrize("seed", range(48))
def test_every_key_of_any_batch_is_met_once(seed):
    import torch
    batch = ab.drawn(seed)
    plan, a, sums, seen = _counted(batch, seed, lambda rng, shape: rng.integers(-8, 9, shape), head_major=seed % 3 == 1, wide=seed % 2 == 1)
    plan.run()
    a.run()
    torch.cuda.synchronize()
    _check(batch, a, sums, seen)
    if seed % 2 == 1:
        whole = a.out._base
        assert (whole[0] == 7).all() and (whole[:, 0] == 7).all() and (whole[..., :8] == 7).all()


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("paged", [True, False])
def test_every_key_of_a_long_cache_is_met_once(paged, bits):
    """70001 keys at the end of a pool whose byte offsets pass 2^32; single tokens, two at once, and enough rows for a large block."""
    import torch
    from paper_2502_02789_amd import device as dev
    page, H_kv, d, m = 16, 8, 128, 70001
    need = -(-m // page)
    pages = (1 << 32) // (page * H_kv * d * (bits // 8)) + need
    g = torch.Generator(device="cuda").manual_seed(3)
    dtype = torch.bfloat16 if bits == 16 else torch.float8_e4m3fn
    kc = torch.full((pages, page, H_kv, d), 0x7F, dtype=torch.uint8, device="cuda") if bits == 8 else torch.full((pages, page, H_kv, d), float("nan"), dtype=dtype, device="cuda")
    vc = kc.clone()
    first = pages - need
    whole = torch.randint(-8, 9, (need, page, H_kv, d), generator=g, device="cuda").float()
    kc[first:] = torch.randn(whole.shape, generator=g, device="cuda").to(dtype).view(kc.dtype)
    vc[first:] = whole.to(dtype).view(kc.dtype)
    table = None
    if paged:
        table = torch.full((2, need), -1, dtype=torch.int32, device="cuda")
        table[1] = torch.randperm(need, generator=g, device="cuda").to(torch.int32) + first
        whole = whole[table[1].long() - first]
    add = torch.cat([torch.zeros((1, H_kv, d), device="cuda", dtype=torch.float64), whole.view(-1, H_kv, d)[:m].double().cumsum(0)]).cpu().numpy()
    for n in (1, 2, 40):
        cache = (kc, vc) if paged else (kc.view(-1, H_kv, d), vc.view(-1, H_kv, d))
        where = dict(block_table=table) if paged else dict(cu_cache=cc.cuda_ints([0, first * page, first * page + m]))
        plan = dev.AttendPlan(cc.cuda_ints([0, 0, n]), cc.cuda_ints([0, m]), cache[0], H=8, total_new=n, **where)
        a = dev.Attender(plan, torch.zeros((n, 8, d), dtype=torch.bfloat16, device="cuda"), *cache, scale=1.0, want_lse=True)
        plan.run()
        a.run()
        torch.cuda.synchronize()
        seen = m - n + 1 + np.arange(n)
        _check(dict(H=8, H_kv=8), a, add[seen], seen)
