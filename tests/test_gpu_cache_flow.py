"""GPU: the calls in the order a server makes them for one layer: the draft's keys appended, scored, tokens selected and gathered, the
kept tokens' keys and values of the base model appended at their original positions, their prefill, and single-token steps behind it."""
import numpy as np
import pytest

from oracle import cache_oracle as co
from oracle.specprefill_oracle import bf16_bits_to_f64
from tests import cache_cases as cc
from tests import test_gpu_attend as attend_checks
from tests.test_gpu_cache_append import _near

pytestmark = pytest.mark.gpu

THETA = 500000.0


class _Prompts:
    """Prompts scored and cut down, everything up to the lists of kept tokens."""

    def __init__(self, lens, H, H_kv, d, page, seed):
        import torch
        from paper_2502_02789_amd import device as dev
        rng = np.random.default_rng(seed)
        self.lens, B, N = lens, len(lens), 4
        T = sum(lens)
        self.ids = rng.integers(0, 97, T).astype(np.int32)
        self.cu = cc.cuda_ints(cc.offsets(lens))
        draft = cc.Cache(rng, lens, H_kv, d, page)
        where, kc, vc, _ = draft.device()
        k = dev.bf16_from_bits(cc.normal_bits(rng, (T, H_kv, d)))
        q = dev.bf16_from_bits(cc.normal_bits(rng, (B * N, H, d)))
        q_pos = cc.cuda_ints([[m + i for i in range(N)] for m in lens])
        dev.CacheAppender(k, k, self.cu, kc, vc, rope_theta=THETA, **where).run()
        spare = torch.zeros((B * N, H_kv, d), dtype=torch.bfloat16, device="cuda")      # (keys of the look-ahead tokens: nobody reads them)
        all_rows = cc.cuda_ints([0, B * N])
        q_rot = dev.CacheAppender(spare.clone(), spare.clone(), all_rows, spare, spare.clone(), q=q, pos=q_pos.view(-1), rope_theta=THETA, cu_cache=all_rows).run()
        common = dict(H_kv=H_kv, scale=co.softmax_scale(d), exclusive_device=False, block_table=where["block_table"], page_size=page, total_tokens=T)
        self.scores = dev.Scorer(q_rot.view(1, B, N, H, d), [kc], self.cu, **common).run()
        # the same prompts out of a cache whose keys are turned by the scoring call
        plain = torch.zeros_like(kc)
        dev.CacheAppender(k, k, self.cu, plain, torch.zeros_like(kc), **where).run()
        self.scores_unrotated_cache = dev.Scorer(q.view(1, B, N, H, d), [plain], self.cu, rope_theta=THETA, q_pos=q_pos, **common).run()
        self.selector = dev.Selector(self.scores, self.cu, chunk=8, pool_window=5, keep_rate=0.3)
        self.selector.run()
        self.gather = dev.Gatherer(self.selector, token_ids=cc.cuda_ints(self.ids))
        self.gather.run()


@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 4, 64)])
@pytest.mark.parametrize("bits", [16, 8])
def test_prompts_scored_cut_down_prefilled_and_continued(heads, bits):
    import torch
    from paper_2502_02789_amd import device as dev
    H, H_kv, d = heads
    lens, page, steps = [400, 33, 1, 700], 16, 3
    B = len(lens)
    p = _Prompts(lens, H, H_kv, d, page, seed=1)
    torch.cuda.synchronize()
    assert (p.scores == p.scores_unrotated_cache).all()
    cu_keep, kept_ids, kept_pos = p.selector.cu_keep, p.gather.kept_ids, p.gather.kept_pos
    kept = cu_keep.cpu().numpy()
    assert all(0 < kept[b + 1] - kept[b] <= lens[b] for b in range(B)) and kept[-1] < sum(lens) // 2
    assert p.gather.decode_pos.cpu().tolist() == lens

    # the base model: a token's projections are a row of a table
    rng = np.random.default_rng(2)
    cap = int(kept_ids.numel())
    table = cc.normal_bits(rng, (97, H + 2 * H_kv, d))
    table_d = dev.bf16_from_bits(table)
    counts = np.diff(kept)
    base = cc.Cache(rng, [int(n) + steps for n in counts], H_kv, d, page, bits)
    base.spoil_unused([0] * B)
    where, kc, vc, scales = base.device()
    x = table_d[kept_ids.clamp(min=0).long()]             # (rows behind the last kept token: of no token)
    q = dev.CacheAppender(x[:, H:H + H_kv], x[:, H + H_kv:], cu_keep, kc, vc, q=x[:, :H], pos=kept_pos, rope_theta=THETA, **where, **scales).run()
    kv_len = cu_keep[1:] - cu_keep[:-1]
    plan = dev.AttendPlan(cu_keep, kv_len, kc, H=H, total_new=cap, block_table=where["block_table"])
    a = dev.Attender(plan, q, kc, vc, scale=co.softmax_scale(d), want_lse=True, **scales)
    a.out.fill_(7.0)
    a.lse.fill_(7.0)
    plan.run()
    a.run()
    torch.cuda.synchronize()

    freq, n = co.rope_frequencies(THETA, d), int(kept[-1])
    ids, pos = kept_ids.cpu().numpy()[:n], kept_pos.cpu().numpy()[:n]
    assert (ids == np.concatenate([p.ids[cc.offsets(lens)[b] + pos[kept[b]:kept[b + 1]]] for b in range(B)])).all()
    host = table[ids]

    def follow(rows, cu, past, pos):
        """The same tokens appended on the host; the device's cache and queries against it, then taken over for what follows."""
        want_q = co.append(rows[:, :H], rows[:, H:H + H_kv], rows[:, H + H_kv:], cu, past, pos, freq, base.k, base.v, base.where(), base.k_scale, base.v_scale)
        for got, want, what in ((cc.host_bits(kc, bits), base.k, "keys"), (cc.host_bits(vc, bits), base.v, "values")):
            _near(got, want, bits, what)
        base.k, base.v = cc.host_bits(kc, bits).copy(), cc.host_bits(vc, bits).copy()
        return want_q
    want_q = follow(host, kept, np.zeros(B, np.int32), pos)
    got_q = cc.host_bits(q, 16)
    _near(got_q[:n], want_q, 16, "queries")
    attend_checks._check(dict(cache=base, q=got_q, new=counts.tolist(), length=counts.tolist(), scale=co.softmax_scale(d)), a)

    # single tokens behind them, as one graph: positions go on from the whole prompt's length, cache indices from the kept tokens'
    new_ids = cc.cuda_ints([0] * B)
    row = torch.empty((B, H + 2 * H_kv, d), dtype=torch.bfloat16, device="cuda")
    past, at, length = kv_len.clone(), p.gather.decode_pos.clone(), kv_len + 1
    one = cc.cuda_ints(range(B + 1))
    append = dev.CacheAppender(row[:, H:H + H_kv], row[:, H + H_kv:], one, kc, vc, q=row[:, :H], cache_len=past, pos=at, rope_theta=THETA, **where, **scales)
    step_plan = dev.AttendPlan(one, length, kc, H=H, total_new=B, block_table=where["block_table"])
    answer = dev.Attender(step_plan, append.q_out, kc, vc, scale=co.softmax_scale(d), want_lse=True, **scales)

    def step():
        row.copy_(table_d[new_ids.long()])
        append.run()
        step_plan.run()
        answer.run()
    room = (kc.clone(), vc.clone())
    step()
    torch.cuda.synchronize()
    kc.copy_(room[0])
    vc.copy_(room[1])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(steps):
        new = rng.integers(0, 97, B).astype(np.int32)
        new_ids.copy_(torch.from_numpy(new))
        graph.replay()
        torch.cuda.synchronize()
        want_q = follow(table[new], np.arange(B + 1, dtype=np.int32), counts + i, np.array(lens, np.int32) + i)
        got_q = cc.host_bits(append.q_out, 16)
        _near(got_q, want_q, 16, "queries")
        attend_checks._check(dict(cache=base, q=got_q, new=[1] * B, length=(counts + i + 1).tolist(), scale=co.softmax_scale(d)), answer)
        past.add_(1)
        at.add_(1)
        length.add_(1)
        torch.cuda.synchronize()


def test_a_batch_that_continues_one_document():
    """Sequences whose tables begin with the same pages: the document appended once through the first, then a question of several tokens and
    single tokens each, against the same calls on copies without a group."""
    import torch
    from paper_2502_02789_amd import device as dev
    rng = np.random.default_rng(3)
    H, H_kv, d, page, prefix, B = 16, 4, 128, 16, 512, 6
    own = [5, 9, 1, 30, 2, 17]
    length = [prefix + n for n in own]
    T = sum(own)
    base = cc.Cache(rng, [m + 4 for m in length], H_kv, d, page, groups=[(0, B, prefix)])
    base.spoil_unused([0] * B)
    where, kc, vc, _ = base.device()
    doc = dev.bf16_from_bits(cc.normal_bits(rng, (prefix, 2 * H_kv, d)))
    dev.CacheAppender(doc[:, :H_kv], doc[:, H_kv:], cc.cuda_ints([0, prefix]), kc, vc, rope_theta=THETA, block_table=where["block_table"][:1].contiguous()).run()
    x = dev.bf16_from_bits(cc.normal_bits(rng, (T, H + 2 * H_kv, d)))
    cu = cc.cuda_ints(cc.offsets(own))
    q = dev.CacheAppender(x[:, H:H + H_kv], x[:, H + H_kv:], cu, kc, vc, q=x[:, :H], cache_len=cc.cuda_ints([prefix] * B), rope_theta=THETA, **where).run()
    base.k, base.v = cc.host_bits(kc, 16), cc.host_bits(vc, 16)
    c = dict(cache=base, q=cc.host_bits(q, 16), new=own, length=length, scale=co.softmax_scale(d), H=H, head_major=False)
    oracle = attend_checks._oracle(c)
    assert np.isfinite(bf16_bits_to_f64(base.k[base.rows(3, length[3])])).all()
    for groups in ([(0, B, prefix)], []):
        plan, a = attend_checks._device(dict(c, groups=groups))
        plan.run()
        a.run()
        torch.cuda.synchronize()
        attend_checks._check(c, a, oracle=oracle)


def test_device_classes_refuse_what_does_not_fit_together():
    import torch
    from paper_2502_02789_amd import device as dev
    kc = torch.zeros((4, 16, 2, 64), dtype=torch.bfloat16, device="cuda")
    k, q = torch.zeros((3, 2, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((3, 8, 64), dtype=torch.bfloat16, device="cuda")
    cu, table, one = cc.cuda_ints([0, 3]), cc.cuda_ints([[0, 1]]), torch.ones(2, device="cuda")
    good = dict(block_table=table)

    def append(k=k, v=k, cu=cu, kc=kc, vc=kc.clone(), **kw):
        return dev.CacheAppender(k, v, cu, kc, vc, **dict(good, **kw))
    append(q=q, cache_len=cc.cuda_ints([1]), rope_theta=1e4)
    for bad in (dict(k=k.float()), dict(v=k[:2]), dict(k=k[..., ::2]), dict(cu=cu.long()), dict(cache_len=cc.cuda_ints([1, 2])), dict(vc=kc[:2]),
                dict(block_table=table.long()), dict(block_table=None), dict(cu_cache=cu), dict(k_scale=one), dict(q=q[:, :, :32]), dict(q_out=q),
                dict(q=q, q_out=q.transpose(0, 1).contiguous().transpose(0, 1)), dict(pos=cc.cuda_ints([1, 2]), rope_theta=1e4),
                dict(inv_freq=torch.ones(32, device="cuda")), dict(kc=kc.float(), vc=kc.float()), dict(kc=kc.view(-1, 2, 64), vc=kc.view(-1, 2, 64))):
        with pytest.raises(ValueError):
            append(**bad)
    plan = dev.AttendPlan(cu, cc.cuda_ints([3]), kc, H=8, total_new=3, **good)
    dev.Attender(plan, q, kc, kc, scale=1.0)
    for bad in (dict(q=q[:2]), dict(q=q[:, :4]), dict(kc=kc[:2], vc=kc[:2]), dict(kc=kc.byte(), vc=kc.byte()), dict(vc=kc.transpose(1, 2).contiguous().transpose(1, 2)),
                dict(out=q.float()), dict(k_scale=one), dict(q=q.cpu())):
        x = dict(dict(q=q, kc=kc, vc=kc), **bad)
        with pytest.raises(ValueError):
            dev.Attender(plan, x.pop("q"), x.pop("kc"), x.pop("vc"), scale=1.0, **x)
    for bad in (dict(total_new=3, H=7), dict(total_new=3, H=8, block_table=cc.cuda_ints([[0], [1]]))):
        with pytest.raises((ValueError, dev.sp.SpError)):
            dev.AttendPlan(cu, cc.cuda_ints([3]), kc, **dict(good, **bad))


def test_steps_without_tokens():
    import torch
    from paper_2502_02789_amd import device as dev
    kc = torch.ones((4, 16, 2, 64), dtype=torch.bfloat16, device="cuda")
    none, cu, table = torch.zeros((0, 2, 64), dtype=torch.bfloat16, device="cuda"), cc.cuda_ints([0, 0]), cc.cuda_ints([[0, 1]])
    q = dev.CacheAppender(none, none, cu, kc, kc.clone(), q=none, rope_theta=1e4, block_table=table).run()
    plan = dev.AttendPlan(cu, cc.cuda_ints([20]), kc, H=2, total_new=0, block_table=table)
    plan.run()
    a = dev.Attender(plan, q, kc, kc, scale=1.0, want_lse=True)
    assert a.run().shape == (0, 2, 64)
    torch.cuda.synchronize()
    assert (kc == 1).all()
