"""GPU: the calls of a decoding step with drafted tokens in the order a server makes them, over a 4-bit cache: the last token and the drafted ones
appended, attention over the cache, logits, verification, and the next step behind what stands; and a 4-bit draft's cache read back and scored."""
import numpy as np
import pytest

from oracle import cache_oracle as co
from oracle import mxfp4_oracle as mx
from oracle import specprefill_oracle as orc
from oracle import verify_oracle as vo
from oracle.specprefill_oracle import bf16_bits_to_f64
from tests import cache_cases as cc
from tests import mxfp4_cases as mc
from tests import test_gpu_attend as attend_checks

pytestmark = pytest.mark.gpu

THETA, VOCAB = 500000.0, 301


class _Step:
    """One layer whose projections are rows of a table and whose logits are a product with its outputs; everything that a step does is on the device."""

    def __init__(self, heads, past, drafted, page, seed):
        import torch
        from paper_2502_02789_amd import device as dev
        self.H, self.H_kv, self.d = heads
        H, H_kv, d = heads
        self.rng = rng = np.random.default_rng(seed)
        B, n = len(past), drafted
        self.B, self.n, T = B, n, B * (n + 1)
        self.cache = mc.FourBitCache(rng, [p + 5 * (n + 1) for p in past], H_kv, d, page, lo=124, hi=128)
        self.cache.spoil_unused(past)
        self.where, self.kc, self.vc, self.scales = self.cache.device(True)
        self.table = cc.normal_bits(rng, (VOCAB, H + 2 * H_kv, d))
        self.table_d = dev.bf16_from_bits(self.table)
        self.head = torch.from_numpy(rng.standard_normal((H * d, VOCAB)).astype(np.float32) / 32).cuda()
        self.past = cc.cuda_ints(past)
        self.last = cc.cuda_ints(rng.integers(0, VOCAB, B))
        self.tokens = torch.zeros(B * n, dtype=torch.int32, device="cuda")
        self.u, self.r = torch.zeros(B * n, device="cuda"), torch.zeros(B, device="cuda")
        self.draft = torch.zeros((B * n, VOCAB), dtype=torch.bfloat16, device="cuda")
        self.cu_new, self.cu_draft = cc.cuda_ints(np.arange(B + 1) * (n + 1)), cc.cuda_ints(np.arange(B + 1) * n)
        self.rows = torch.empty((T, H + 2 * H_kv, d), dtype=torch.bfloat16, device="cuda")
        self.logits = torch.empty((T, VOCAB), dtype=torch.bfloat16, device="cuda")
        self.kv_len = self.past + (n + 1)
        x = self.rows
        self.append = dev.CacheAppender(x[:, H:H + H_kv], x[:, H + H_kv:], self.cu_new, self.kc, self.vc, q=x[:, :H], cache_len=self.past, rope_theta=THETA,
                                        **self.where, **self.scales)
        self.plan = dev.AttendPlan(self.cu_new, self.kv_len, self.kc, H=H, total_new=T, **self.where)
        self.attend = dev.Attender(self.plan, self.append.q_out, self.kc, self.vc, scale=co.softmax_scale(d), want_lse=True, **self.scales)
        self.verify = dev.Verifier(self.logits, self.tokens, self.cu_draft, self.u, self.r, draft=self.draft, past_len=self.past, want_logprob=True)

    def draw(self, k):
        """What the draft hands over for step k."""
        import torch
        g = torch.Generator(device="cuda")
        g.manual_seed(k)
        self.draft.copy_(torch.randn(self.draft.shape, generator=g, device="cuda"))
        self.tokens.copy_(torch.multinomial(self.draft.float().softmax(-1), 1, generator=g)[:, 0])
        self.u.copy_(0.4 * torch.rand(self.u.shape, generator=g, device="cuda"))
        self.r.copy_(torch.rand(self.r.shape, generator=g, device="cuda"))

    def step(self):
        import torch
        ids = torch.cat([self.last.view(self.B, 1), self.tokens.view(self.B, self.n)], dim=1).view(-1)
        self.rows.copy_(self.table_d[ids.long()])
        self.append.run()
        torch.add(self.past, self.n + 1, out=self.kv_len)
        self.plan.run()
        out = self.attend.run()
        self.logits.copy_(out.float().flatten(1) @ self.head)
        accepted, said = self.verify.run()
        at = torch.arange(self.B, device="cuda") * (self.n + 1) + accepted
        self.next = said[at]

    def go_on(self):
        self.last.copy_(self.next)
        self.past.copy_(self.verify.kept_len)


@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 4, 64)])
def test_steps_with_drafted_tokens(heads):
    import torch
    past = [300, 17, 64, 1]
    s = _Step(heads, past, 3, 16, seed=1)
    H, H_kv, d = heads
    freq, c, stood = co.rope_frequencies(THETA, d), s.cache, 0
    last = s.last.cpu().numpy()
    for k in range(4):
        s.draw(k)
        s.step()
        torch.cuda.synchronize()
        ids = np.concatenate([last[:, None], s.tokens.cpu().numpy().reshape(s.B, s.n)], axis=1).reshape(-1)
        x = s.table[ids]
        mx.append(x[:, :H], x[:, H:H + H_kv], x[:, H + H_kv:], s.cu_new.cpu().numpy(), past, None, freq, (c.k, c.k_blocks), (c.v, c.v_blocks), c.where())
        for got, want, name in ((mc.host_codes(s.kc), c.k, "keys"), (mc.host_codes(s.vc), c.v, "values")):
            assert (got != want).sum() <= 2, name
        c.k, c.v = mc.host_codes(s.kc), mc.host_codes(s.vc)
        c.k_blocks, c.v_blocks = mc.host_scales(s.scales["k_block_scale"]), mc.host_scales(s.scales["v_block_scale"])
        q = cc.host_bits(s.append.q_out, 16)
        attend_checks._check(dict(cache=c, q=q, new=[s.n + 1] * s.B, length=[p + s.n + 1 for p in past], scale=co.softmax_scale(d)), s.attend)
        want = vo.verify(s.logits.double().cpu().numpy(), s.tokens.cpu().numpy(), s.cu_draft.cpu().numpy(), s.u.double().cpu().numpy(),
                         s.r.double().cpu().numpy(), draft=s.draft.double().cpu().numpy(), past_len=past)
        assert s.verify.n_accepted.tolist() == want[0].tolist() and s.verify.out_tokens.tolist() == want[1].tolist()
        assert s.verify.kept_len.tolist() == want[3].tolist() == [p + 1 + a for p, a in zip(past, want[0])]
        stood += int(want[0].sum())
        s.go_on()
        past = want[3].tolist()
        last = s.last.cpu().numpy()
        assert (last >= 0).all()
    assert 0 < stood < 4 * s.B * s.n


def test_a_captured_step_replayed_is_the_eager_one():
    import torch
    s, e = (_Step((8, 2, 128), [300, 17, 64, 1], 3, 16, seed=2) for _ in range(2))
    s.draw(0)
    s.step()                       # (one-time set-up)
    torch.cuda.synchronize()
    s = _Step((8, 2, 128), [300, 17, 64, 1], 3, 16, seed=2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.step()
    s.past.copy_(e.past)
    for k in range(4):
        s.draw(k)
        e.draw(k)
        graph.replay()
        e.step()
        torch.cuda.synchronize()
        for a, b in ((s.kc.view(torch.uint8), e.kc.view(torch.uint8)), (s.attend.out, e.attend.out), (s.attend.lse, e.attend.lse),
                     (s.verify.out_tokens, e.verify.out_tokens), (s.verify.logprob, e.verify.logprob), (s.verify.kept_len, e.verify.kept_len)):
            assert torch.equal(a, b)
        s.go_on()
        e.go_on()


def test_a_4_bit_draft_cache_read_back_and_scored():
    """Prompts' keys in a 4-bit cache, read back as the bf16 rows that scoring takes: the scores are those of the codes' values."""
    import torch
    from paper_2502_02789_amd import device as dev
    rng = np.random.default_rng(3)
    lens, H, H_kv, d, N = [400, 33, 1, 700], 8, 2, 128, 4
    T, B = sum(lens), len(lens)
    cache = mc.FourBitCache(rng, lens, H_kv, d, 16)
    where, kc, vc, scales = cache.device(True)
    cu = cc.cuda_ints(cc.offsets(lens))
    k = dev.bf16_from_bits(cc.normal_bits(rng, (T, H_kv, d)))
    dev.CacheAppender(k, k, cu, kc, vc, rope_theta=THETA, **where, **scales).run()
    keys, none = dev.CacheReader(kc, None, cu, total=T, **where, k_block_scale=scales["k_block_scale"]).run()
    assert none is None
    q_bits = cc.normal_bits(rng, (1, B, N, H, d))
    scores = dev.Scorer(dev.bf16_from_bits(q_bits), [keys], cu, H_kv=H_kv, scale=co.softmax_scale(d), exclusive_device=False).run()
    torch.cuda.synchronize()
    codes, blocks = mc.host_codes(kc), mc.host_scales(scales["k_block_scale"])
    rows = np.concatenate([cache.rows(b, m) for b, m in enumerate(lens)])
    values = mx.values(codes[rows], blocks[rows])
    assert (bf16_bits_to_f64(cc.host_bits(keys, 16)) == values).all()
    for b, m in enumerate(lens):
        lo = cc.offsets(lens)[b]
        w, _ = orc.layer_attention(bf16_bits_to_f64(q_bits[0, b]), values[lo:lo + m], co.softmax_scale(d))
        want = w.max(axis=2).mean(axis=0)
        got = scores[lo:lo + m].double().cpu().numpy()
        assert (np.abs(got - want) <= 2e-3 * want).all()
