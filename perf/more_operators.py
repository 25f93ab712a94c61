"""Performance cases of the operators of a decoding step behind a kept prompt, whose cache is held in 4 bits.

The base model's cache of a long prompt, or of many requests, is held as OCP MXFP4: E2M1 codes, one E8M0 scale to 32 elements of a head.
A case is one pass through one of these, for one layer where a layer is meant:

  "store"   CacheAppender.run, CacheReader.run -- queries and keys rotated, keys and values quantised as they are written, and the new
            tokens' keys and values read back as bf16: what the layers that follow see of them, and what scoring takes
  "read"    CacheReader.run   -- tokens of the cache as bf16 keys and values: the kept ones of a prompt, or all of it
  "attend"  Attender.run      -- attention of the new tokens over the cache; sequences of a group share their first tokens
  "verify"  Verifier.run      -- drafted tokens against the target's probabilities from given random numbers, and the token behind them

The shapes are those of the repository's workloads (drafts shaped like Llama-3.x 1B and 8B, a base model with 64 query
heads, prompts of 1K to 128K tokens, batches of 64, a vocabulary of 128256) and odd sizes between.
"""
import math
import random

import torch

own = False  # False: the operators in plain form; True: through the framework

THETA = 5.0e5


def listed():
    return [
        # the look-ahead tokens of 24 requests, to be checked at once: the smallest append that is read back
        _store("store 24 of 1-8 tokens", b=24, lo=1, hi=8, past=1000, page=16, heads_first=True),
        # the base model's prefill of what was kept of a 128K prompt: original positions, far apart
        _store("store kept 6592 of 128K", lo=6592, hi=6592, H=64, page=64, heads_first=True, stretch=19.8),
        # the kept tokens' keys and values of a 32K prompt, out of the cache of the whole prompt
        _read("read kept 3200 of 32K", total_lo=32768, total_hi=32768, lo=3200, hi=3200, page=64, heads_first=True, chosen=True),
        # a full batch of ragged prompts of the small draft, read back for scoring
        _read("read batch 64 ragged 1b", b=64, total_lo=300, total_hi=3000, d=64, page=16),
        # the smallest request: one sequence, one token, a short context
        _attend("one token 1000", own_lo=1000, own_hi=1000, page=16, heads_first=True),
        # one decoding step of a full ragged batch
        _attend("decode batch 64", b=64, own_lo=1024, own_hi=4096, page=16, heads_first=True),
        # one decoding step of the base model behind the longest prompt
        _attend("decode 128K", own_lo=131072, own_hi=131072, H=64, page=64, heads_first=True),
        # three few-shot prompts, eight requests on each, up to eight look-ahead tokens checked at once
        _attend("look-ahead 24 share 8K", b=24, own_lo=100, own_hi=900, new_lo=1, new_hi=8, prefix=8003, groups=3, page=32),
        # the base model's prefill of what was kept of a 128K prompt, over its own quantised cache
        _attend("kept prompt 6592", own_lo=6592, own_hi=6592, new_lo=0, H=64, page=64, heads_first=True),
        # the smallest request: four drafted tokens of one sequence
        _verify("verify one of 4", lo=4, hi=4),
        # one step of a full batch, requests of all temperatures
        _verify("verify batch 64", b=64, lo=1, hi=8, temperature="mixed"),
        # tokens looked up in the prompt instead of drafted by a model: no draft probabilities, fp32 logits, an odd vocabulary
        _verify("verify 16 looked up", b=16, lo=0, hi=10, vocab=50257, bits=32, draft=False, temperature="warm"),
    ]


def _store(name=None, **kw):
    # lo..hi: new tokens per sequence; past: most tokens already cached; page 0: contiguous; stretch > 0: positions of kept tokens
    return _named(name, dict(kind="store", b=1, lo=1, hi=1, past=0, H=32, H_kv=8, d=128, page=0, heads_first=False, stretch=0.0), kw)


def _read(name=None, **kw):
    # total_lo..total_hi: tokens in the cache; chosen: lo..hi of them, ascending, else all
    return _named(name, dict(kind="read", b=1, total_lo=1, total_hi=1, lo=0, hi=0, H_kv=8, d=128, page=0, heads_first=False, chosen=False), kw)


def _attend(name=None, **kw):
    # own_lo..own_hi: keys per sequence behind the shared prefix; new_lo..new_hi: new tokens among them (new_lo 0: all of them are new)
    return _named(name, dict(kind="attend", b=1, own_lo=1, own_hi=1, new_lo=1, new_hi=1, prefix=0, groups=0, H=32, H_kv=8, d=128,
                             page=0, heads_first=False), kw)


def _verify(name=None, **kw):
    # lo..hi: drafted tokens per sequence; draft: the draft's logits are there; temperature: "one", "warm" (0.6 to 1.2) or "mixed" (some 0)
    return _named(name, dict(kind="verify", b=1, lo=1, hi=1, vocab=128256, bits=16, draft=True, temperature="one"), kw)


def _named(name, c, kw):
    c.update(kw)
    if name is not None:
        c["name"] = name
    return c


def _full(case):
    return {"store": _store, "read": _read, "attend": _attend, "verify": _verify}[case["kind"]](**case)


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case: batch, lengths and options over the whole ranges."""
    r = rng.random()
    if r < 0.2:
        b, hi = _log_int(rng, 1, 64), rng.choice([0, 1, 2, 4, 8, 10])
        b = min(b, 512 // (hi + 1))
        return _verify(b=b, lo=rng.randint(0, hi), hi=hi, vocab=rng.choice([128256, _log_int(rng, 1000, 128256), _log_int(rng, 1000, 128256)]),
                       bits=16 if b * (hi + 1) > 320 else rng.choice([16, 16, 32]), draft=rng.random() < 0.7,
                       temperature=rng.choice(["one", "warm", "mixed"]))
    H, H_kv = rng.choice([(32, 8), (32, 8), (64, 8), (8, 2), (128, 8), (24, 8), (16, 16)])
    opt = dict(H_kv=H_kv, d=rng.choice([64, 128, 128]), page=rng.choice([0, 8, 16, 16, 64]), heads_first=rng.random() < 0.5)
    if r < 0.35:
        b = _log_int(rng, 1, 64)
        hi = _log_int(rng, 1, max(1, 6592 * 64 * 128 // (b * max(H, 16) * opt["d"])))
        return _store(b=b, lo=rng.randint(1, hi), hi=hi, past=rng.choice([0, rng.randrange(1000)]), H=H,
                      stretch=rng.choice([0.0, rng.uniform(1.0, 20.0)]) if hi <= 6592 else 0.0, **opt)
    if r < 0.5:
        b = _log_int(rng, 1, 64)
        hi = _log_int(rng, 8, 100000 // (b * max(1, H_kv * opt["d"] // 512)))
        n = _log_int(rng, 1, hi)
        return _read(b=b, total_lo=rng.randint(1, hi), total_hi=hi, lo=rng.randint(0, n), hi=n, chosen=rng.random() < 0.5, **opt)
    opt["H"] = H
    if r < 0.65:  # whole prompts
        hi = _log_int(rng, 30, 5000)
        b = _log_int(rng, 1, 16)
        while b > 1 and b * hi * hi * H > 3000 * 3000 * 32 * 8:
            b -= 1
        return _attend(b=b, own_lo=rng.randint(max(1, hi // 4), hi), own_hi=hi, new_lo=0, **opt)
    if r < 0.7:  # pieces of prompts
        hi, new = _log_int(rng, 1000, 20000), _log_int(rng, 10, 600)
        return _attend(b=rng.randint(1, 4), own_lo=max(new, hi // 2), own_hi=hi, new_lo=rng.randint(1, new), new_hi=new, **opt)
    new = rng.choice([1, 1, 1, 2, 4, 8])
    if r < 0.88:  # decoding, nothing shared
        b = _log_int(rng, 1, 64)
        hi = _log_int(rng, 20, 131072 if b == 1 else min(65536, 200000 // b))
        return _attend(b=b, own_lo=rng.randint(8, hi), own_hi=hi, new_lo=1, new_hi=new, **opt)
    groups = rng.choice([1, 1, 2, 3])  # decoding with shared prefixes
    b = groups * _log_int(rng, 2, 64 // groups)
    own_hi = _log_int(rng, 20, 1000)
    opt["page"] = opt["page"] or 32
    return _attend(b=b, own_lo=rng.randint(8, own_hi), own_hi=own_hi, new_lo=1, new_hi=new, prefix=_log_int(rng, 100, 32768),
                   groups=groups, **opt)


def _lens(c):
    """Lengths of the batch, part of the case and the same for every seed: per sequence (new, read or drafted tokens, tokens of the cache
    with the new ones, tokens shared with the group)."""
    r = random.Random(repr(sorted((k, v) for k, v in c.items() if k != "name")))
    lens = []
    for b in range(c["b"]):
        if c["kind"] == "verify":
            n = r.randint(c["lo"], c["hi"])
            lens.append((n, 100 + n + 1, 0))
        elif c["kind"] == "store":
            n = r.randint(c["lo"], c["hi"])
            lens.append((n, n + r.randint(0, c["past"]), 0))
        elif c["kind"] == "read":
            m = r.randint(c["total_lo"], c["total_hi"])
            lens.append((min(m, r.randint(c["lo"], c["hi"])) if c["chosen"] else m, m, 0))
        else:
            o = r.randint(c["own_lo"], c["own_hi"])
            n = min(o, r.randint(c["new_lo"], c["new_hi"])) if c["new_lo"] else o
            shared = max(1, c["prefix"] - 37 * (b * c["groups"] // c["b"])) if c["groups"] else 0
            lens.append((n, shared + o, shared))
    return lens


def _group_starts(c):
    first = [b for b in range(c["b"]) if b == 0 or b * c["groups"] // c["b"] != (b - 1) * c["groups"] // c["b"]]
    return first + [c["b"]]


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _offsets(v):
    return torch.tensor([0] + v, dtype=torch.int64).cumsum(0).to(torch.int32).cuda()


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _inputs(c, seed):
    return _verify_inputs(c, seed) if c["kind"] == "verify" else _cache_inputs(c, seed)


def _cache_inputs(c, seed):
    """What a layer has in hand, made on the GPU from the seed: projections of unit variance, a cache that holds the earlier tokens
    (pages of all sequences shuffled over one pool), lengths and block table."""
    dev = torch.device("cuda")
    g = _generator(seed)
    lens, B, H_kv, d, page = _lens(c), c["b"], c["H_kv"], c["d"], c["page"]
    x = dict(c)
    new, total = [n for n, _, _ in lens], [m for _, m, _ in lens]
    T = sum(new)
    x.update(T=T, n_max=max(new), m_max=max(total), cu_new=_offsets(new), kv_len=_ints(total), past_len=_ints([m - n for n, m, _ in lens]))
    if page:
        shared_pages = [s // page for _, _, s in lens]  # whole pages of the prefix are the group's, the rest each member's own
        need = [-(-m // page) for m in total]
        starts = _group_starts(c) if c["kind"] == "attend" and c["groups"] else list(range(B + 1))
        used, table = 0, []
        n_pages = 1
        for lo, hi in zip(starts[:-1], starts[1:]):
            n_pages += shared_pages[lo] + sum(need[b] - shared_pages[lo] for b in range(lo, hi))
        order = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32).cpu().tolist()
        for lo, hi in zip(starts[:-1], starts[1:]):
            common = order[used:used + shared_pages[lo]]
            used += shared_pages[lo]
            for b in range(lo, hi):
                more = need[b] - shared_pages[lo]
                table.append(common + order[used:used + more] + [0] * (max(need) - need[b]))
                used += more
        x["table"], x["cu_cache"], n_rows = _ints(table), None, n_pages * page
    else:
        x["table"], x["cu_cache"], n_rows = None, _offsets(total), max(1, sum(total))
    if c["kind"] == "attend":
        H = c["H"]
        x["q"] = torch.randn((T, H, d), generator=g, device=dev, dtype=torch.float32).to(torch.bfloat16)
        # one key in fifty is aligned with the first query of its group of heads: such tokens get much of the weight
        some = torch.randperm(n_rows, generator=g, device=dev)[: max(1, n_rows // 50)]
    for name in ("k", "v"):
        z = torch.randn((n_rows, H_kv, d), generator=g, device=dev, dtype=torch.float32)
        if name == "k" and c["kind"] == "attend":
            z[some] += 0.4 * x["q"][0, :: H // H_kv].float()
        codes, scales = _quantised(z)
        x[name + "_codes"], x[name + "_scales"] = _laid_out(codes, c), _laid_out(scales, c)
    if page and c["kind"] == "attend" and c["groups"]:
        _copy_tails(x, lens, starts)
        x["cu_group"], x["prefix_len"] = _ints(starts), _ints([lens[b][2] for b in starts[:-1]])
    else:
        x["cu_group"] = x["prefix_len"] = None
    if c["kind"] == "store":
        # one projection's output holds queries, keys and values of a token side by side
        H = c["H"]
        qkv = torch.randn((T, H + 2 * H_kv, d), generator=g, device=dev, dtype=torch.float32).to(torch.bfloat16)
        x["q"], x["k"], x["v"] = qkv[:, :H], qkv[:, H:H + H_kv], qkv[:, H + H_kv:]
        x["pos"] = None
        if c["stretch"]:
            gaps = torch.randint(1, max(2, int(2 * c["stretch"])), (T,), generator=g, device=dev)
            x["pos"] = gaps.cumsum(0).to(torch.int32)
    if c["kind"] == "read":
        x["first"] = _ints([0] * B)
        x["index"] = None
        if c["chosen"]:
            picks = [torch.randperm(m, generator=g, device=dev)[:n].sort().values for n, m, _ in lens]
            x["index"] = torch.cat(picks).to(torch.int32)
    return x


def _laid_out(rows, c):
    """[rows, H_kv, n] -> the cache as [pages, page, H_kv, n] or [rows, H_kv, n], the heads outermost of a page where the case says so."""
    if c["page"]:
        z = rows.view(-1, c["page"], c["H_kv"], rows.shape[-1])
        return z.transpose(1, 2).contiguous().transpose(1, 2) if c["heads_first"] else z
    return rows.transpose(0, 1).contiguous().transpose(0, 1) if c["heads_first"] else rows


def _copy_tails(x, lens, starts):
    """The tokens of a prefix that do not fill a page lie in a page of each member's own: the same tokens in all of them."""
    page = x["page"]
    for lo, hi in zip(starts[:-1], starts[1:]):
        at, rest = lens[lo][2] // page, lens[lo][2] % page
        for pool in (x["k_codes"], x["v_codes"], x["k_scales"], x["v_scales"]):
            if rest and hi - lo > 1:
                pool[x["table"][lo + 1:hi, at].long(), :rest] = pool[x["table"][lo, at].long(), :rest].clone()


def _verify_inputs(c, seed):
    """Logits of a peaked distribution and of a draft that is near it, tokens sampled from the draft, and the random numbers."""
    dev = torch.device("cuda")
    g = _generator(seed)
    lens, B, V = _lens(c), c["b"], c["vocab"]
    n = [k for k, _, _ in lens]
    T, dtype = sum(n), torch.bfloat16 if c["bits"] == 16 else torch.float32
    x = dict(c)
    x.update(T=T, n_max=max(n), cu=_offsets(n), past_len=_ints([m - k - 1 for k, m, _ in lens]))
    z = 2.5 * torch.randn((T + B, V), generator=g, device=dev)
    # a few tokens of every row stand out, as in text
    peaks = torch.randint(0, V, (T + B, 4), generator=g, device=dev)
    z.scatter_add_(1, peaks, 7.0 + 2.0 * torch.randn((T + B, 4), generator=g, device=dev))
    temperature = {"one": torch.ones(B, device=dev), "warm": 0.6 + 0.6 * torch.rand(B, generator=g, device=dev),
                   "mixed": (torch.arange(B, device=dev) % 4) * 0.4}[c["temperature"]].float()
    seq = torch.searchsorted(x["cu"][1:].long(), torch.arange(T, device=dev), right=True)
    rows = torch.arange(T, device=dev) + seq
    near = z[rows] + 0.7 * torch.randn((T, V), generator=g, device=dev) if T else z[:0]
    # drawn from the draft's distribution at the sequence's temperature
    noise = -torch.log(-torch.log(torch.rand((T, V), generator=g, device=dev).clamp(1e-20, 1 - 1e-7)))
    x["target"], draft = z.to(dtype), near.to(dtype)
    x["tokens"] = (draft.float() + temperature[seq][:, None] * noise).argmax(dim=-1).to(torch.int32) if T else torch.zeros(0, dtype=torch.int32, device=dev)
    x["draft_logits"] = draft if c["draft"] else None
    x["temperature"] = None if c["temperature"] == "one" else temperature
    x["u"] = torch.rand(T, generator=g, device=dev)
    x["r"] = torch.rand(B, generator=g, device=dev)
    return x


def prepare(case, seed):
    c = _full(case)
    s = _inputs(c, seed)
    if own:
        from paper_2502_02789_amd import device as spd
        if c["kind"] == "verify":
            s["op"] = spd.Verifier(s["target"], s["tokens"], s["cu"], s["u"], s["r"], draft=s["draft_logits"], temperature=s["temperature"],
                                   past_len=s["past_len"], want_logprob=True)
            return s
        where = dict(block_table=s["table"], cu_cache=s["cu_cache"], k_block_scale=s["k_scales"], v_block_scale=s["v_scales"])
        k_cache, v_cache = s["k_codes"].view(torch.float4_e2m1fn_x2), s["v_codes"].view(torch.float4_e2m1fn_x2)
        if c["kind"] == "store":
            s["op"] = spd.CacheAppender(s["k"], s["v"], s["cu_new"], k_cache, v_cache, q=s["q"], cache_len=s["past_len"],
                                        pos=s["pos"], rope_theta=THETA, **where)
            s["back"] = spd.CacheReader(k_cache, v_cache, s["cu_new"], total=s["T"], first=s["past_len"], **where)
        elif c["kind"] == "read":
            s["op"] = spd.CacheReader(k_cache, v_cache, s["cu_new"], total=s["T"], first=s["first"], index=s["index"], **where)
        else:
            # the plan follows from the lengths alone: a step makes it once for all of a model's layers
            plan = spd.AttendPlan(s["cu_new"], s["kv_len"], k_cache, total_new=s["T"], H=c["H"], block_table=s["table"],
                                  cu_cache=s["cu_cache"], cu_group=s["cu_group"], prefix_len=s["prefix_len"])
            plan.run()
            s["op"] = spd.Attender(plan, s["q"], k_cache, v_cache, scale=1.0 / math.sqrt(c["d"]), k_block_scale=s["k_scales"],
                                   v_block_scale=s["v_scales"], want_lse=True)
    return s


def run(state):
    s = state
    if s["kind"] == "store":
        if not own:
            return _store_plain(s)
        q = s["op"].run()
        k, v = s["back"].run()
        return {"q": q, "k": k, "v": v}
    if s["kind"] == "read":
        k, v = s["op"].run() if own else _read_plain(s)
        return {"k": k, "v": v}
    if s["kind"] == "verify":
        if not own:
            return _verify_plain(s)
        op = s["op"]
        op.run()
        return {"accepted": op.n_accepted, "tokens": op.out_tokens, "logprob": op.logprob, "kept_len": op.kept_len}
    if own:
        out = s["op"].run()
        return {"out": out, "lse": s["op"].lse}
    return _attend_plain(s)


# ---------------------------------------------------------------- plain forms
def _quantised(z):
    """fp32 [..., d] -> E2M1 codes, two to a byte, uint8 [..., d/2], and E8M0 scales of 32 elements, uint8 [..., d/32]: the smallest power
    of two (2^-125 at least) whose seven-fold no magnitude exceeds; values over it, to the nearest code (even where two are as near)."""
    blocks = z.reshape(*z.shape[:-1], -1, 32)
    top = blocks.abs().amax(dim=-1)
    m, e = torch.frexp(top)  # top = m 2^e, 0.5 <= m < 1
    e = torch.where(8.0 * m <= 7.0, e - 3, e - 2).clamp(min=-125)
    y = blocks * torch.exp2(-e.float())[..., None]
    a = y.abs()
    code = (a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
    code = (code + 8 * torch.signbit(y)).to(torch.uint8).reshape(*z.shape[:-1], -1, 2)
    return code[..., 0] | code[..., 1] << 4, (e + 127).to(torch.uint8)


def _values(codes, scales):
    """The fp32 values that codes [..., d/2] and scales [..., d/32] stand for."""
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=codes.device)
    table = torch.cat([table, -table])
    z = torch.stack([table[(codes & 15).long()], table[(codes >> 4).long()]], dim=-1)
    z = z.reshape(*codes.shape[:-1], -1, 32) * torch.exp2(scales.float() - 127.0)[..., None]
    return z.reshape(*codes.shape[:-1], -1)


def _token_places(s):
    """Per flat row: its sequence, its number among the sequence's rows."""
    t = torch.arange(s["T"], device=s["cu_new"].device)
    seq = torch.searchsorted(s["cu_new"][1:], t.to(torch.int32), right=True)
    return seq, t - s["cu_new"].long()[seq]


def _at(s, seq, i):
    """Index of the cache's leading axes for token i of sequence seq."""
    if s["table"] is None:
        return (s["cu_cache"].long()[seq] + i,)
    return s["table"].long()[seq, i // s["page"]], i % s["page"]


def _store_plain(s):
    d = s["d"]
    seq, j = _token_places(s)
    i = s["past_len"].long()[seq] + j
    pos = i if s["pos"] is None else s["pos"]
    freq = THETA ** (-torch.arange(d // 2, device=pos.device, dtype=torch.float64) / (d // 2))
    angle = pos.double()[:, None, None] * freq  # far positions need 64 bits
    cos, sin = angle.cos().float(), angle.sin().float()

    def turned(z):
        lo, hi = z.float().split(d // 2, dim=-1)
        return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], dim=-1)

    at, out = _at(s, seq, i), {}
    for name, z in (("k", turned(s["k"])), ("v", s["v"].float())):
        codes, scales = _quantised(z)
        s[name + "_codes"][at], s[name + "_scales"][at] = codes, scales
        out[name] = _values(s[name + "_codes"][at], s[name + "_scales"][at]).to(torch.bfloat16)
    return {"q": turned(s["q"]).to(torch.bfloat16), **out}


def _read_plain(s):
    seq, j = _token_places(s)
    at = _at(s, seq, s["first"].long()[seq] + j if s["index"] is None else s["index"].long())
    return [_values(s[name + "_codes"][at], s[name + "_scales"][at]).to(torch.bfloat16) for name in ("k", "v")]


def _attend_plain(s):
    B, H, H_kv, d, N, M = s["b"], s["H"], s["H_kv"], s["d"], s["n_max"], s["m_max"]
    G, dev = H // H_kv, s["q"].device
    # keys and values of all sequences, padded to the longest
    i = torch.arange(M, device=dev).expand(B, M)
    i = torch.minimum(i, s["kv_len"].long()[:, None] - 1)
    at = _at(s, torch.arange(B, device=dev)[:, None], i)
    k, v = (_values(s[name + "_codes"][at], s[name + "_scales"][at]) for name in ("k", "v"))
    k, v = k.permute(0, 2, 3, 1).contiguous(), v.transpose(1, 2).contiguous()
    j = torch.arange(N, device=dev)
    t = (s["cu_new"].long()[:-1, None] + j).clamp(max=s["T"] - 1)
    q = s["q"].float()[t].view(B, N, H_kv, G, d).transpose(1, 2).reshape(B, H_kv, N * G, d)
    logits = torch.matmul(q, k).view(B, H_kv, N, G, M) * (1.0 / math.sqrt(d))
    visible = s["past_len"].long()[:, None] + j + 1
    hidden = torch.arange(M, device=dev) >= visible[:, :, None]                    # [B, N, M]
    logits = logits.masked_fill(hidden[:, None, :, None, :], -math.inf)
    top = logits.amax(dim=-1, keepdim=True)
    p = torch.exp(logits - top)
    total = p.sum(dim=-1, keepdim=True)
    out = torch.matmul(p.view(B, H_kv, N * G, M), v).view(B, H_kv, N, G, d) / total
    lse = (top + total.log()).squeeze(-1)
    seq, j = _token_places(s)
    return {"out": out.transpose(1, 2)[seq, j].reshape(s["T"], H, d).to(torch.bfloat16),
            "lse": lse.transpose(1, 2)[seq, j].reshape(s["T"], H)}


def _probabilities(logits, temperature):
    """softmax(logits / temperature) of each row in 64 bits; at temperature 0 all of it at the largest logit (the first of equal ones)."""
    z, t = logits.double(), temperature.double()[:, None]
    top = z.amax(dim=-1, keepdim=True)
    w = torch.exp((z - top) / torch.where(t > 0, t, torch.ones_like(t)))
    index = torch.arange(z.shape[1], device=z.device)
    first = torch.where(z == top, index, z.shape[1]).amin(dim=-1, keepdim=True)
    return torch.where(t > 0, w / w.sum(dim=-1, keepdim=True), (index == first).double())


def _verify_plain(s):
    B, V, T, n_max, cu, dev = s["b"], s["vocab"], s["T"], s["n_max"], s["cu"].long(), s["u"].device
    n, b = cu[1:] - cu[:-1], torch.arange(B, device=dev)
    temperature = torch.ones(B, device=dev) if s["temperature"] is None else s["temperature"]
    j = torch.arange(n_max + 1, device=dev)
    row = torch.minimum(cu[:-1, None] + j, cu[1:, None])      # of the drafted tokens; the last is nobody's where j = n
    there = j < n[:, None]
    of = torch.searchsorted(cu[1:], torch.arange(T, device=dev), right=True)  # sequence of a drafted token
    of_target = torch.searchsorted(cu[1:] + b + 1, torch.arange(T + B, device=dev), right=True)
    p = _probabilities(s["target"], temperature[of_target])
    token = s["tokens"].long()
    x = torch.cat([token, token.new_zeros(1)])[row.clamp(max=T)]  # [B, n_max + 1]
    if s["draft_logits"] is None:
        q = torch.zeros((T, V), dtype=torch.float64, device=dev).scatter_(1, token[:, None], 1.0)
    else:
        q = _probabilities(s["draft_logits"], temperature[of])
    q = torch.cat([q, q.new_zeros((1, V))])                   # behind the last drafted token nothing is taken off
    u = torch.cat([s["u"].double(), s["u"].new_ones(1).double()])
    flat = torch.where(there, row, T)
    px, qx = p[row + b[:, None], x], q[flat, x]
    accepted = (there & (u[flat] * qx < px)).long().cumprod(dim=1).sum(dim=1)
    last = cu[:-1] + b + accepted
    rest = (p[last] - q[torch.where(accepted < n, cu[:-1] + accepted, T)]).clamp(min=0)
    rest = torch.where(rest.sum(dim=-1, keepdim=True) > 0, rest, p[last])
    cum = rest.cumsum(dim=-1)
    drawn = (cum <= s["r"].double()[:, None] * cum[:, -1:]).sum(dim=-1)
    index = torch.arange(V, device=dev)
    drawn = torch.minimum(drawn, torch.where(rest > 0, index, 0).amax(dim=-1))
    tokens = torch.full((T + B,), -1, dtype=torch.int64, device=dev)
    taken = j < accepted[:, None]
    tokens[(row + b[:, None])[taken]] = x[taken]
    tokens[last] = drawn
    logprob = torch.where(tokens >= 0, p.gather(1, tokens.clamp(min=0)[:, None])[:, 0].log(), -math.inf)
    return {"accepted": accepted.to(torch.int32), "tokens": tokens.to(torch.int32), "logprob": logprob.float(),
            "kept_len": (s["past_len"] + 1 + accepted).to(torch.int32)}


# ---------------------------------------------------------------- work and definitions
def work(case):
    c = _full(case)
    lens = _lens(c)
    T = sum(n for n, _, _ in lens)
    if c["kind"] == "verify":
        rows = 2 * T + c["b"] if c["draft"] else T + c["b"]
        return {"bytes": rows * c["vocab"] * c["bits"] // 8 + 12 * T + 8 * c["b"] + 8 * (T + c["b"]), "flops": 4 * rows * c["vocab"]}
    H_kv, d = c["H_kv"], c["d"]
    row = d // 2 + d // 32  # bytes of a token's key or value of one head
    if c["kind"] == "store":
        return {"bytes": T * (4 * c["H"] * d + 2 * H_kv * (2 * d + row + 2 * d)) + 4 * T, "flops": 3 * T * d * (c["H"] + 3 * H_kv)}
    if c["kind"] == "read":
        return {"bytes": 2 * T * H_kv * (row + 2 * d) + 4 * T, "flops": 2 * T * H_kv * d}
    H = c["H"]
    shared = sum(lens[b][2] for b in _group_starts(c)[:-1]) if c["groups"] else 0
    keys = shared + sum(m - s for _, m, s in lens)
    seen = sum(n * (m - n) + n * (n + 1) // 2 for n, m, _ in lens)
    return {"bytes": 2 * keys * H_kv * row + T * H * (4 * d + 4), "flops": 4 * seen * H * d}


def _decoded(codes, scales):
    """Values in 64 bits, from the fields of the codes: sign, two bits of exponent (bias 1, 0: subnormal), one of mantissa."""
    z = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2).to(torch.int64)
    sign, e, m = 1 - 2 * (z >> 3), (z >> 1) & 3, z & 1
    y = torch.where(e > 0, torch.ldexp(1.0 + 0.5 * m.double(), e - 1), 0.5 * m.double()) * sign
    return torch.ldexp(y, (scales.long() - 127).repeat_interleave(32, dim=-1))


def _nearest(z):
    """What quantising and reading back makes of z in 64 bits, a block of 32 after the other."""
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=z.device)
    blocks = z.reshape(-1, 32)
    unit = torch.exp2(torch.ceil(torch.log2(blocks.abs().amax(dim=1, keepdim=True) / 7.0)).clamp(min=-125.0))
    y = blocks / unit
    hi = torch.searchsorted(grid, y.abs()).clamp(max=7)
    lo = (hi - 1).clamp(min=0)
    below, above = y.abs() - grid[lo], grid[hi] - y.abs()
    pick = torch.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)
    return (torch.copysign(grid[pick], y) * unit).reshape(z.shape)


def exact(case, seed):
    """The definitions in 64 bits, sequence by sequence."""
    c = _full(case)
    x = _inputs(c, seed)
    if c["kind"] == "verify":
        return _verify_exact(c, x)
    lens, H_kv, d, page = _lens(c), c["H_kv"], c["d"], c["page"]

    def rows_of(b, name):
        m = lens[b][1]
        codes, scales = x[name + "_codes"], x[name + "_scales"]
        if not page:
            first = sum(k for _, k, _ in lens[:b])
            return _decoded(codes[first:first + m], scales[first:first + m])
        pages = x["table"][b, :-(-m // page)].long()
        return _decoded(codes[pages].flatten(0, 1)[:m], scales[pages].flatten(0, 1)[:m])

    at = 0
    if c["kind"] == "read":
        out = {"k": [], "v": []}
        for b, (n, m, _) in enumerate(lens):
            for name in out:
                z = rows_of(b, name)
                out[name].append(z if x["index"] is None else z[x["index"][at:at + n].long()])
            at += n
        return {name: torch.cat(z) for name, z in out.items()}
    if c["kind"] == "store":
        half = d // 2
        pairs = torch.exp(torch.arange(half, device="cuda", dtype=torch.float64) * (-math.log(THETA) / half))
        p = torch.cat([torch.arange(m - n, m, device="cuda") for n, m, _ in lens]) if x["pos"] is None else x["pos"]
        w = torch.polar(torch.ones((x["T"], half), dtype=torch.float64, device="cuda"), p.double()[:, None] * pairs)[:, None]

        def turn(z):
            r = torch.complex(z[..., :half].double(), z[..., half:].double()) * w
            return torch.cat([r.real, r.imag], dim=-1)

        return {"q": turn(x["q"]), "k": _nearest(turn(x["k"])), "v": _nearest(x["v"].double())}
    H = c["H"]
    if sum(n * m for n, m, _ in lens) * H > 6e9:
        return None
    G = H // H_kv
    out = torch.zeros((x["T"], H, d), dtype=torch.float64, device="cuda")
    lse = torch.empty((x["T"], H), dtype=torch.float64, device="cuda")
    for b, (n, m, _) in enumerate(lens):
        keys, values = rows_of(b, "k"), rows_of(b, "v")
        for g in range(H_kv):
            q = x["q"][at:at + n, g * G:(g + 1) * G].double().reshape(n * G, d)
            s = torch.mm(q, keys[:, g].t().contiguous()).view(n, G, m) / math.sqrt(d)
            s.masked_fill_(torch.ones((n, m), dtype=torch.bool, device="cuda").triu(m - n + 1)[:, None], -math.inf)
            lse[at:at + n, g * G:(g + 1) * G] = torch.logsumexp(s, dim=-1)
            out[at:at + n, g * G:(g + 1) * G] = torch.mm(torch.softmax(s, dim=-1).view(n * G, m), values[:, g].contiguous()).view(n, G, d)
        at += n
    return {"out": out, "lse": lse}


def _verify_exact(c, x):
    V = c["vocab"]
    accepted, tokens, logprob, kept = [], [], [], []
    at = 0

    def log_p(logits, t):
        z = logits.double()
        if t == 0.0:
            z = torch.full_like(z, -math.inf)
            z[int((logits == logits.max()).nonzero()[0])] = 0.0
            return z
        return torch.log_softmax(z / t, dim=0)

    for b, (n, m, _) in enumerate(_lens(c)):
        t = 1.0 if x["temperature"] is None else float(x["temperature"][b])
        said, logs = [], []
        for j in range(n + 1):
            lp = log_p(x["target"][at + b + j], t)
            if j < n:
                token = int(x["tokens"][at + j])
                if x["draft_logits"] is None:
                    q = torch.zeros(V, dtype=torch.float64, device="cuda")
                    q[token] = 1.0
                else:
                    q = log_p(x["draft_logits"][at + j], t).exp()
                if float(x["u"][at + j]) * float(q[token]) < float(lp[token].exp()):
                    said.append(token)
                    logs.append(float(lp[token]))
                    continue
                w = torch.relu(lp.exp() - q)
                w = w if float(w.sum()) > 0.0 else lp.exp()
            else:
                w = lp.exp()
            cum = torch.cumsum(w, dim=0)
            k = int(torch.searchsorted(cum, float(x["r"][b]) * float(cum[-1]), right=True))
            k = min(k, int(w.nonzero().max()))
            said.append(k)
            logs.append(float(lp[k]))
            break
        accepted.append(len(said) - 1)
        kept.append(m - n - 1 + len(said))
        tokens += said + [-1] * (n + 1 - len(said))
        logprob += logs + [-math.inf] * (n + 1 - len(logs))
        at += n
    return {"accepted": _ints(accepted), "tokens": _ints(tokens), "logprob": torch.tensor(logprob, dtype=torch.float64, device="cuda"),
            "kept_len": _ints(kept)}
