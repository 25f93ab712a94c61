"""Performance cases of the cache operators: filling a key/value cache, and attention that reads it.

Between its matrix products a model's layer, draft or base, does two things with the cache that the token-importance
path later scores: it appends the new tokens' keys and values, turned to their positions, and it attends.  A case is one
pass through one of the two, for one layer:

  "append"  CacheAppender.run -- queries and keys rotated, keys and values written behind what the cache holds
  "attend"  Attender.run      -- attention of the new tokens over the cache; sequences of a group share their first tokens

The shapes are those of the repository's workloads (drafts shaped like Llama-3.x 1B and 8B, a base model with 64 query
heads, prompts of 1K to 128K tokens, batches of 64) and odd sizes between.
"""
import math
import random

import torch

own = False  # False: the operators in plain form; True: through the framework

THETA = 5.0e5


def listed():
    return [
        # one decoding step of a full batch: one token per sequence behind caches of all lengths
        _append("append decode batch 64", b=64, lo=1, hi=1, past=1000, page=16),
        # a draft's prompt into an empty cache of 8-bit floats
        _append("append prompt 8K 8-bit", lo=8192, hi=8192, page=64, bits=8),
        # the base model's prefill of what was kept of a 128K prompt: original positions, far apart
        _append("append kept 6592 of 128K", lo=6592, hi=6592, H=64, stretch=19.8),
        # a full batch of ragged prompts of the small draft
        _append("append batch 64 ragged 1b", b=64, lo=200, hi=3000, past=77, d=64, page=16),
        # the smallest request: one sequence, one token, a short context
        _attend("one token 1000", own_lo=1000, own_hi=1000, page=16),
        # one decoding step of a full ragged batch
        _attend("decode batch 64", b=64, own_lo=1024, own_hi=4096, page=16),
        # one decoding step of the base model behind the longest prompt, 8-bit cache
        _attend("decode 128K 8-bit", own_lo=131072, own_hi=131072, H=64, page=64, bits=8),
        # 64 answers to one long document, computed together
        _attend("decode 64 share 32K", b=64, own_lo=40, own_hi=600, prefix=32768, groups=1, page=64),
        # three few-shot prompts, eight requests on each, up to eight look-ahead tokens checked at once, 8-bit cache
        _attend("look-ahead 24 share 8K", b=24, own_lo=100, own_hi=900, new_lo=1, new_hi=8, prefix=8003, groups=3, page=32, bits=8),
        # the base model's prefill of what was kept of a 128K prompt
        _attend("kept prompt 6592", own_lo=6592, own_hi=6592, new_lo=0, H=64),
        # a ragged batch of prompts of the small draft
        _attend("prompts batch 8 1b", b=8, own_lo=300, own_hi=3000, new_lo=0, d=64, page=16),
        # two requests whose prompts come in pieces: some hundred new tokens behind a long cache
        _attend("piece of a prompt 20K", b=2, own_lo=15000, own_hi=20000, new_lo=400, new_hi=600, page=16),
    ]


def _append(name=None, **kw):
    # lo..hi: new tokens per sequence; past: most tokens already cached; page 0: contiguous; stretch > 0: positions of kept tokens
    return _named(name, dict(kind="append", b=1, lo=1, hi=1, past=0, H=32, H_kv=8, d=128, page=0, bits=16, stretch=0.0), kw)


def _attend(name=None, **kw):
    # own_lo..own_hi: keys per sequence behind the shared prefix; new_lo..new_hi: new tokens among them (new_lo 0: all of them are new)
    return _named(name, dict(kind="attend", b=1, own_lo=1, own_hi=1, new_lo=1, new_hi=1, prefix=0, groups=0, H=32, H_kv=8, d=128,
                             page=0, bits=16), kw)


def _named(name, c, kw):
    c.update(kw)
    if name is not None:
        c["name"] = name
    return c


def _full(case):
    return (_append if case["kind"] == "append" else _attend)(**case)


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case: batch, lengths and options over the whole ranges."""
    H, H_kv = rng.choice([(32, 8), (32, 8), (64, 8), (8, 2), (128, 8), (24, 8), (16, 16)])
    opt = dict(H=H, H_kv=H_kv, d=rng.choice([64, 128, 128]), bits=8 if rng.random() < 0.3 else 16, page=rng.choice([0, 8, 16, 16, 64]))
    if rng.random() < 0.3:
        b = _log_int(rng, 1, 64)
        hi = _log_int(rng, 1, max(1, 100000 // (b * max(1, H * opt["d"] // 2048))))
        return _append(b=b, lo=rng.randint(1, hi), hi=hi, past=rng.choice([0, rng.randrange(1000)]),
                       stretch=rng.choice([0.0, rng.uniform(1.0, 20.0)]) if hi <= 6592 else 0.0, **opt)
    r = rng.random()
    if r < 0.3:  # whole prompts
        hi = _log_int(rng, 30, 5000)
        b = _log_int(rng, 1, 16)
        while b > 1 and b * hi * hi * H > 3000 * 3000 * 32 * 8:
            b -= 1
        return _attend(b=b, own_lo=rng.randint(max(1, hi // 4), hi), own_hi=hi, new_lo=0, **opt)
    if r < 0.45:  # pieces of prompts
        hi, new = _log_int(rng, 1000, 20000), _log_int(rng, 10, 600)
        return _attend(b=rng.randint(1, 4), own_lo=max(new, hi // 2), own_hi=hi, new_lo=rng.randint(1, new), new_hi=new, **opt)
    new = rng.choice([1, 1, 1, 2, 4, 8])
    if r < 0.7:  # decoding, nothing shared
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
    """Lengths of the batch, part of the case and the same for every seed: per sequence (new tokens, tokens of the cache with them,
    tokens shared with the group)."""
    r = random.Random(repr(sorted((k, v) for k, v in c.items() if k != "name")))
    lens = []
    for b in range(c["b"]):
        if c["kind"] == "append":
            n = r.randint(c["lo"], c["hi"])
            lens.append((n, n + r.randint(0, c["past"]), 0))
            continue
        o = r.randint(c["own_lo"], c["own_hi"])
        n = min(o, r.randint(c["new_lo"], c["new_hi"])) if c["new_lo"] else o
        shared = max(1, c["prefix"] - 37 * (b * c["groups"] // c["b"])) if c["groups"] else 0
        lens.append((n, shared + o, shared))
    return lens


def _group_starts(c):
    first = [b for b in range(c["b"]) if b == 0 or b * c["groups"] // c["b"] != (b - 1) * c["groups"] // c["b"]]
    return first + [c["b"]]


def _inputs(c, seed):
    """What a layer has in hand, made on the GPU from the seed: projections of unit variance, a cache that holds the earlier tokens
    (pages of all sequences shuffled over one pool), lengths and block table."""
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    lens, B, H, H_kv, d, page = _lens(c), c["b"], c["H"], c["H_kv"], c["d"], c["page"]
    x = dict(c)
    new, total = [n for n, _, _ in lens], [m for _, m, _ in lens]
    T = sum(new)

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device=dev)

    def offsets(v):
        return torch.tensor([0] + v, dtype=torch.int64).cumsum(0).to(torch.int32).to(dev)

    x.update(T=T, n_max=max(new), m_max=max(total), cu_new=offsets(new), kv_len=ints(total), past_len=ints([m - n for n, m, _ in lens]))
    if page:
        shared_pages = [s // page for _, _, s in lens]  # whole pages of the prefix are the group's, the rest each member's own
        need = [-(-m // page) for m in total]
        starts = _group_starts(c) if c["kind"] == "attend" and c["groups"] else list(range(B + 1))
        order, used, table = None, 0, []
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
        x["table"], x["cu_cache"], n_rows = ints(table), None, n_pages * page
    else:
        x["table"], x["cu_cache"], n_rows = None, offsets(total), sum(total)
    x["k_scale"] = x["v_scale"] = None
    for name in ("k", "v"):
        z = torch.randn((n_rows, H_kv, d), generator=g, device=dev, dtype=torch.bfloat16)
        if name == "k" and c["kind"] == "attend":
            # one key in fifty is aligned with the first query of its group of heads: such tokens get much of the weight
            x["q"] = torch.randn((T, H, d), generator=g, device=dev, dtype=torch.float32).to(torch.bfloat16)
            some = torch.randperm(n_rows, generator=g, device=dev)[: max(1, n_rows // 50)]
            z[some] += 0.4 * x["q"][0, :: H // H_kv]
        if c["bits"] == 8:
            sc = z.abs().amax(dim=(0, 2)).float() / 448.0
            z = (z.float() / sc[None, :, None]).to(torch.float8_e4m3fn).view(torch.uint8)
            x[name + "_scale"] = sc
        x[name + "_cache"] = z.view(-1, page, H_kv, d) if page else z
    if page and c["kind"] == "attend" and c["groups"]:
        _copy_tails(x, lens, starts)
        x["cu_group"], x["prefix_len"] = ints(starts), ints([lens[b][2] for b in starts[:-1]])
    else:
        x["cu_group"] = x["prefix_len"] = None
    if c["kind"] == "append":
        # one projection's output holds queries, keys and values of a token side by side
        qkv = torch.randn((T, H + 2 * H_kv, d), generator=g, device=dev, dtype=torch.float32).to(torch.bfloat16)
        x["q"], x["k"], x["v"] = qkv[:, :H], qkv[:, H:H + H_kv], qkv[:, H + H_kv:]
        x["pos"] = None
        if c["stretch"]:
            gaps = torch.randint(1, int(2 * c["stretch"]), (T,), generator=g, device=dev)
            x["pos"] = gaps.cumsum(0).to(torch.int32)
    return x


def _copy_tails(x, lens, starts):
    """The tokens of a prefix that do not fill a page lie in a page of each member's own: the same tokens in all of them."""
    page = x["page"]
    for lo, hi in zip(starts[:-1], starts[1:]):
        at, rest = lens[lo][2] // page, lens[lo][2] % page
        for pool in (x["k_cache"], x["v_cache"]):
            if rest and hi - lo > 1:
                pool[x["table"][lo + 1:hi, at].long(), :rest] = pool[x["table"][lo, at].long(), :rest].clone()


def prepare(case, seed):
    c = _full(case)
    s = _inputs(c, seed)
    if own:
        from paper_2502_02789_amd import device as spd
        if c["kind"] == "append":
            s["op"] = spd.CacheAppender(s["k"], s["v"], s["cu_new"], s["k_cache"], s["v_cache"], q=s["q"], cache_len=s["past_len"],
                                        pos=s["pos"], rope_theta=THETA, block_table=s["table"], cu_cache=s["cu_cache"],
                                        k_scale=s["k_scale"], v_scale=s["v_scale"])
        else:
            # the plan follows from the lengths alone: a step makes it once for all of a model's layers
            plan = spd.AttendPlan(s["cu_new"], s["kv_len"], s["k_cache"], total_new=s["T"], H=c["H"], block_table=s["table"],
                                  cu_cache=s["cu_cache"], cu_group=s["cu_group"], prefix_len=s["prefix_len"])
            plan.run()
            s["op"] = spd.Attender(plan, s["q"], s["k_cache"], s["v_cache"], scale=1.0 / math.sqrt(c["d"]), k_scale=s["k_scale"],
                                   v_scale=s["v_scale"], want_lse=True)
    return s


def run(state):
    s = state
    if s["kind"] == "append":
        q = s["op"].run() if own else _append_plain(s)
        as_values = (lambda z: z.view(torch.float8_e4m3fn)) if s["bits"] == 8 else (lambda z: z)
        return {"q": q, "k_cache": as_values(s["k_cache"]), "v_cache": as_values(s["v_cache"])}
    if own:
        out = s["op"].run()
        return {"out": out, "lse": s["op"].lse}
    return _attend_plain(s)


def _token_places(s):
    """Per new token: its sequence, its number among the sequence's new tokens."""
    t = torch.arange(s["T"], device=s["cu_new"].device)
    seq = torch.searchsorted(s["cu_new"][1:], t.to(torch.int32), right=True)
    return seq, t - s["cu_new"].long()[seq]


def _cache_rows(s, seq, i):
    """Row of the cache's flat token axis that holds token i of sequence seq."""
    if s["table"] is None:
        return s["cu_cache"].long()[seq] + i
    return s["table"].long()[seq, i // s["page"]] * s["page"] + i % s["page"]


def _append_plain(s):
    H_kv, d = s["H_kv"], s["d"]
    seq, j = _token_places(s)
    i = s["past_len"].long()[seq] + j
    pos = i if s["pos"] is None else s["pos"]
    freq = THETA ** (-torch.arange(d // 2, device=pos.device, dtype=torch.float64) / (d // 2))
    angle = pos.double()[:, None, None] * freq  # far positions need 64 bits
    cos, sin = angle.cos().float(), angle.sin().float()

    def turned(z):
        lo, hi = z.float().split(d // 2, dim=-1)
        return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], dim=-1)

    rows = _cache_rows(s, seq, i)
    for name, z in (("k", turned(s["k"])), ("v", s["v"].float())):
        cache = s[name + "_cache"].view(-1, H_kv, d)
        if s["bits"] == 8:
            cache[rows] = (z / s[name + "_scale"][:, None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
        else:
            cache[rows] = z.to(torch.bfloat16)
    return turned(s["q"]).to(torch.bfloat16)


def _attend_plain(s):
    B, H, H_kv, d, N, M = s["b"], s["H"], s["H_kv"], s["d"], s["n_max"], s["m_max"]
    G, dev = H // H_kv, s["q"].device
    # keys and values of all sequences, padded to the longest
    i = torch.arange(M, device=dev).expand(B, M)
    i = torch.minimum(i, s["kv_len"].long()[:, None] - 1)
    rows = _cache_rows(s, torch.arange(B, device=dev)[:, None], i)

    def padded(name):
        z = s[name + "_cache"].view(-1, H_kv, d)[rows]
        if s["bits"] == 8:
            return z.view(torch.float8_e4m3fn).float() * s[name + "_scale"][:, None]
        return z.float()

    k, v = padded("k").permute(0, 2, 3, 1).contiguous(), padded("v").transpose(1, 2).contiguous()
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


def work(case):
    c = _full(case)
    lens, H, H_kv, d, e = _lens(c), c["H"], c["H_kv"], c["d"], c["bits"] // 8
    T = sum(n for n, _, _ in lens)
    if c["kind"] == "append":
        return {"bytes": T * d * (2 * 2 * H + 2 * H_kv * (2 + e)) + 4 * T, "flops": 3 * T * d * (H + H_kv)}
    shared = sum(lens[b][2] for b in _group_starts(c)[:-1]) if c["groups"] else 0
    keys = shared + sum(m - s for _, m, s in lens)
    seen = sum(n * (m - n) + n * (n + 1) // 2 for n, m, _ in lens)
    return {"bytes": 2 * keys * H_kv * d * e + T * H * (4 * d + 4), "flops": 4 * seen * H * d}


def exact(case, seed):
    """The definitions in 64 bits, sequence by sequence."""
    c = _full(case)
    x = _inputs(c, seed)
    lens, H, H_kv, d, page = _lens(c), c["H"], c["H_kv"], c["d"], c["page"]
    flat = {}
    for name in ("k", "v"):
        z = x[name + "_cache"].view(-1, H_kv, d)
        flat[name] = z.view(torch.float8_e4m3fn).float().double() if c["bits"] == 8 else z.double()
    first, at, places = 0, 0, []
    for b, (n, m, _) in enumerate(lens):
        i = torch.arange(m, device="cuda")
        places.append(x["table"][b].long().repeat_interleave(page)[:m] * page + i % page if page else first + i)
        first += m
    if c["kind"] == "append":
        half = d // 2
        pairs = torch.exp(torch.arange(half, device="cuda", dtype=torch.float64) * (-math.log(THETA) / half))
        q_out = torch.empty((x["T"], H, d), dtype=torch.float64, device="cuda")
        for b, (n, m, _) in enumerate(lens):
            t = slice(at, at + n)
            p = torch.arange(m - n, m, device="cuda") if x["pos"] is None else x["pos"][t]
            w = torch.polar(torch.ones((n, half), dtype=torch.float64, device="cuda"), p.double()[:, None] * pairs)[:, None]

            def turn(z):
                r = torch.complex(z[..., :half].double(), z[..., half:].double()) * w
                return torch.cat([r.real, r.imag], dim=-1)

            q_out[t] = turn(x["q"][t])
            for name, z in (("k", turn(x["k"][t])), ("v", x["v"][t].double())):
                if c["bits"] == 8:
                    z = (z / x[name + "_scale"].double()[:, None]).clamp(-448.0, 448.0)
                flat[name][places[b][m - n:]] = z
            at += n
        return {"q": q_out, "k_cache": flat["k"].view(x["k_cache"].shape), "v_cache": flat["v"].view(x["v_cache"].shape)}
    if sum(n * m for n, m, _ in lens) * H > 6e9:
        return None
    G = H // H_kv
    out = torch.zeros((x["T"], H, d), dtype=torch.float64, device="cuda")
    lse = torch.empty((x["T"], H), dtype=torch.float64, device="cuda")
    for b, (n, m, _) in enumerate(lens):
        for g in range(H_kv):
            k, v = flat["k"][places[b], g], flat["v"][places[b], g]
            if c["bits"] == 8:
                k, v = k * x["k_scale"][g].double(), v * x["v_scale"][g].double()
            q = x["q"][at:at + n, g * G:(g + 1) * G].double().reshape(n * G, d)
            s = torch.mm(q, k.t().contiguous()).view(n, G, m) / math.sqrt(d)
            s.masked_fill_(torch.ones((n, m), dtype=torch.bool, device="cuda").triu(m - n + 1)[:, None], -math.inf)
            lse[at:at + n, g * G:(g + 1) * G] = torch.logsumexp(s, dim=-1)
            out[at:at + n, g * G:(g + 1) * G] = torch.mm(torch.softmax(s, dim=-1).view(n * G, m), v).view(n, G, d)
        at += n
    return {"out": out, "lse": lse}
