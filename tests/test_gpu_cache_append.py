"""GPU: sp_cache_append against the CPU oracle: the caches bit for bit (a handful of values may take the neighbouring
step where the device's and the host's fp64 cosine round to different fp32 values), rows outside untouched."""
import numpy as np
import pytest

from oracle import cache_oracle as co
from oracle.specprefill_oracle import bf16_bits_to_f64
from tests import cache_cases as cc

pytestmark = pytest.mark.gpu


def _run(rng, new, past, H, H_kv, d, page=0, bits=16, theta=5e5, freq=None, pos=None, with_q=True, in_place=False, room=None, spare=3,
         head_major=False, fused=True, cache=None, prepare=None):
    import torch
    from paper_2502_02789_amd import device as dev
    T = sum(new) + spare
    cache = cache or cc.Cache(rng, room or [n + p for n, p in zip(new, past)], H_kv, d, page, bits)
    qkv = cc.normal_bits(rng, (T, H + 2 * H_kv, d))
    if prepare:
        prepare(cache, qkv)
    cu = cc.offsets(new)
    where, kc, vc, scales = cache.device(head_major)
    x = dev.bf16_from_bits(qkv)
    q, k, v = x[:, :H], x[:, H:H + H_kv], x[:, H + H_kv:]
    if not fused:
        q, k, v = q.contiguous(), k.transpose(0, 1).contiguous().transpose(0, 1), v.contiguous()
    q_out = q if in_place else torch.full((T, H, d), 7.0, dtype=torch.bfloat16, device="cuda")
    a = dev.CacheAppender(k, v, cc.cuda_ints(cu), kc, vc, q=q if with_q else None, q_out=q_out if with_q else None,
                          cache_len=None if past is None else cc.cuda_ints(past), pos=None if pos is None else cc.cuda_ints(pos),
                          rope_theta=theta if freq is None else 0.0, inv_freq=None if freq is None else torch.from_numpy(freq).cuda(), **where, **scales)
    a.run()
    torch.cuda.synchronize()
    inv = freq if freq is not None else co.rope_frequencies(theta, d) if theta else None
    want_k, want_v = cache.k.copy(), cache.v.copy()
    want_q = co.append(qkv[:, :H] if with_q else None, qkv[:, H:H + H_kv], qkv[:, H + H_kv:], cu, past, pos, inv, want_k, want_v, cache.where(),
                       cache.k_scale, cache.v_scale)
    got_k, got_v = cc.host_bits(kc, bits), cc.host_bits(vc, bits)
    if bits == 8:   # S.1111.111 is NaN with either sign, and a NaN's sign means nothing
        for x in (got_k, got_v, want_k, want_v):
            x[x == 0xFF] = 0x7F
    assert (got_v == want_v).all(), "values"
    _near(got_k, want_k, bits, "keys")
    if with_q:
        got_q = cc.host_bits(q_out, 16)
        n = int(cu[-1])
        _near(got_q[:n], want_q[:n], 16, "queries")
        tail = qkv[n:, :H] if in_place else np.full_like(got_q[n:], 0x40E0)
        assert (got_q[n:] == tail).all(), "rows behind the last sequence"
    return cache, got_k


def _near(got, want, bits, what):
    differ = got != want
    assert differ.sum() <= 2 + want.size // 50000, f"{what}: {differ.sum()} of {want.size} differ"
    step = np.abs(got.astype(np.int32) - want.astype(np.int32))
    assert step.max(initial=0) <= 1, what


LAYOUTS = [dict(page=16), dict(page=8, bits=8), dict(), dict(bits=8), dict(page=64, head_major=True)]


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("heads", [(32, 8, 128), (8, 2, 64), (3, 1, 128), (32, 2, 64), (5, 5, 64)])
def test_ragged_batches(layout, heads):
    rng = np.random.default_rng(1)
    H, H_kv, d = heads
    _run(rng, [5, 0, 1, 17, 3, 0, 40], [0, 4, 31, 7, 8, 0, 100], H, H_kv, d, **layout)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("T", [1, 2, 511, 513, 1500, 5003])
def test_one_sequence_of_any_length(T, bits):
    _run(np.random.default_rng(T), [T], [3], 4, 2, 64, page=16, bits=bits, spare=0)


def test_many_sequences():
    rng = np.random.default_rng(2)
    _run(rng, [1] * 300, list(rng.integers(0, 40, 300)), 8, 8, 64, page=8)
    _run(rng, [int(x) for x in rng.integers(0, 3, 300)], list(rng.integers(0, 40, 300)), 2, 1, 128)


@pytest.mark.parametrize("bits", [16, 8])
def test_positions_far_apart_and_given_frequencies(bits):
    rng = np.random.default_rng(3)
    T = 200
    pos = np.concatenate([np.sort(rng.choice(131072, T, replace=False)), [5, 5, 5]])
    _run(rng, [T], [0], 8, 2, 128, page=16, bits=bits, pos=pos)
    pos[:4] = [2**31 - 1, 2**30 + 1, 0, 1]
    _run(rng, [T], [0], 8, 2, 64, bits=bits, pos=pos, freq=co.rope_frequencies(10000.0, 64) / np.linspace(1, 8, 32))


def test_no_rotation_no_queries_in_place_and_other_strides():
    rng = np.random.default_rng(4)
    _run(rng, [9, 30], [2, 0], 4, 4, 64, page=16, theta=0.0)
    _run(rng, [9, 30], [2, 0], 4, 4, 128, page=16, with_q=False)
    _run(rng, [9, 30], [2, 0], 16, 4, 128, page=16, fused=False, in_place=True)


def test_every_8_bit_code_and_what_lies_between():
    """Inputs at, between and beyond the format's values, both signs, NaN and infinities; a scale of zero; a negative one."""
    rng = np.random.default_rng(5)
    T = 256
    bits16 = (np.arange(T * 64, dtype=np.uint32) * 4 + 1).astype(np.uint16).reshape(T, 1, 64)

    def prepare(cache, qkv):
        cache.k_scale = np.array([1.0, 0.0, -0.5], np.float32)
        cache.v_scale = np.array([1.0, 0.37, 0.0], np.float32)
        qkv[:T, 3:6] = bits16
        qkv[:T, 6:] = bits16
    cache, _ = _run(rng, [T], [0], 3, 3, 64, page=16, bits=8, theta=0.0, prepare=prepare)


@pytest.mark.parametrize("page", [0, 16])
def test_tokens_without_room_and_bad_pages_write_nothing(page):
    rng = np.random.default_rng(6)
    cache = cc.Cache(rng, [20, 16, 40], 2, 64, page)
    if page:
        cache.table[0, 1] = -1
        cache.table[2, 0] = cache.n_rows // page
        cache.table[2, 1] = 2**31 - 1
    else:
        cache.cu_cache[:] = [0, 20, 36, 90]      # beyond the cache
    before = cache.k.copy()
    _, got = _run(rng, [18, 10, 60], [0, 9, 0], 4, 2, 64, page=page, cache=cache)
    assert (got != before).any()


def test_negative_cached_lengths_write_nothing_in_front():
    rng = np.random.default_rng(7)
    cache = cc.Cache(rng, [20, 20], 2, 64, 0)
    _run(rng, [6, 6], [-3, -6], 4, 2, 64, cache=cache, theta=0.0)


def test_tokens_in_front_of_the_first_sequence_write_nothing():
    import torch
    from paper_2502_02789_amd import device as dev
    k = torch.randn((8, 2, 64), device="cuda").to(torch.bfloat16)
    for where in (dict(cu_cache=cc.cuda_ints([0, 30])), dict(block_table=cc.cuda_ints([[0, 1]]))):
        kc = torch.full((30, 2, 64) if "cu_cache" in where else (2, 16, 2, 64), 3.0, dtype=torch.bfloat16, device="cuda")
        vc = kc.clone()
        dev.CacheAppender(k, k, cc.cuda_ints([5, 8]), kc, vc, cache_len=cc.cuda_ints([10]), **where).run()
        torch.cuda.synchronize()
        got = kc.view(-1, 2, 64)
        assert (got[10:13] == k[5:]).all() and (got[:10] == 3).all() and (got[13:] == 3).all()


def test_fills_what_scoring_an_unrotated_cache_makes_of_it():
    """A cache filled by the append gives, scored as it is, the scores of the unrotated cache with rope_theta: the same two-pass
    kernels (batches of unstated length) run in both cases, so bit for bit."""
    import torch
    from paper_2502_02789_amd import device as dev
    rng = np.random.default_rng(8)
    lens, H, H_kv, d, N, theta = [300, 77, 1], 8, 2, 64, 2, 500000.0
    T, B = sum(lens), len(lens)
    k_raw, q_raw = cc.normal_bits(rng, (T, H_kv, d)), cc.normal_bits(rng, (1, B, N, H, d))
    cu = cc.cuda_ints(cc.offsets(lens))
    q_pos = cc.cuda_ints([[m, m + 1] for m in lens])
    raw = dev.Scorer(dev.bf16_from_bits(q_raw), [dev.bf16_from_bits(k_raw)], cu, H_kv=H_kv, scale=0.125, rope_theta=theta, q_pos=q_pos, exclusive_device=False)
    want = raw.run().clone()
    k = dev.bf16_from_bits(k_raw)
    kc, vc = torch.zeros_like(k), torch.zeros_like(k)
    dev.CacheAppender(k, k, cu, kc, vc, rope_theta=theta, cu_cache=cu).run()
    # the queries' rotation through the same call: a token per query row, its keys into a cache that nobody reads
    flat = dev.bf16_from_bits(q_raw.reshape(B * N, H, d))
    bin_ = torch.zeros((B * N, H_kv, d), dtype=torch.bfloat16, device="cuda")
    q_rot = dev.CacheAppender(bin_.clone(), bin_.clone(), cc.cuda_ints([0, B * N]), bin_, bin_.clone(), q=flat, pos=q_pos.view(-1),
                              rope_theta=theta, cu_cache=cc.cuda_ints([0, B * N])).run()
    got = dev.Scorer(q_rot.view(1, B, N, H, d), [kc], cu, H_kv=H_kv, scale=0.125, exclusive_device=False).run()
    torch.cuda.synchronize()
    assert (vc == k).all() and (got == want).all()


def test_long_cache_offsets_beyond_32_bits():
    """Rows whose element offset passes 2^31 and whose byte offset passes 2^32: the last pages of a large pool."""
    import torch
    from paper_2502_02789_amd import device as dev
    pages, page, H_kv, d = 140000, 16, 8, 128
    kc = torch.zeros((pages, page, H_kv, d), dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros_like(kc)
    k = torch.randn((20, H_kv, d), device="cuda").to(torch.bfloat16)
    table = cc.cuda_ints([[pages - 1, 3]])
    dev.CacheAppender(k, k, cc.cuda_ints([0, 20]), kc, vc, block_table=table).run()
    torch.cuda.synchronize()
    assert (vc[pages - 1] == k[:16]).all() and (kc[3, :4] == k[16:]).all() and int((kc != 0).sum()) <= k.numel()
    assert float(kc.abs().sum(dtype=torch.float64)) == float(k.abs().sum(dtype=torch.float64))


def test_captured_call_follows_its_inputs():
    import torch
    from paper_2502_02789_amd import device as dev
    H_kv, d, page = 2, 64, 16
    k = torch.randn((8, H_kv, d), device="cuda").to(torch.bfloat16)
    kc = torch.zeros((9, page, H_kv, d), dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros_like(kc)
    table, past = cc.cuda_ints([[0, 1, 2, 3], [4, 5, 6, 7]]), cc.cuda_ints([0, 5])
    a = dev.CacheAppender(k, k, cc.cuda_ints([0, 5, 8]), kc, vc, cache_len=past, block_table=table)
    a.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.run()
    for step in range(4):
        past.copy_(torch.tensor([7 * step, 5 + 11 * step], dtype=torch.int32))
        k.copy_(torch.randn(k.shape, device="cuda"))
        kc.zero_()
        vc.zero_()
        graph.replay()
        torch.cuda.synchronize()
        want = torch.zeros_like(kc)
        for b, lo, hi in ((0, 0, 5), (1, 5, 8)):
            for t in range(lo, hi):
                i = int(past[b]) + t - lo
                want[int(table[b, i // page]), i % page] = k[t]
        assert (kc == want).all() and (vc == want).all()
