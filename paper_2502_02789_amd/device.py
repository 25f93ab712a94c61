"""Device-memory plumbing around the binding: allocate outputs and workspaces with torch,
fill the argument structs, call the C entry points.  No arithmetic of the method happens here."""
from __future__ import annotations

from typing import List, Optional, Sequence

import numpy as np
import torch

from . import binding as sp


def bf16_from_bits(bits: np.ndarray, device="cuda") -> torch.Tensor:
    """numpy uint16 bit patterns -> torch.bfloat16 tensor on the device (bit-exact)."""
    t = torch.from_numpy(np.ascontiguousarray(bits).view(np.int16))
    return t.to(device).view(torch.bfloat16)


def bits_from_bf16(t: torch.Tensor) -> np.ndarray:
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


# The three configurations the paper compares (Sec. 4, list of evaluated variants), as settings
# of the same three calls: the plain variant scores with the last prompt token only and keeps
# single tokens by their un-smoothed scores; "full" adds pooling and chunk selection; "full_lah"
# adds the look-ahead queries.  (Window and chunk size are the synthetic workloads' choices.)
VARIANTS = {
    "raw": dict(n_queries=1, chunk=1, pool_window=1),
    "full": dict(n_queries=1, chunk=32, pool_window=13),
    "full_lah": dict(n_queries=8, chunk=32, pool_window=13),
}


class Scorer:
    """Holds the argument struct, outputs and workspace of one sp_score problem."""

    def __init__(self, q: torch.Tensor, k_layers: Sequence[torch.Tensor], cu_seqlens: torch.Tensor, *,
                 H_kv: int, scale: float, layer_reduce: int = sp.SP_LAYER_MAX,
                 n_valid: Optional[torch.Tensor] = None, want_lse: bool = False,
                 rope_theta: float = 0.0, q_pos: Optional[torch.Tensor] = None,
                 block_table: Optional[torch.Tensor] = None, page_size: int = 0, total_tokens: Optional[int] = None,
                 exclusive_device: bool = True, keep_workspace: bool = False, max_seqlen: int = 0,
                 k_scale: Optional[torch.Tensor] = None):
        """exclusive_device: promise that nothing else runs on the GPU during the call
        (SP_SCORE_EXCLUSIVE_DEVICE), which lets the workgroups of its single-pass kernels rely on one another.
        keep_workspace: from the second run() on, pass SP_SCORE_WORKSPACE_KEPT (this object owns
        its workspace, so the promise holds as long as run() is the only thing that writes it;
        anything else that does -- run(general=True), score_pool_select, a failed check() --
        makes the next run() start from a fresh workspace again)."""
        L, B, N, H, d = q.shape
        T = int(k_layers[0].shape[0]) if block_table is None else int(total_tokens)
        self.block_table = block_table
        dev = q.device
        self.q, self.k_layers, self.cu, self.n_valid, self.q_pos = q, list(k_layers), cu_seqlens, n_valid, q_pos
        self.scores = torch.empty(T, dtype=torch.float32, device=dev)
        self.lse = torch.empty((L, B, N, H), dtype=torch.float32, device=dev) if want_lse else None
        flags = sp.SP_SCORE_EXCLUSIVE_DEVICE if exclusive_device else 0
        probe = sp.make_score_args(q, self.k_layers, cu_seqlens, self.scores, H_kv=H_kv, scale=scale,
                                   layer_reduce=layer_reduce, n_valid=n_valid, lse=self.lse,
                                   rope_theta=rope_theta, q_pos=q_pos, T=T, block_table=block_table,
                                   page_size=page_size, flags=flags, max_seqlen=max_seqlen, k_scale=k_scale)
        need = sp.sp_score_workspace_bytes(probe)
        if need == 0:
            raise sp.SpError("sp_score_workspace_bytes", sp.SP_EINVAL)
        self.workspace = torch.empty(need, dtype=torch.uint8, device=dev)
        self.args = sp.make_score_args(q, self.k_layers, cu_seqlens, self.scores, H_kv=H_kv, scale=scale,
                                       layer_reduce=layer_reduce, n_valid=n_valid, lse=self.lse,
                                       workspace=self.workspace, rope_theta=rope_theta, q_pos=q_pos, T=T,
                                       block_table=block_table, page_size=page_size, flags=flags, max_seqlen=max_seqlen, k_scale=k_scale)

        self._base_flags, self._keep, self._kept = flags, keep_workspace, False

    def forget_workspace(self):
        """The workspace has been written by something other than sp_score."""
        self._kept = False

    def run(self, stream=None, general: bool = False) -> torch.Tensor:
        if general:
            self._kept = False
            sp.sp_score_general(self.args, stream)
            return self.scores
        self.args.flags = self._base_flags | (sp.SP_SCORE_WORKSPACE_KEPT if self._keep and self._kept else 0)
        sp.sp_score(self.args, stream)
        self._kept = True
        return self.scores

    def check(self, stream=None):
        """sp_score_check; raises SpError(SP_ETIMEOUT) if a bounded wait of the last run expired."""
        try:
            sp.sp_score_check(self.args, stream)
        except sp.SpError:
            self._kept = False
            raise


class Selector:
    """Outputs and workspace of one sp_pool_select (+ optional sp_gather) problem."""

    def __init__(self, scores: torch.Tensor, cu_seqlens: torch.Tensor, *, chunk: int, pool_window: int,
                 keep_rate: float, capacity: Optional[int] = None, want_chunk_scores: bool = False):
        dev = scores.device
        T = int(scores.numel())
        B = int(cu_seqlens.numel()) - 1
        cap = T if capacity is None else int(capacity)
        self.scores, self.cu = scores, cu_seqlens
        self.kept_idx = torch.full((max(cap, 1),), -1, dtype=torch.int32, device=dev)
        self.cu_keep = torch.zeros(B + 1, dtype=torch.int32, device=dev)
        self.chunk_scores = (torch.zeros(T // chunk + B, dtype=torch.float32, device=dev)
                             if want_chunk_scores else None)
        probe = sp.make_pool_select_args(scores, cu_seqlens, self.kept_idx, self.cu_keep, chunk=chunk,
                                         pool_window=pool_window, keep_rate=keep_rate, kept_capacity=cap)
        need = sp.sp_pool_select_workspace_bytes(probe)
        if need == 0:
            raise sp.SpError("sp_pool_select_workspace_bytes", sp.SP_EINVAL)
        self.workspace = torch.empty(need, dtype=torch.uint8, device=dev)
        self.args = sp.make_pool_select_args(scores, cu_seqlens, self.kept_idx, self.cu_keep, chunk=chunk,
                                             pool_window=pool_window, keep_rate=keep_rate,
                                             chunk_scores=self.chunk_scores, workspace=self.workspace,
                                             kept_capacity=cap)
        self.capacity = cap

    def run(self, stream=None):
        sp.sp_pool_select(self.args, stream)
        return self.kept_idx, self.cu_keep


def score_pool_select(scorer: Scorer, selector: Selector, stream=None):
    """One short prompt scored and selected in a single launch (sp_score_pool_select); the selector
    must have been built on scorer.scores and the same cu_seqlens."""
    scorer.forget_workspace()  # the logits pass through it
    sp.sp_score_pool_select(scorer.args, selector.args, stream)
    return scorer.scores, selector.kept_idx, selector.cu_keep


class Gatherer:
    def __init__(self, sel: Selector, *, token_ids: Optional[torch.Tensor] = None,
                 embed: Optional[torch.Tensor] = None):
        dev = sel.kept_idx.device
        cap = sel.capacity
        B = int(sel.cu.numel()) - 1
        self.kept_pos = torch.full((max(cap, 1),), -1, dtype=torch.int32, device=dev)
        self.kept_ids = torch.full((max(cap, 1),), -1, dtype=torch.int32, device=dev) if token_ids is not None else None
        self.decode_pos = torch.zeros(B, dtype=torch.int32, device=dev)
        self.out_embed = (torch.zeros((max(cap, 1), embed.shape[1]), dtype=torch.bfloat16, device=dev)
                          if embed is not None else None)
        self.token_ids, self.embed = token_ids, embed
        self.args = sp.make_gather_args(sel.cu, sel.cu_keep, sel.kept_idx, self.kept_pos, self.decode_pos,
                                        token_ids=token_ids, kept_ids=self.kept_ids, embed=embed,
                                        out_embed=self.out_embed, kept_capacity=cap)

    def run(self, stream=None):
        sp.sp_gather(self.args, stream)
        return self.kept_ids, self.kept_pos, self.decode_pos, self.out_embed


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _on_one_device(*tensors) -> torch.device:
    """The device that all of them (None aside) lie on."""
    devices = {t.device for t in tensors if t is not None}
    _need(len(devices) == 1 and next(iter(devices)).type == "cuda", "all tensors must lie on one GPU")
    return next(iter(devices))


def _head_dim(cache) -> int:
    return (2 if sp.is_4bit(cache) else 1) * int(cache.shape[-1])


def _check_block_scales(cache, scales, name: str):
    _need((scales is not None) == sp.is_4bit(cache), f"{name} belongs to a 4-bit cache (float4_e2m1fn_x2), and that needs it")
    if scales is None:
        return
    _need(scales.dtype in (torch.uint8, torch.float8_e8m0fnu) and cache.shape[-1] % 16 == 0 and
          scales.shape == cache.shape[:-1] + (cache.shape[-1] // 16,), f"{name}: uint8 or float8_e8m0fnu, the shape of the cache with d/32 for its last axis")
    _need(scales.stride(-1) == 1 and all(n == 1 or 16 * y == x for n, x, y in zip(cache.shape[:-1], cache.stride()[:-1], scales.stride()[:-1])),
          f"{name} must be laid out as the cache is: each stride a sixteenth of the cache's")


def _check_cache(k_cache, v_cache, block_table, cu_cache, B: int, scales=()):
    _need((block_table is None) != (cu_cache is None), "a cache is paged (block_table) or contiguous (cu_cache)")
    for c in (k_cache, v_cache):
        _need(c is None or sp.is_4bit(c) or c.dtype in (torch.bfloat16, torch.uint8, torch.float8_e4m3fn),
              "the cache holds bf16, E4M3 (uint8, float8_e4m3fn) or E2M1 codes (float4_e2m1fn_x2)")
    if block_table is not None:
        _need(block_table.dtype == torch.int32 and block_table.dim() == 2 and block_table.is_contiguous() and block_table.shape[0] == B,
              "block_table: contiguous int32 [B, blocks_per_seq]")
    else:
        _check_ints(cu_cache, B + 1, "cu_cache")
    for s in scales:
        if s is not None:
            _need(k_cache.element_size() == 1 and not sp.is_4bit(k_cache), "scales belong to 8-bit caches")
            _need(s.dtype == torch.float32 and s.is_contiguous() and s.numel() == k_cache.shape[-2], "scales: contiguous fp32 [H_kv]")


def _check_ints(t, n: int, name: str):
    _need(t.dtype == torch.int32 and t.is_contiguous() and t.numel() == n, f"{name}: contiguous int32 [{n}]")


def _check_rows(t, T: int, heads: Optional[int], d: int, name: str):
    _need(t.dtype == torch.bfloat16 and t.dim() == 3 and t.shape[0] == T and (heads is None or t.shape[1] == heads) and
          t.shape[2] == d and t.stride(2) == 1, f"{name}: bf16 [{T}, {'H' if heads is None else heads}, {d}], contiguous along the head dim")


class _OnDevice:
    """Calls go to the tensors' own device, whatever the current one is, and to its current stream unless one is given.  What a constructor
    allocates (the plan is cleared, so that none is taken for one) belongs to the stream that is current then: as with any tensor, a caller lets another
    stream wait for it before the first call there."""

    def _call(self, fn, args, stream):
        if torch.cuda.current_device() == self._device.index:
            fn(args, stream)
        else:
            with torch.cuda.device(self._device):
                fn(args, stream)


class CacheAppender(_OnDevice):
    """One sp_cache_append problem: new tokens' keys and values, rotated to their positions, into a cache; the queries
    rotated alike into q_out."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, cu_new: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, *,
                 q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                 cache_len: Optional[torch.Tensor] = None, pos: Optional[torch.Tensor] = None, rope_theta: float = 0.0,
                 inv_freq: Optional[torch.Tensor] = None, block_table: Optional[torch.Tensor] = None,
                 cu_cache: Optional[torch.Tensor] = None, k_scale: Optional[torch.Tensor] = None,
                 v_scale: Optional[torch.Tensor] = None, k_block_scale: Optional[torch.Tensor] = None,
                 v_block_scale: Optional[torch.Tensor] = None):
        """k, v: bf16 [T, H_kv, d] and q: bf16 [T, H, d], any token and head strides (slices of one projection's output);
        cu_new int32 [B+1] bounds the sequences' new tokens; cache_len int32 [B]: tokens cached before (None: none).
        k_cache, v_cache: [pages, page_size, H_kv, d] with block_table int32 [B, blocks_per_seq], or [rows, H_kv, d] with cu_cache
        int32 [B+1]; bf16, or 8-bit (uint8 or float8_e4m3fn) with k_scale, v_scale fp32 [H_kv], or 4-bit (float4_e2m1fn_x2
        [.., d/2]; see mxfp4_cache()) with k_block_scale, v_block_scale (uint8 or float8_e8m0fnu [.., d/32]), which are written too.
        pos: int32 [T] positions (the Gatherer's kept_pos, say), None: the index in the cache.  rope_theta or inv_freq (fp64
        [d/2]) asks for the rotation.  q_out: where the rotated queries go (a contiguous tensor, q itself allowed; default: a new one)."""
        T, B, d = int(k.shape[0]), int(cu_new.numel()) - 1, _head_dim(k_cache)
        H_kv = int(k_cache.shape[-2])
        self._device = _on_one_device(k, v, cu_new, k_cache, v_cache, q, q_out, cache_len, pos, inv_freq, block_table, cu_cache, k_scale, v_scale,
                                      k_block_scale, v_block_scale)
        _need(B >= 1, "cu_new: int32 [B+1]")
        _check_ints(cu_new, B + 1, "cu_new")
        _check_cache(k_cache, v_cache, block_table, cu_cache, B, (k_scale, v_scale))
        _check_block_scales(k_cache, k_block_scale, "k_block_scale")
        _check_block_scales(v_cache, v_block_scale, "v_block_scale")
        _check_rows(k, T, H_kv, d, "k")
        _check_rows(v, T, H_kv, d, "v")
        if q is not None:
            _check_rows(q, T, None, d, "q")
            if q_out is None:
                q_out = torch.empty(q.shape, dtype=torch.bfloat16, device=q.device)
            _check_rows(q_out, T, int(q.shape[1]), d, "q_out")
            _need(q_out.is_contiguous(), "q_out must be contiguous")
        else:
            _need(q_out is None, "q_out without q")
        if cache_len is not None:
            _check_ints(cache_len, B, "cache_len")
        if pos is not None:
            _need(pos.dtype == torch.int32 and pos.is_contiguous() and pos.numel() >= T, f"pos: contiguous int32 [{T}]")
        if inv_freq is not None:
            _need(inv_freq.dtype == torch.float64 and inv_freq.is_contiguous() and inv_freq.numel() == d // 2, f"inv_freq: fp64 [{d // 2}]")
        self.q_out = q_out
        self._held = (k, v, cu_new, k_cache, v_cache, q, cache_len, pos, inv_freq, block_table, cu_cache, k_scale, v_scale, k_block_scale,
                      v_block_scale)
        self.args = sp.make_cache_append_args(k, v, cu_new, k_cache, v_cache, q=q, q_out=q_out, cache_len=cache_len, pos=pos,
                                              rope_theta=rope_theta, inv_freq=inv_freq, block_table=block_table,
                                              cu_cache=cu_cache, k_scale=k_scale, v_scale=v_scale,
                                              k_block_scale=k_block_scale, v_block_scale=v_block_scale)

    def run(self, stream=None) -> Optional[torch.Tensor]:
        self._call(sp.sp_cache_append, self.args, stream)
        return self.q_out


def mxfp4_cache(rows, H_kv: int, d: int, *, device="cuda"):
    """An empty 4-bit cache (zeros) of keys or of values: float4_e2m1fn_x2 codes [.., H_kv, d/2] and float8_e8m0fnu scales [.., H_kv, d/32], `rows` the
    leading axes: (pages, page_size), or a number of rows.  The heads lie outermost in a page (or in all): the layout that attention reads fastest."""
    lead = (int(rows),) if isinstance(rows, int) else tuple(int(n) for n in rows)
    _need(d in (64, 128) and len(lead) in (1, 2), "rows: a number, or (pages, page_size); d: 64 or 128")

    def empty(n):
        return torch.zeros((*lead[:-1], H_kv, lead[-1], n), dtype=torch.uint8, device=device).transpose(-3, -2)

    return empty(d // 2).view(torch.float4_e2m1fn_x2), empty(d // 32).view(torch.float8_e8m0fnu)


class CacheReader(_OnDevice):
    """One sp_cache_read problem: tokens of a cache as bf16 keys and values [T, H_kv, d], for what takes no quantised cache or no block table
    (the Scorer, say, of a 4-bit one)."""

    def __init__(self, k_cache: torch.Tensor, v_cache: Optional[torch.Tensor], cu_rows: torch.Tensor, *, total: int,
                 first: Optional[torch.Tensor] = None, index: Optional[torch.Tensor] = None, block_table: Optional[torch.Tensor] = None,
                 cu_cache: Optional[torch.Tensor] = None, k_scale: Optional[torch.Tensor] = None, v_scale: Optional[torch.Tensor] = None,
                 k_block_scale: Optional[torch.Tensor] = None, v_block_scale: Optional[torch.Tensor] = None,
                 k_out: Optional[torch.Tensor] = None, v_out: Optional[torch.Tensor] = None):
        """Rows cu_rows[b] .. cu_rows[b+1]-1 (int32 [B+1], at most `total` in all) are tokens of sequence b: those from first[b] on (int32 [B],
        None: 0), or first[b] + index[t] (int32 [total]: the Gatherer's kept_pos, say).  The cache as the CacheAppender takes it;
        v_cache None: keys only.  k_out, v_out: bf16 [total, H_kv, d], any token and head strides (default: new ones)."""
        B, H_kv, d, T = int(cu_rows.numel()) - 1, int(k_cache.shape[-2]), _head_dim(k_cache), int(total)
        self._device = _on_one_device(k_cache, v_cache, cu_rows, first, index, block_table, cu_cache, k_scale, v_scale, k_block_scale,
                                      v_block_scale, k_out, v_out)
        _need(B >= 1, "cu_rows: int32 [B+1]")
        _check_ints(cu_rows, B + 1, "cu_rows")
        _check_cache(k_cache, v_cache, block_table, cu_cache, B, (k_scale, v_scale))
        _check_block_scales(k_cache, k_block_scale, "k_block_scale")
        if v_cache is not None:
            _check_block_scales(v_cache, v_block_scale, "v_block_scale")
        else:
            _need(v_scale is None and v_block_scale is None and v_out is None, "values without v_cache")
        if first is not None:
            _check_ints(first, B, "first")
        if index is not None:
            _need(index.dtype == torch.int32 and index.is_contiguous() and index.numel() >= T, f"index: contiguous int32 [{T}]")
        if k_out is None:
            k_out = torch.empty((T, H_kv, d), dtype=torch.bfloat16, device=self._device)
        if v_out is None and v_cache is not None:
            v_out = torch.empty((T, H_kv, d), dtype=torch.bfloat16, device=self._device)
        _check_rows(k_out, T, H_kv, d, "k_out")
        if v_out is not None:
            _check_rows(v_out, T, H_kv, d, "v_out")
        self.k_out, self.v_out = k_out, v_out
        self._held = (k_cache, v_cache, cu_rows, first, index, block_table, cu_cache, k_scale, v_scale, k_block_scale, v_block_scale)
        self.args = sp.make_cache_read_args(k_cache, v_cache, cu_rows, k_out, v_out, first=first, index=index, block_table=block_table,
                                            cu_cache=cu_cache, k_scale=k_scale, v_scale=v_scale, k_block_scale=k_block_scale,
                                            v_block_scale=v_block_scale)

    def run(self, stream=None):
        self._call(sp.sp_cache_read, self.args, stream)
        return self.k_out, self.v_out


class AttendPlan(_OnDevice):
    """The plan of one step's attention (sp_attend_plan) and the workspace that its layers use one after the other.  run() after every
    change of cu_new, kv_len, cu_group or prefix_len."""

    def __init__(self, cu_new: torch.Tensor, kv_len: torch.Tensor, k_cache: torch.Tensor, *, H: int, total_new: int,
                 block_table: Optional[torch.Tensor] = None, cu_cache: Optional[torch.Tensor] = None,
                 cu_group: Optional[torch.Tensor] = None, prefix_len: Optional[torch.Tensor] = None):
        """kv_len int32 [B]: tokens in the cache, the new ones included; total_new: rows of the queries; k_cache: any layer's
        (for shape and type).  cu_group int32 [n_groups+1], prefix_len int32 [n_groups]: sequences cu_group[g] .. cu_group[g+1]-1
        hold the same first prefix_len[g] tokens."""
        B = int(cu_new.numel()) - 1
        self._device = _on_one_device(cu_new, kv_len, k_cache, block_table, cu_cache, cu_group, prefix_len)
        _need(B >= 1, "cu_new: int32 [B+1]")
        _check_ints(cu_new, B + 1, "cu_new")
        _check_ints(kv_len, B, "kv_len")
        _check_cache(k_cache, None, block_table, cu_cache, B)
        _need((cu_group is None) == (prefix_len is None), "cu_group and prefix_len go together")
        if cu_group is not None:
            _check_ints(cu_group, int(cu_group.numel()), "cu_group")
            _check_ints(prefix_len, int(cu_group.numel()) - 1, "prefix_len")
        self.cu_new, self.kv_len, self.block_table, self.cu_cache = cu_new, kv_len, block_table, cu_cache
        self.cu_group, self.prefix_len, self.H, self.total_new = cu_group, prefix_len, int(H), int(total_new)
        self.shape, self.bytes, self.four_bits = k_cache.shape, k_cache.element_size(), sp.is_4bit(k_cache)
        kw = dict(H=H, total_new=total_new, block_table=block_table, cu_cache=cu_cache, cu_group=cu_group, prefix_len=prefix_len)
        probe = sp.make_attend_plan_args(cu_new, kv_len, k_cache, **kw)
        need = sp.sp_attend_plan_bytes(probe)
        if need == 0:
            raise sp.SpError("sp_attend_plan_bytes", sp.SP_EINVAL)
        self.plan = torch.zeros(need, dtype=torch.uint8, device=self._device)
        self.workspace = torch.empty(sp.sp_attend_workspace_bytes(probe), dtype=torch.uint8, device=self._device)
        self.args = sp.make_attend_plan_args(cu_new, kv_len, k_cache, plan=self.plan, **kw)

    def run(self, stream=None) -> None:
        self._call(sp.sp_attend_plan, self.args, stream)


class Attender(_OnDevice):
    """One layer's sp_attend: out bf16 [T, H, d] (and lse fp32 [T, H]) of queries q over the cache, by a plan."""

    def __init__(self, plan: AttendPlan, q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, *, scale: float,
                 k_scale: Optional[torch.Tensor] = None, v_scale: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                 want_lse: bool = False, workspace: Optional[torch.Tensor] = None, k_block_scale: Optional[torch.Tensor] = None,
                 v_block_scale: Optional[torch.Tensor] = None):
        """k_scale, v_scale, k_block_scale, v_block_scale: as the CacheAppender takes them.  workspace: uint8 of plan.workspace's size, for layers that
        run at the same time (default: the plan's)."""
        self._device = _on_one_device(plan.plan, q, k_cache, v_cache, k_scale, v_scale, out, workspace, k_block_scale, v_block_scale)
        d = _head_dim(k_cache)
        _check_cache(k_cache, v_cache, plan.block_table, plan.cu_cache, int(plan.cu_new.numel()) - 1, (k_scale, v_scale))
        _check_block_scales(k_cache, k_block_scale, "k_block_scale")
        _check_block_scales(v_cache, v_block_scale, "v_block_scale")
        _need(k_cache.shape == plan.shape and k_cache.element_size() == plan.bytes and sp.is_4bit(k_cache) == plan.four_bits, "the cache must have the shape and type that the plan was made for")
        _check_rows(q, plan.total_new, plan.H, d, "q")
        if out is None:
            out = torch.empty(q.shape, dtype=torch.bfloat16, device=q.device)
        _check_rows(out, plan.total_new, plan.H, d, "out")
        self.plan, self.out = plan, out
        self.lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device) if want_lse else None
        self.workspace = plan.workspace if workspace is None else workspace
        self._held = (q, k_cache, v_cache, k_scale, v_scale, k_block_scale, v_block_scale)
        self.args = sp.add_attend_args(plan.args, q, k_cache, v_cache, out, scale=scale, block_table=plan.block_table,
                                       cu_cache=plan.cu_cache, k_scale=k_scale, v_scale=v_scale, k_block_scale=k_block_scale,
                                       v_block_scale=v_block_scale, lse=self.lse, workspace=self.workspace)

    def run(self, stream=None) -> torch.Tensor:
        self._call(sp.sp_attend, self.args, stream)
        return self.out


class Verifier(_OnDevice):
    """One sp_verify problem: which drafted tokens stand against the target's probabilities, and the token behind them."""

    def __init__(self, target: torch.Tensor, tokens: torch.Tensor, cu_draft: torch.Tensor, u: torch.Tensor, r: torch.Tensor, *,
                 draft: Optional[torch.Tensor] = None, temperature: Optional[torch.Tensor] = None, past_len: Optional[torch.Tensor] = None,
                 want_logprob: bool = False):
        """cu_draft int32 [B+1] bounds the sequences' drafted tokens (tokens: int32 [T]).  target: bf16 or fp32 [T + B, V] logits, one row more
        for each sequence than it has drafted tokens; draft: alike [T, V], None for tokens that were not sampled.  u: fp32 [T] and r: fp32 [B], random
        numbers in [0, 1).  temperature: fp32 [B] (None: 1; 0 takes the largest logit).  past_len int32 [B]: tokens of the cache before the step.
        After run(): n_accepted int32 [B], out_tokens int32 [T + B] (-1 behind a sequence's last), logprob fp32 [T + B] if wanted, kept_len
        int32 [B] if past_len is given: the tokens of the cache that stand, the next step's past_len."""
        T, B = int(tokens.numel()), int(cu_draft.numel()) - 1
        self._device = _on_one_device(target, tokens, cu_draft, u, r, draft, temperature, past_len)
        _need(B >= 1, "cu_draft: int32 [B+1]")
        _check_ints(cu_draft, B + 1, "cu_draft")
        _check_ints(tokens, T, "tokens")
        _need(target.dtype in (torch.bfloat16, torch.float32), "target: bf16 or fp32 logits")
        for t, n, name in ((target, T + B, "target"), (draft, T, "draft")):
            _need(t is None or (t.dtype == target.dtype and t.dim() == 2 and t.shape[0] == n and t.shape[1] == target.shape[1] and t.stride(1) == 1),
                  f"{name}: [{n}, V] of the target's type, contiguous rows")
        for t, n, name in ((u, T, "u"), (r, B, "r"), (temperature, B, "temperature")):
            _need(t is None or (t.dtype == torch.float32 and t.is_contiguous() and t.numel() == n), f"{name}: contiguous fp32 [{n}]")
        if past_len is not None:
            _check_ints(past_len, B, "past_len")
        new = dict(device=self._device)
        self.n_accepted = torch.empty(B, dtype=torch.int32, **new)
        self.out_tokens = torch.empty(T + B, dtype=torch.int32, **new)
        self.logprob = torch.empty(T + B, dtype=torch.float32, **new) if want_logprob else None
        self.kept_len = torch.empty(B, dtype=torch.int32, **new) if past_len is not None else None
        self._held = (target, tokens, cu_draft, u, r, draft, temperature, past_len)
        kw = dict(draft=draft, temperature=temperature, past_len=past_len, logprob=self.logprob, kept_len=self.kept_len)
        probe = sp.make_verify_args(target, tokens, cu_draft, u, r, self.n_accepted, self.out_tokens, **kw)
        need = sp.sp_verify_workspace_bytes(probe)
        if need == 0:
            raise sp.SpError("sp_verify_workspace_bytes", sp.SP_EINVAL)
        self.workspace = torch.empty(need, dtype=torch.uint8, **new)
        self.args = sp.make_verify_args(target, tokens, cu_draft, u, r, self.n_accepted, self.out_tokens, workspace=self.workspace, **kw)

    def run(self, stream=None):
        self._call(sp.sp_verify, self.args, stream)
        return self.n_accepted, self.out_tokens
