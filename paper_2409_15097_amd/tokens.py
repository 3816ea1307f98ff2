"""ctypes binding of the operators on packed tokens.  Argument marshalling only; see include/bbm_tokens.h for the contract.

Tensors of a call lie on one GPU, which need not be the current one; work goes to that GPU's current stream, or to `stream`, and what a
call allocates belongs to the stream that the kernels run on."""
import ctypes as C
import math
from dataclasses import dataclass
from typing import Optional

import torch

from .binding import _check, _null_ctx, _ptr, _stream, lib


class _CPacked(C.Structure):
    _fields_ = [("ptr", C.c_void_p), ("row_stride", C.c_int64), ("head_stride", C.c_int64)]


class _CCache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("k_scale", C.c_void_p), ("v", C.c_void_p), ("v_scale", C.c_void_p),
                ("pages", C.c_int64), ("Hk", C.c_int64), ("page", C.c_int32), ("d", C.c_int32)]


def _declare(L):
    i64, vp, ci, cf, pk = C.c_int64, C.c_void_p, C.c_int, C.c_float, C.POINTER(_CPacked)
    cache = C.POINTER(_CCache)
    for name, args in {
        "bbm_build_slots": [vp, vp, i64, vp, i64, i64, ci, vp, i64, vp, i64, vp, vp, vp, vp, vp, vp],
        "bbm_rope": [pk, pk, i64, pk, pk, i64, i64, ci, ci, ci, ci, vp, vp, cf, vp],
        "bbm_prompt_attn_fwd": [pk, pk, pk, pk, vp, i64, i64, vp, i64, i64, ci, cf, vp],
        "bbm_prompt_attn_bwd": [pk, pk, pk, pk, pk, vp, pk, pk, pk, i64, i64, vp, i64, i64, ci, cf, vp, C.c_size_t, vp],
        "bbm_kv4_append": [pk, pk, i64, vp, cache, vp],
        "bbm_kv4_read": [vp, i64, cache, pk, pk, vp],
        "bbm_kv4_attn": [pk, pk, vp, i64, i64, vp, vp, vp, i64, i64, vp, i64, cache, i64, cf, i64, vp, C.c_size_t, vp],
    }.items():
        f = getattr(L, name)
        f.restype, f.argtypes = ci, args
    L.bbm_prompt_attn_bwd_workspace_bytes.restype = C.c_size_t
    L.bbm_prompt_attn_bwd_workspace_bytes.argtypes = [i64, i64]
    L.bbm_kv4_attn_workspace_bytes.restype = C.c_size_t
    L.bbm_kv4_attn_workspace_bytes.argtypes = [i64, i64, i64, i64, ci, i64]


_declare(lib)


def _on(device, stream, *others):
    """The context in which a call on `device` allocates and launches; every tensor of `others` has to be there too."""
    for t in others:
        assert t is None or t.device == device, "the tensors of a call lie on one device"
    if stream is not None:
        assert stream.device == device, "the stream is another device's"
        return torch.cuda.stream(stream)
    return _null_ctx() if device.index == torch.cuda.current_device() else torch.cuda.device(device)


def _packed(x: torch.Tensor, T: int, heads: int, d: int) -> _CPacked:
    assert x.is_cuda and x.dtype == torch.bfloat16 and x.shape == (T, heads, d), "a packed bf16 tensor of this many tokens, heads and elements"
    row, head, one = x.stride()
    assert one == 1, "the elements of a head lie one behind the other"
    return _CPacked(x.data_ptr(), row if T > 1 else 0, head if heads > 1 else 0)   # (a stride that is never taken may be anything)


def _ints(x: torch.Tensor, n: Optional[int] = None):
    assert x.is_cuda and x.dtype == torch.int32 and x.is_contiguous() and x.dim() == 1 and (n is None or x.numel() == n)


@dataclass
class Slots:
    """What bbm_build_slots writes for a step (int32 device tensors)."""
    cu_new: torch.Tensor      # [R + 1] packed offsets of the new tokens
    lens: torch.Tensor        # [R] tokens in the cache behind the step
    positions: torch.Tensor   # [T]
    slots: torch.Tensor       # [T] slot in the cache, -1: none
    free_next: torch.Tensor   # [1] index of the next free page; beyond the list's length, the list was too short


def bbm_build_slots(ctx_lens: torch.Tensor, new_lens: torch.Tensor, block_table: torch.Tensor, free_pages: torch.Tensor, free_at: torch.Tensor,
                    num_tokens: int, page: int, stream=None) -> Slots:
    """ctx_lens, new_lens: int32 [R]; block_table: int32 [R, max_pages] (row stride may exceed max_pages), gets the pages that the step
    takes from free_pages (int32 [n]), index free_at (int32 [1]) on; num_tokens: rows of the step's tensors."""
    R = ctx_lens.numel()
    _ints(ctx_lens), _ints(new_lens, R), _ints(free_pages), _ints(free_at, 1)
    assert block_table.is_cuda and block_table.dtype == torch.int32 and block_table.dim() == 2 and block_table.shape[0] == R and block_table.stride(1) == 1
    width = block_table.shape[1]
    with _on(ctx_lens.device, stream, new_lens, block_table, free_pages, free_at):
        buf = torch.empty(2 * R + 2 + 2 * num_tokens, dtype=torch.int32, device=ctx_lens.device)
        cu, lens, pos, slots, nxt = buf.split((R + 1, R, num_tokens, num_tokens, 1))
        at = buf.data_ptr()
        _check(lib.bbm_build_slots(_ptr(ctx_lens), _ptr(new_lens), R, _ptr(block_table), block_table.stride(0) if R > 1 else width, width, page,
                                   _ptr(free_pages), free_pages.numel(), _ptr(free_at), num_tokens, at, at + 4 * (R + 1), at + 4 * (2 * R + 1),
                                   at + 4 * (2 * R + 1 + num_tokens), at + 4 * (2 * R + 1 + 2 * num_tokens), _stream()))
    return Slots(cu, lens, pos, slots, nxt)


def rope_freqs(rot: int, base: float = 10000.0, factor: float = 1.0, method: Optional[str] = None, trained_len: Optional[int] = None,
               beta_fast: float = 32.0, beta_slow: float = 1.0, device="cuda"):
    """(freqs fp32 [rot/2], mscale) for bbm_rope, from base^(-2j/rot), formed in 64 bits.  For contexts `factor` times as long as those trained on:
    "linear" divides all frequencies by it; "ntk" raises the base so that the slowest pair is slowed by it and the fastest not at all;
    "yarn" slows a pair that makes fewer than beta_slow turns in trained_len tokens by it, one with more than beta_fast not at all and
    those between in proportion, and scales both sine and cosine by 0.1 ln(factor) + 1 (published as YaRN, arXiv 2309.00071)."""
    if rot < 2 or rot % 2 or not base > 0 or not factor >= 1:
        raise ValueError(f"rot={rot} must be even and positive, base={base} positive, factor={factor} no less than 1")
    j = torch.arange(0, rot, 2, dtype=torch.float64)
    mscale = 1.0
    if method == "ntk":
        if rot < 4:
            raise ValueError("ntk needs two pairs")
        base *= factor ** (rot / (rot - 2))
    freqs = base ** (-j / rot)
    if method == "linear":
        freqs = freqs / factor
    elif method == "yarn":
        if not trained_len or not beta_fast > beta_slow:
            raise ValueError("yarn needs trained_len, and beta_fast above beta_slow")
        turns = trained_len * freqs / (2 * math.pi)
        keep = ((turns - beta_slow) / (beta_fast - beta_slow)).clamp(0, 1)
        freqs = freqs * (keep + (1 - keep) / factor)
        mscale = 0.1 * math.log(factor) + 1.0
    elif method not in (None, "ntk"):
        raise ValueError(f"method {method!r} is none of linear, ntk, yarn")
    return freqs.to(torch.float32).to(device), mscale


def bbm_rope(q: torch.Tensor, k: Optional[torch.Tensor], positions: torch.Tensor, freqs: torch.Tensor, interleaved: bool = False, mscale: float = 1.0,
             inverse: bool = False, out_q: Optional[torch.Tensor] = None, out_k: Optional[torch.Tensor] = None, stream=None):
    """q: packed [T, H, d], k: packed [T, Hk, d] or None; positions int32 [T]; freqs fp32 [rot/2] (rope_freqs).  Returns (q, k) turned,
    contiguous unless out_q and out_k are given (out_q=q turns in place).  inverse=True is the gradient: of the outputs to that of the inputs."""
    T, H, d = q.shape
    Hk = 0 if k is None else k.shape[1]
    _ints(positions, T)
    assert freqs.is_cuda and freqs.dtype == torch.float32 and freqs.is_contiguous() and freqs.dim() == 1
    with _on(q.device, stream, k, positions, freqs, out_q, out_k):
        if out_q is None:
            out_q = torch.empty((T, H, d), dtype=q.dtype, device=q.device)
        if k is not None and out_k is None:
            out_k = torch.empty((T, Hk, d), dtype=k.dtype, device=k.device)
        _check(lib.bbm_rope(_packed(q, T, H, d), _packed(out_q, T, H, d), H, None if k is None else _packed(k, T, Hk, d),
                            None if k is None else _packed(out_k, T, Hk, d), Hk, T, d, 2 * freqs.numel(), int(interleaved), int(inverse), _ptr(positions),
                            _ptr(freqs), mscale, _stream()))
    return out_q, out_k


def bbm_prompt_attn_fwd(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu: torch.Tensor, softmax_scale: Optional[float] = None,
                        out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, stream=None):
    """q: packed [T, H, d], k, v: packed [T, Hk, d]; cu int32 [R + 1].  Returns (O bf16 [T, H, d], lse fp32 [H, T])."""
    T, H, d = q.shape
    Hk = k.shape[1]
    _ints(cu)
    assert lse is None or (lse.is_cuda and lse.dtype == torch.float32 and lse.is_contiguous() and lse.shape == (H, T))
    with _on(q.device, stream, k, v, cu, out, lse):
        if out is None:
            out = torch.empty((T, H, d), dtype=q.dtype, device=q.device)
        if lse is None:
            lse = torch.empty((H, T), dtype=torch.float32, device=q.device)
        _check(lib.bbm_prompt_attn_fwd(_packed(q, T, H, d), _packed(k, T, Hk, d), _packed(v, T, Hk, d), _packed(out, T, H, d), _ptr(lse), T, cu.numel() - 1,
                                       _ptr(cu), H, Hk, d, float(d) ** -0.5 if softmax_scale is None else softmax_scale, _stream()))
    return out, lse


def bbm_prompt_attn_bwd_workspace_bytes(T: int, H: int) -> int:
    return int(lib.bbm_prompt_attn_bwd_workspace_bytes(T, H))


def bbm_prompt_attn_bwd(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, o: torch.Tensor, d_o: torch.Tensor, lse: torch.Tensor, cu: torch.Tensor,
                        softmax_scale: Optional[float] = None, dq: Optional[torch.Tensor] = None, dk: Optional[torch.Tensor] = None,
                        dv: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None):
    """Of what bbm_prompt_attn_fwd took and gave, and d_o as o: (dQ [T, H, d], dK, dV [T, Hk, d]), bf16."""
    T, H, d = q.shape
    Hk = k.shape[1]
    _ints(cu)
    assert lse.is_cuda and lse.dtype == torch.float32 and lse.is_contiguous() and lse.shape == (H, T)
    with _on(q.device, stream, k, v, o, d_o, lse, cu, dq, dk, dv, workspace):
        dq = torch.empty((T, H, d), dtype=q.dtype, device=q.device) if dq is None else dq
        dk = torch.empty((T, Hk, d), dtype=q.dtype, device=q.device) if dk is None else dk
        dv = torch.empty((T, Hk, d), dtype=q.dtype, device=q.device) if dv is None else dv
        if workspace is None:
            workspace = torch.empty(bbm_prompt_attn_bwd_workspace_bytes(T, H), dtype=torch.uint8, device=q.device)
        assert workspace.is_contiguous()
        _check(lib.bbm_prompt_attn_bwd(_packed(q, T, H, d), _packed(k, T, Hk, d), _packed(v, T, Hk, d), _packed(o, T, H, d), _packed(d_o, T, H, d), _ptr(lse),
                                       _packed(dq, T, H, d), _packed(dk, T, Hk, d), _packed(dv, T, Hk, d), T, cu.numel() - 1, _ptr(cu), H, Hk, d,
                                       float(d) ** -0.5 if softmax_scale is None else softmax_scale, _ptr(workspace), workspace.numel() * workspace.element_size(),
                                       _stream()))
    return dq, dk, dv


@dataclass
class KV4Cache:
    """The tensors of a paged cache in 4 bits (uint8, contiguous): k, v [pages, Hk, page, d/2], k_scale [pages, Hk, page, d/32],
    v_scale [pages, Hk, d/32, page]."""
    k: torch.Tensor
    k_scale: torch.Tensor
    v: torch.Tensor
    v_scale: torch.Tensor

    def c_struct(self) -> _CCache:
        pages, Hk, page, half = self.k.shape
        for t, shape in ((self.k, (pages, Hk, page, half)), (self.v, (pages, Hk, page, half)), (self.k_scale, (pages, Hk, page, half // 16)),
                         (self.v_scale, (pages, Hk, half // 16, page))):
            assert t.is_cuda and t.dtype == torch.uint8 and t.is_contiguous() and t.shape == shape, "a cache's tensors have the shapes of KV4Cache"
        return _CCache(_ptr(self.k), _ptr(self.k_scale), _ptr(self.v), _ptr(self.v_scale), pages, Hk, page, 2 * half)


def kv4_cache(pages: int, heads: int, d: int, page: int, device="cuda") -> KV4Cache:
    """An empty cache: zeros."""
    z = lambda *shape: torch.zeros(shape, dtype=torch.uint8, device=device)  # noqa: E731
    return KV4Cache(z(pages, heads, page, d // 2), z(pages, heads, page, d // 32), z(pages, heads, page, d // 2), z(pages, heads, d // 32, page))


def bbm_kv4_append(k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, cache: KV4Cache, stream=None) -> KV4Cache:
    """k, v: packed [T, Hk, d] into the slots (int32 [T]) of the cache; rows with a slot outside the cache are left out."""
    T, Hk, d = k.shape
    _ints(slots, T)
    c = cache.c_struct()
    assert (Hk, d) == (c.Hk, c.d), "the cache has other heads"
    with _on(k.device, stream, v, slots, cache.k, cache.k_scale, cache.v, cache.v_scale):
        _check(lib.bbm_kv4_append(_packed(k, T, Hk, d), _packed(v, T, Hk, d), T, _ptr(slots), c, _stream()))
    return cache


def bbm_kv4_read(slots: torch.Tensor, cache: KV4Cache, out_k: Optional[torch.Tensor] = None, out_v: Optional[torch.Tensor] = None, stream=None):
    """The values (k, v) bf16 [T, Hk, d] that the cache holds for the slots (int32 [T]); zeros for a slot outside the cache."""
    _ints(slots)
    c, T = cache.c_struct(), slots.numel()
    with _on(slots.device, stream, cache.k, cache.k_scale, cache.v, cache.v_scale, out_k, out_v):
        out_k = torch.empty((T, c.Hk, c.d), dtype=torch.bfloat16, device=slots.device) if out_k is None else out_k
        out_v = torch.empty((T, c.Hk, c.d), dtype=torch.bfloat16, device=slots.device) if out_v is None else out_v
        _check(lib.bbm_kv4_read(_ptr(slots), T, c, _packed(out_k, T, c.Hk, c.d), _packed(out_v, T, c.Hk, c.d), _stream()))
    return out_k, out_v


def bbm_kv4_attn_workspace_bytes(T: int, R: int, H: int, Hk: int, d: int, max_len: int) -> int:
    return int(lib.bbm_kv4_attn_workspace_bytes(T, R, H, Hk, d, max_len))


def bbm_kv4_attn(q: torch.Tensor, cache: KV4Cache, block_table: torch.Tensor, lens: torch.Tensor, cu: torch.Tensor, mask: Optional[torch.Tensor] = None,
                 max_len: Optional[int] = None, softmax_scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                 lse: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None):
    """q: packed [T, H, d], the last cu[r+1] - cu[r] of the lens[r] tokens that request r has in the cache (append first); block_table int32
    [R, max_pages]; mask: int64 [T, words], bit j of a row's words: the row sees new token j of its request (None: causal); max_len: an upper
    bound of lens, for the work split (None: what the table holds).  Returns (O bf16 [T, H, d], lse fp32 [H, T])."""
    T, H, d = q.shape
    R = lens.numel()
    c = cache.c_struct()
    _ints(lens), _ints(cu, R + 1)
    assert d == c.d, "the cache has another head size"
    assert block_table.is_cuda and block_table.dtype == torch.int32 and block_table.dim() == 2 and block_table.shape[0] == R and block_table.stride(1) == 1
    assert mask is None or (mask.is_cuda and mask.dtype == torch.int64 and mask.is_contiguous() and mask.dim() == 2 and mask.shape[0] == T)
    assert lse is None or (lse.is_cuda and lse.dtype == torch.float32 and lse.is_contiguous() and lse.shape == (H, T))
    width = block_table.shape[1]
    max_len = width * c.page if max_len is None else max_len
    with _on(q.device, stream, cache.k, cache.k_scale, cache.v, cache.v_scale, block_table, lens, cu, mask, out, lse, workspace):
        if out is None:
            out = torch.empty((T, H, d), dtype=q.dtype, device=q.device)
        if lse is None:
            lse = torch.empty((H, T), dtype=torch.float32, device=q.device)
        if workspace is None:
            need = bbm_kv4_attn_workspace_bytes(T, R, H, c.Hk, d, max_len)
            workspace = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
        assert workspace is None or workspace.is_contiguous()
        _check(lib.bbm_kv4_attn(_packed(q, T, H, d), _packed(out, T, H, d), _ptr(lse), T, R, _ptr(cu), _ptr(lens), _ptr(block_table),
                                block_table.stride(0) if R > 1 else width, width, _ptr(mask), 0 if mask is None else mask.shape[1], c, H,
                                float(d) ** -0.5 if softmax_scale is None else softmax_scale, max_len, _ptr(workspace),
                                0 if workspace is None else workspace.numel() * workspace.element_size(), _stream()))
    return out, lse
