"""ctypes binding of the operators on packed tokens.  Argument marshalling only; see include/bbm_tokens.h for the contract.

Tensors of a call lie on one GPU, which need not be the current one; work goes to that GPU's current stream, or to `stream`, and what a
call allocates belongs to the stream that the kernels run on."""
import ctypes as C
import math
from dataclasses import dataclass
from typing import Optional

import torch

from .binding import _check, _current_device, _null_ctx, _raw_stream, lib


class _CPacked(C.Structure):
    _fields_ = [("ptr", C.c_void_p), ("row_stride", C.c_int64), ("head_stride", C.c_int64)]


class _CCache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("k_scale", C.c_void_p), ("v", C.c_void_p), ("v_scale", C.c_void_p),
                ("pages", C.c_int64), ("Hk", C.c_int64), ("page", C.c_int32), ("d", C.c_int32)]


# A small call is all submission: of 10.8 us that a rotation of 33 tokens took the host, the launch is 3.2, allocating two results 2.9; structures a tensor,
# contexts, devices compared as objects were the rest.  So: the current device's stream is asked for by its number, packed tensors go into one
# array, and only a call for another device or stream enters a context (and then calls itself).
_I64x6, _I64x12, _I64x24 = C.c_int64 * 6, C.c_int64 * 12, C.c_int64 * 24
_address = C.addressof


def _elsewhere(device: int, stream) -> bool:
    if stream is None and _raw_stream is not None and _current_device is not None:
        return device != _current_device()
    return True


def _context(device: int, stream):
    """For a call on another device than the current one, or on a stream of its own."""
    if stream is not None:
        assert stream.device.index == device, "the stream is another device's"
        return torch.cuda.stream(stream)
    return torch.cuda.device(device) if device != torch.cuda.current_device() else _null_ctx()


def _here(device: int) -> int:
    return _raw_stream(device) if _raw_stream is not None else torch.cuda.current_stream(device).cuda_stream


def _packed(x: torch.Tensor, device: int, T: int, heads: int, d: int):
    """(address, row stride, head stride) of a packed tensor."""
    assert x.dtype is torch.bfloat16 and x.shape == (T, heads, d), "a packed bf16 tensor of this many tokens, heads and elements"
    assert x.get_device() == device, "the tensors of a call lie on one GPU"
    row, head, one = x.stride()
    assert one == 1, "the elements of a head lie one behind the other"
    return x.data_ptr(), row if T > 1 else 0, head if heads > 1 else 0   # (a stride that is never taken may be anything)


def _out(x: Optional[torch.Tensor], like: torch.Tensor, device: int, T: int, heads: int, d: int):
    """A packed output, allocated if there is none, and what _packed says of it."""
    if x is not None:
        return x, _packed(x, device, T, heads, d)
    x = like.new_empty((T, heads, d), dtype=torch.bfloat16)
    return x, (x.data_ptr(), heads * d if T > 1 else 0, d if heads > 1 else 0)


def _ints(x: torch.Tensor, device: int, n: Optional[int] = None) -> int:
    assert x.dtype is torch.int32 and x.is_contiguous() and x.dim() == 1 and (n is None or x.numel() == n), "a contiguous int32 vector of this length"
    assert x.get_device() == device, "the tensors of a call lie on one GPU"
    return x.data_ptr()


def _table(x: torch.Tensor, device: int, R: int):
    """(address, row stride, width) of a block table."""
    assert x.dtype is torch.int32 and x.dim() == 2 and x.shape[0] == R and x.stride(1) == 1, "an int32 table of a row for each request"
    assert x.get_device() == device, "the tensors of a call lie on one GPU"
    width = x.shape[1]
    return x.data_ptr(), x.stride(0) if R > 1 else width, width


def _lse(x: torch.Tensor, device: int, H: int, T: int) -> int:
    assert x.dtype is torch.float32 and x.is_contiguous() and x.shape == (H, T), "a contiguous fp32 log-sum-exp [H, T]"
    assert x.get_device() == device, "the tensors of a call lie on one GPU"
    return x.data_ptr()


def _lse_out(x: Optional[torch.Tensor], like: torch.Tensor, device: int, H: int, T: int):
    if x is not None:
        return x, _lse(x, device, H, T)
    x = like.new_empty((H, T), dtype=torch.float32)
    return x, x.data_ptr()


def _gpu(x: torch.Tensor) -> int:
    device = x.get_device()
    assert device >= 0, "the tensors of a call lie on one GPU"
    return device


def _workspace(x: Optional[torch.Tensor], device: int):
    if x is None:
        return None, 0
    assert x.is_contiguous() and x.get_device() == device, "a contiguous workspace on the GPU of the call"
    return x.data_ptr(), x.numel() * x.element_size()


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
    dev, R = _gpu(ctx_lens), ctx_lens.numel()
    if _elsewhere(dev, stream):
        with _context(dev, stream):
            return _build_slots(dev, R, ctx_lens, new_lens, block_table, free_pages, free_at, num_tokens, page)
    return _build_slots(dev, R, ctx_lens, new_lens, block_table, free_pages, free_at, num_tokens, page)


def _build_slots(dev, R, ctx_lens, new_lens, block_table, free_pages, free_at, T, page):
    table, stride, width = _table(block_table, dev, R)
    args = _ints(ctx_lens, dev), _ints(new_lens, dev, R), R, table, stride, width, page, _ints(free_pages, dev), free_pages.numel(), _ints(free_at, dev, 1)
    buf = ctx_lens.new_empty(2 * R + 2 + 2 * T)
    at = buf.data_ptr()
    _check(lib.bbm_build_slots(*args, T, at, at + 4 * (R + 1), at + 4 * (2 * R + 1), at + 4 * (2 * R + 1 + T), at + 4 * (2 * R + 1 + 2 * T), _here(dev)))
    return Slots(*torch.split_with_sizes(buf, (R + 1, R, T, T, 1)))


def rope_freqs(rot: int, base: float = 10000.0, factor: float = 1.0, method: Optional[str] = None, trained_len: Optional[int] = None,
               beta_fast: float = 32.0, beta_slow: float = 1.0, device="cuda"):
    """(freqs fp32 [rot/2], mscale) for bbm_rope, from base^(-2j/rot), formed in 64 bits.  For contexts `factor` times as long as those trained on:
    "linear" divides all frequencies by it; "ntk" raises the base so that the slowest pair is slowed by it and the fastest not at all;
    "yarn" slows a pair that makes fewer than beta_slow turns in trained_len tokens by it, one with more than beta_fast not at all and
    those between in proportion, and scales both sine and cosine by 0.1 ln(factor) + 1 (published as YaRN, arXiv 2309.00071)."""
    if rot < 2 or rot % 2 or not base > 0 or not factor >= 1:
        raise ValueError(f"rot={rot} must be even and positive, base={base} positive, factor={factor} no less than 1")
    if method is None and factor != 1:
        raise ValueError(f"factor={factor} needs a method: linear, ntk or yarn")
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
    dev = _gpu(q)
    if _elsewhere(dev, stream):
        with _context(dev, stream):
            return _rope(dev, q, k, positions, freqs, interleaved, mscale, inverse, out_q, out_k)
    return _rope(dev, q, k, positions, freqs, interleaved, mscale, inverse, out_q, out_k)


def _rope(dev, q, k, positions, freqs, interleaved, mscale, inverse, out_q, out_k):
    T, H, d = q.shape
    assert freqs.dtype is torch.float32 and freqs.is_contiguous() and freqs.dim() == 1 and freqs.get_device() == dev, "fp32 frequencies on the GPU of the call"
    pos, packed = _ints(positions, dev, T), _packed(q, dev, T, H, d)
    out_q, to = _out(out_q, q, dev, T, H, d)
    if k is None:
        Hk, keep = 0, _I64x12(*packed, *to)
    else:
        Hk = k.shape[1]
        more = _packed(k, dev, T, Hk, d)
        out_k, to_k = _out(out_k, k, dev, T, Hk, d)
        keep = _I64x12(*packed, *to, *more, *to_k)
    at = _address(keep)
    _check(lib.bbm_rope(at, at + 24, H, at + 48, at + 72, Hk, T, d, 2 * freqs.shape[0], interleaved, inverse, pos, freqs.data_ptr(), mscale, _here(dev)))
    return out_q, out_k


def bbm_prompt_attn_fwd(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu: torch.Tensor, softmax_scale: Optional[float] = None,
                        out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, stream=None):
    """q: packed [T, H, d], k, v: packed [T, Hk, d]; cu int32 [R + 1].  Returns (O bf16 [T, H, d], lse fp32 [H, T])."""
    dev = _gpu(q)
    if _elsewhere(dev, stream):
        with _context(dev, stream):
            return _prompt_fwd(dev, q, k, v, cu, softmax_scale, out, lse)
    return _prompt_fwd(dev, q, k, v, cu, softmax_scale, out, lse)


def _prompt_fwd(dev, q, k, v, cu, softmax_scale, out, lse):
    T, H, d = q.shape
    Hk, offsets = k.shape[1], _ints(cu, dev)
    packed = _packed(q, dev, T, H, d) + _packed(k, dev, T, Hk, d) + _packed(v, dev, T, Hk, d)
    out, to = _out(out, q, dev, T, H, d)
    lse, lse_at = _lse_out(lse, q, dev, H, T)
    keep = _I64x12(*packed, *to)
    at = _address(keep)
    _check(lib.bbm_prompt_attn_fwd(at, at + 24, at + 48, at + 72, lse_at, T, cu.shape[0] - 1, offsets, H, Hk, d,
                                   d ** -0.5 if softmax_scale is None else softmax_scale, _here(dev)))
    return out, lse


def bbm_prompt_attn_bwd_workspace_bytes(T: int, R: int, H: int, Hk: int, d: int) -> int:
    return int(lib.bbm_prompt_attn_bwd_workspace_bytes(T, R, H, Hk, d))


def bbm_prompt_attn_bwd(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, o: torch.Tensor, d_o: torch.Tensor, lse: torch.Tensor, cu: torch.Tensor,
                        softmax_scale: Optional[float] = None, dq: Optional[torch.Tensor] = None, dk: Optional[torch.Tensor] = None,
                        dv: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None):
    """Of what bbm_prompt_attn_fwd took and gave, and d_o as o: (dQ [T, H, d], dK, dV [T, Hk, d]), bf16."""
    dev = _gpu(q)
    if _elsewhere(dev, stream):
        with _context(dev, stream):
            return _prompt_bwd(dev, q, k, v, o, d_o, lse, cu, softmax_scale, dq, dk, dv, workspace)
    return _prompt_bwd(dev, q, k, v, o, d_o, lse, cu, softmax_scale, dq, dk, dv, workspace)


def _prompt_bwd(dev, q, k, v, o, d_o, lse, cu, softmax_scale, dq, dk, dv, workspace):
    T, H, d = q.shape
    Hk, offsets = k.shape[1], _ints(cu, dev)
    packed = _packed(q, dev, T, H, d) + _packed(k, dev, T, Hk, d) + _packed(v, dev, T, Hk, d) + _packed(o, dev, T, H, d) + _packed(d_o, dev, T, H, d)
    (dq, to_q), (dk, to_k), (dv, to_v) = _out(dq, q, dev, T, H, d), _out(dk, k, dev, T, Hk, d), _out(dv, v, dev, T, Hk, d)
    if workspace is None:
        workspace = q.new_empty(lib.bbm_prompt_attn_bwd_workspace_bytes(T, cu.shape[0] - 1, H, Hk, d), dtype=torch.uint8)
    keep = _I64x24(*packed, *to_q, *to_k, *to_v)
    at = _address(keep)
    _check(lib.bbm_prompt_attn_bwd(at, at + 24, at + 48, at + 72, at + 96, _lse(lse, dev, H, T), at + 120, at + 144, at + 168, T, cu.shape[0] - 1, offsets, H, Hk, d,
                                   d ** -0.5 if softmax_scale is None else softmax_scale, *_workspace(workspace, dev), _here(dev)))
    return dq, dk, dv


class KV4Cache:
    """The tensors of a paged cache in 4 bits (uint8, contiguous, on one GPU): k, v [pages, Hk, page, d/2], k_scale [pages, Hk, page, d/32],
    v_scale [pages, Hk, d/32, page]."""
    __slots__ = ("k", "k_scale", "v", "v_scale", "device", "c_struct")

    def __init__(self, k: torch.Tensor, k_scale: torch.Tensor, v: torch.Tensor, v_scale: torch.Tensor):
        device = _gpu(k)
        pages, Hk, page, half = k.shape
        values, groups = (pages, Hk, page, half), half // 16
        assert v.shape == values and k_scale.shape == (pages, Hk, page, groups) and v_scale.shape == (pages, Hk, groups, page), "a cache's tensors have the shapes of KV4Cache"
        u8 = torch.uint8
        assert k.dtype is u8 and v.dtype is u8 and k_scale.dtype is u8 and v_scale.dtype is u8, "a cache's tensors are uint8"
        assert k.is_contiguous() and v.is_contiguous() and k_scale.is_contiguous() and v_scale.is_contiguous(), "a cache's tensors are contiguous"
        assert v.get_device() == device and k_scale.get_device() == device and v_scale.get_device() == device, "a cache's tensors lie on one GPU"
        put = object.__setattr__
        put(self, "k", k), put(self, "k_scale", k_scale), put(self, "v", v), put(self, "v_scale", v_scale), put(self, "device", device)
        put(self, "c_struct", _CCache(k.data_ptr(), k_scale.data_ptr(), v.data_ptr(), v_scale.data_ptr(), pages, Hk, page, 2 * half))

    def __setattr__(self, name, value):
        raise AttributeError("a cache's tensors are what it was made of: make another KV4Cache")


def kv4_cache(pages: int, heads: int, d: int, page: int, device="cuda") -> KV4Cache:
    """An empty cache: zeros."""
    z = lambda *shape: torch.zeros(shape, dtype=torch.uint8, device=device)  # noqa: E731
    return KV4Cache(z(pages, heads, page, d // 2), z(pages, heads, page, d // 32), z(pages, heads, page, d // 2), z(pages, heads, d // 32, page))


def bbm_kv4_append(k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, cache: KV4Cache, stream=None) -> KV4Cache:
    """k, v: packed [T, Hk, d] into the slots (int32 [T]) of the cache; rows with a slot outside the cache are left out."""
    dev = _gpu(k)
    if _elsewhere(dev, stream):
        with _context(dev, stream):
            return _kv4_append(dev, k, v, slots, cache)
    return _kv4_append(dev, k, v, slots, cache)


def _kv4_append(dev, k, v, slots, cache):
    T, Hk, d = k.shape
    c = cache.c_struct
    assert (Hk, d) == (c.Hk, c.d) and cache.device == dev, "the cache has other heads, or lies elsewhere"
    keep = _I64x6(*_packed(k, dev, T, Hk, d), *_packed(v, dev, T, Hk, d))
    at = _address(keep)
    _check(lib.bbm_kv4_append(at, at + 24, T, _ints(slots, dev, T), _address(c), _here(dev)))
    return cache


def bbm_kv4_read(slots: torch.Tensor, cache: KV4Cache, out_k: Optional[torch.Tensor] = None, out_v: Optional[torch.Tensor] = None, stream=None):
    """The values (k, v) bf16 [T, Hk, d] that the cache holds for the slots (int32 [T]); zeros for a slot outside the cache."""
    dev = _gpu(slots)
    if _elsewhere(dev, stream):
        with _context(dev, stream):
            return _kv4_read(dev, slots, cache, out_k, out_v)
    return _kv4_read(dev, slots, cache, out_k, out_v)


def _kv4_read(dev, slots, cache, out_k, out_v):
    c, T = cache.c_struct, slots.shape[0]
    Hk, d = c.Hk, c.d
    assert cache.device == dev, "the cache lies elsewhere"
    (out_k, to_k), (out_v, to_v) = _out(out_k, slots, dev, T, Hk, d), _out(out_v, slots, dev, T, Hk, d)
    keep = _I64x6(*to_k, *to_v)
    at = _address(keep)
    _check(lib.bbm_kv4_read(_ints(slots, dev), T, _address(c), at, at + 24, _here(dev)))
    return out_k, out_v


def bbm_kv4_attn_workspace_bytes(T: int, R: int, H: int, Hk: int, d: int, max_len: int) -> int:
    return int(lib.bbm_kv4_attn_workspace_bytes(T, R, H, Hk, d, max_len))


def bbm_kv4_attn(q: torch.Tensor, cache: KV4Cache, block_table: torch.Tensor, lens: torch.Tensor, cu: torch.Tensor, mask: Optional[torch.Tensor] = None,
                 max_len: Optional[int] = None, softmax_scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                 lse: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None):
    """q: packed [T, H, d], the last cu[r+1] - cu[r] of the lens[r] tokens that request r has in the cache (append first); block_table int32
    [R, max_pages]; mask: int64 [T, words], bit j of a row's words: the row sees new token j of its request (None: causal); max_len: an upper
    bound of lens, for the work split (None: what the table holds).  Returns (O bf16 [T, H, d], lse fp32 [H, T])."""
    dev = _gpu(q)
    if _elsewhere(dev, stream):
        with _context(dev, stream):
            return _kv4_attn(dev, q, cache, block_table, lens, cu, mask, max_len, softmax_scale, out, lse, workspace)
    return _kv4_attn(dev, q, cache, block_table, lens, cu, mask, max_len, softmax_scale, out, lse, workspace)


def _kv4_attn(dev, q, cache, block_table, lens, cu, mask, max_len, softmax_scale, out, lse, workspace):
    T, H, d = q.shape
    R, c = lens.shape[0], cache.c_struct
    assert d == c.d and cache.device == dev, "the cache has another head size, or lies elsewhere"
    table, stride, width = _table(block_table, dev, R)
    bits, words = None, 0
    if mask is not None:
        assert mask.dtype is torch.int64 and mask.is_contiguous() and mask.dim() == 2 and mask.shape[0] == T and mask.get_device() == dev, "an int64 mask of words for every row"
        bits, words = mask.data_ptr(), mask.shape[1]
    max_len = width * c.page if max_len is None else max_len
    packed = _packed(q, dev, T, H, d)
    out, to = _out(out, q, dev, T, H, d)
    lse, lse_at = _lse_out(lse, q, dev, H, T)
    if workspace is None:
        need = lib.bbm_kv4_attn_workspace_bytes(T, R, H, c.Hk, d, max_len)
        workspace = q.new_empty(need, dtype=torch.uint8) if need else None
    keep = _I64x6(*packed, *to)
    at = _address(keep)
    _check(lib.bbm_kv4_attn(at, at + 24, lse_at, T, R, _ints(cu, dev, R + 1), _ints(lens, dev, R), table, stride, width, bits, words, _address(c), H,
                            d ** -0.5 if softmax_scale is None else softmax_scale, max_len, *_workspace(workspace, dev), _here(dev)))
    return out, lse
