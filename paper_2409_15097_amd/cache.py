"""ctypes binding of the operators on the 4-bit cache of many and long answers.  Argument marshalling only; see include/bbm_cache.h for the contract.

Devices, streams and what a call allocates are as in tokens.py."""
from dataclasses import dataclass
from functools import lru_cache
from typing import Optional

import torch

from .binding import _check, lib
from .tokens import KV4Cache, _address, _context, _elsewhere, _gpu, _here, _I64x6, _ints, _lse, _lse_out, _out, _packed, _table, _workspace


def _mask(mask: Optional[torch.Tensor], device: int, T: int):
    """(address, words of a row) of a mask over new tokens."""
    if mask is None:
        return None, 0
    assert mask.dtype is torch.int64 and mask.is_contiguous() and mask.dim() == 2 and mask.shape[0] == T and mask.get_device() == device, "an int64 mask of words for every row"
    return mask.data_ptr(), mask.shape[1]


def _groups(group_cu: Optional[torch.Tensor], shared_lens: Optional[torch.Tensor], device: int):
    """(number, addresses) of the groups that share prefixes."""
    assert (group_cu is None) == (shared_lens is None), "groups have offsets and shared lengths"
    if group_cu is None:
        return 0, None, None
    S = shared_lens.shape[0]
    return S, _ints(group_cu, device, S + 1), _ints(shared_lens, device, S)


@lru_cache(maxsize=256)   # (of sizes alone; asking the library is 0.5 us of a call that takes the host 12)
def bbm_kv4_shared_attn_workspace_bytes(T: int, R: int, S: int, H: int, Hk: int, d: int, max_shared: int, max_own: int) -> int:
    return int(lib.bbm_kv4_shared_attn_workspace_bytes(T, R, S, H, Hk, d, max_shared, max_own))


def bbm_kv4_shared_attn(q: torch.Tensor, cache: KV4Cache, block_table: torch.Tensor, lens: torch.Tensor, cu: torch.Tensor, group_cu: Optional[torch.Tensor],
                        shared_lens: Optional[torch.Tensor], mask: Optional[torch.Tensor] = None, max_shared: Optional[int] = None, max_own: Optional[int] = None,
                        softmax_scale: Optional[float] = None, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                        workspace: Optional[torch.Tensor] = None, stream=None):
    """bbm_kv4_attn where requests group_cu[g] .. group_cu[g+1] - 1 (int32 [S + 1]) have their first shared_lens[g] (int32 [S]) keys in common, which are read once for all of them;
    max_shared, max_own: upper bounds of shared_lens and of the keys behind them, for the work split (None: what the table holds).  Returns (O bf16 [T, H, d], lse fp32 [H, T])."""
    dev = _gpu(q)
    if _elsewhere(dev, stream):
        with _context(dev, stream):
            return _kv4_shared_attn(dev, q, cache, block_table, lens, cu, group_cu, shared_lens, mask, max_shared, max_own, softmax_scale, out, lse, workspace)
    return _kv4_shared_attn(dev, q, cache, block_table, lens, cu, group_cu, shared_lens, mask, max_shared, max_own, softmax_scale, out, lse, workspace)


def _kv4_shared_attn(dev, q, cache, block_table, lens, cu, group_cu, shared_lens, mask, max_shared, max_own, softmax_scale, out, lse, workspace):
    T, H, d = q.shape
    R, c = lens.shape[0], cache.c_struct
    assert d == c.d and cache.device == dev, "the cache has another head size, or lies elsewhere"
    table, stride, width = _table(block_table, dev, R)
    S, group_at, shared_at = _groups(group_cu, shared_lens, dev)
    most = width * c.page
    max_shared, max_own = most if max_shared is None else max(1, max_shared), most if max_own is None else max(1, max_own)
    packed = _packed(q, dev, T, H, d)
    out, to = _out(out, q, dev, T, H, d)
    lse, lse_at = _lse_out(lse, q, dev, H, T)
    if workspace is None:
        need = bbm_kv4_shared_attn_workspace_bytes(T, R, S, H, c.Hk, d, max_shared, max_own)
        workspace = q.new_empty(need, dtype=torch.uint8) if need else None
    keep = _I64x6(*packed, *to)
    at = _address(keep)
    _check(lib.bbm_kv4_shared_attn(at, at + 24, lse_at, T, R, _ints(cu, dev, R + 1), _ints(lens, dev, R), table, stride, width, S, group_at, shared_at, *_mask(mask, dev, T),
                                   _address(c), H, d ** -0.5 if softmax_scale is None else softmax_scale, max_shared, max_own, *_workspace(workspace, dev), _here(dev)))
    return out, lse


def kv4_weights(cache: KV4Cache) -> torch.Tensor:
    """What each token and key head of the cache has gathered before anything looked at it: zeros, fp32 [pages, Hk, page]."""
    pages, Hk, page = cache.k.shape[:3]
    return torch.zeros((pages, Hk, page), dtype=torch.float32, device=cache.k.device)


def _weights(x: torch.Tensor, cache: KV4Cache) -> int:
    assert x.dtype is torch.float32 and x.is_contiguous() and x.shape == cache.k.shape[:3], "contiguous fp32 weights [pages, Hk, page] of the cache"
    assert x.get_device() == cache.device, "the tensors of a call lie on one GPU"
    return x.data_ptr()


def bbm_kv4_weights(q: torch.Tensor, lse: torch.Tensor, cache: KV4Cache, block_table: torch.Tensor, lens: torch.Tensor, cu: torch.Tensor, weights: torch.Tensor,
                    group_cu: Optional[torch.Tensor] = None, shared_lens: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None, decay: float = 1.0,
                    out: Optional[torch.Tensor] = None, max_shared: Optional[int] = None, max_own: Optional[int] = None, softmax_scale: Optional[float] = None,
                    stream=None) -> torch.Tensor:
    """Adds to decay * weights (fp32 [pages, Hk, page], see kv4_weights) the probabilities which the step's queries gave to their keys, from the lse of the step's
    attention; the other arguments are those of bbm_kv4_shared_attn.  Writes out (None: weights themselves), of which only the requests' keys change, and returns it."""
    dev = _gpu(q)
    if _elsewhere(dev, stream):
        with _context(dev, stream):
            return _kv4_weights(dev, q, lse, cache, block_table, lens, cu, weights, group_cu, shared_lens, mask, decay, out, max_shared, max_own, softmax_scale)
    return _kv4_weights(dev, q, lse, cache, block_table, lens, cu, weights, group_cu, shared_lens, mask, decay, out, max_shared, max_own, softmax_scale)


def _kv4_weights(dev, q, lse, cache, block_table, lens, cu, weights, group_cu, shared_lens, mask, decay, out, max_shared, max_own, softmax_scale):
    T, H, d = q.shape
    R, c = lens.shape[0], cache.c_struct
    assert d == c.d and cache.device == dev, "the cache has another head size, or lies elsewhere"
    table, stride, width = _table(block_table, dev, R)
    S, group_at, shared_at = _groups(group_cu, shared_lens, dev)
    most = width * c.page
    max_shared, max_own = most if max_shared is None else max(1, max_shared), most if max_own is None else max(1, max_own)
    out = weights if out is None else out
    keep = _I64x6(*_packed(q, dev, T, H, d), 0, 0, 0)
    _check(lib.bbm_kv4_weights(_address(keep), _lse(lse, dev, H, T), T, R, _ints(cu, dev, R + 1), _ints(lens, dev, R), table, stride, width, S, group_at, shared_at, *_mask(mask, dev, T),
                               _address(c), H, d ** -0.5 if softmax_scale is None else softmax_scale, decay, _weights(weights, cache), _weights(out, cache), max_shared, max_own, _here(dev)))
    return out


@dataclass
class Evicted:
    """What bbm_kv4_evict writes besides the cache (int32 device tensors)."""
    lens: torch.Tensor                   # [R] tokens of each request in the cache
    free_next: Optional[torch.Tensor]    # [1] index of the next free page of the list, for the next bbm_build_slots; None without a list


def bbm_kv4_evict_workspace_bytes(R: int, Hk: int, max_keys: int) -> int:
    return int(lib.bbm_kv4_evict_workspace_bytes(R, Hk, max_keys))


def bbm_kv4_evict(cache: KV4Cache, weights: torch.Tensor, block_table: torch.Tensor, lens: torch.Tensor, budget: int, recent: int = 0, first: Optional[torch.Tensor] = None,
                  free_pages: Optional[torch.Tensor] = None, free_at: Optional[torch.Tensor] = None, max_len: Optional[int] = None, new_lens: Optional[torch.Tensor] = None,
                  workspace: Optional[torch.Tensor] = None, stream=None) -> Evicted:
    """Thins requests of more than `budget` keys to that many, for each key head those of largest weight beside the first[r] (int32 [R]) and the last `recent` ones, in place;
    the pages that this frees go back to free_pages (int32 [n]) in front of free_at (int32 [1]).  max_len: an upper bound of lens (None: what the table holds).  Later tokens are
    turned (bbm_rope) by the positions of bbm_build_slots plus the sums of lens - Evicted.lens."""
    dev = _gpu(lens)
    if _elsewhere(dev, stream):
        with _context(dev, stream):
            return _kv4_evict(dev, cache, weights, block_table, lens, budget, recent, first, free_pages, free_at, max_len, new_lens, workspace)
    return _kv4_evict(dev, cache, weights, block_table, lens, budget, recent, first, free_pages, free_at, max_len, new_lens, workspace)


def _kv4_evict(dev, cache, weights, block_table, lens, budget, recent, first, free_pages, free_at, max_len, new_lens, workspace):
    R, c = lens.shape[0], cache.c_struct
    assert cache.device == dev, "the cache lies elsewhere"
    table, stride, width = _table(block_table, dev, R)
    assert (free_pages is None) == (free_at is None), "a list of free pages and its index"
    # (one allocation for what the call gives and what it needs)
    need = 0 if workspace is not None else -(-lib.bbm_kv4_evict_workspace_bytes(R, c.Hk, width * c.page) // 16) * 4
    own, lens_out, free_next = torch.split_with_sizes(lens.new_empty(need + R + 1), (need, R, 1))
    workspace = own if workspace is None else workspace
    new_lens = lens_out if new_lens is None else new_lens
    free_next = None if free_at is None else free_next
    free = (None, 0, None, None) if free_at is None else (_ints(free_pages, dev), free_pages.shape[0], _ints(free_at, dev, 1), free_next.data_ptr())
    _check(lib.bbm_kv4_evict(_address(c), _weights(weights, cache), R, _ints(lens, dev), table, stride, width, budget, recent, None if first is None else _ints(first, dev, R),
                             _ints(new_lens, dev, R), *free, width * c.page if max_len is None else max(1, max_len), *_workspace(workspace, dev), _here(dev)))
    return Evicted(new_lens, free_next)
