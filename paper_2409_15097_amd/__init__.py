"""Binary Block Masking flash attention (forward and backward) for AMD MI355X: thin Python binding over libbbm.so.

The names below are those of the C ABI (include/bbm.h, bbm_tokens.h, bbm_cache.h); the functions only marshal arguments: device memory and the
stream come from PyTorch, every computation runs in the library's HIP kernels.  There is no CPU fallback: the
binding is loaded at the first use of any of these names and raises ImportError if the library is not built (the
package itself imports without it, so that `python -m paper_2409_15097_amd.build` can build it).
"""
_NAMES = (
    "BBM_MODE_BITMAP", "BBM_MODE_RUNS", "BBM_MODE_LIST", "BBM_MODE_DENSE_BASELINE", "BBM_MODE_AUTO",
    "BBM_OK", "BBM_EINVAL", "BBM_EUNSUPPORTED", "BBM_EWORKSPACE", "BBM_EHIP",
    "BbmError", "BlockIndex", "lib", "library_path",
    "bbm_last_error", "bbm_version", "bbm_build_block_mask", "bbm_build_block_mask_rect", "bbm_attn_fwd_rect",
    "bbm_attn_fwd_static", "bbm_build_runs", "bbm_build_sparse_index", "bbm_build_index", "bbm_build_col_index",
    "bbm_col_sched_bytes", "bbm_attn_bwd_workspace_bytes", "bbm_attn_bwd", "bbm_attn_fwd_workspace_bytes", "bbm_attn_fwd",
    "bbm_sched_bytes", "build_index", "bf16_from_bits", "bbm_rcm_workspace_bytes", "bbm_rcm_order", "bbm_permute_mask",
    "bbm_gather_rows", "bbm_probe_mfma_bf16", "bbm_probe_mfma_bf16_flop",
)
# operators on packed tokens (include/bbm_tokens.h)
_TOKEN_NAMES = (
    "Slots", "KV4Cache", "kv4_cache", "rope_freqs", "bbm_build_slots", "bbm_rope", "bbm_prompt_attn_fwd",
    "bbm_prompt_attn_bwd_workspace_bytes", "bbm_prompt_attn_bwd", "bbm_kv4_append", "bbm_kv4_read", "bbm_kv4_attn_workspace_bytes", "bbm_kv4_attn",
)
# operators on the cache of many and long answers (include/bbm_cache.h)
_CACHE_NAMES = ("bbm_kv4_shared_attn_workspace_bytes", "bbm_kv4_shared_attn", "kv4_weights", "bbm_kv4_weights", "Evicted", "bbm_kv4_evict_workspace_bytes",
                "bbm_kv4_evict")
__all__ = list(_NAMES + _TOKEN_NAMES + _CACHE_NAMES)


def __getattr__(name):
    if name in _NAMES:
        from . import binding          # loads libbbm.so; ImportError if it is not built
        value = getattr(binding, name)
        globals()[name] = value
        return value
    if name in _TOKEN_NAMES:
        from . import tokens
        value = getattr(tokens, name)
        globals()[name] = value
        return value
    if name in _CACHE_NAMES:
        from . import cache
        value = getattr(cache, name)
        globals()[name] = value
        return value
    raise AttributeError(f"module {__name__!r} has no attribute {name!r}")


def __dir__():
    return sorted(list(globals()) + list(_NAMES + _TOKEN_NAMES + _CACHE_NAMES))
