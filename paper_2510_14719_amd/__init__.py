"""MI355X-native fused attention forward (gfx950 HIP kernels behind a C ABI).

``attn_fwd`` and friends live in :mod:`paper_2510_14719_amd.binding`, the operators
around a paged cache of keys and values in :mod:`paper_2510_14719_amd.kv_cache`; they are
imported lazily so that the input generators can be used on a machine that has
no built library.
"""

_KV_CACHE = ["attn_paged", "attn_paged_workspace", "rope", "rope_frequencies", "kv_append", "kv_reserve", "kv_free", "kv_fork", "kv_compact",
             "kv_compact_workspace", "kv_copy_pages", "KvCacheError"]
__all__ = ["attn_fwd", "attn_fwd_f16", "attn_fwd_bf16", "attn_fwd_fp8", "AttnFwdError", "load_library"] + _KV_CACHE


def __getattr__(name):
    if name in _KV_CACHE:
        from . import kv_cache
        return getattr(kv_cache, name)
    if name in __all__:
        from . import binding
        return getattr(binding, name)
    raise AttributeError(name)
