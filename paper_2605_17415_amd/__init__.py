"""IVF-TQ hot path for AMD MI355X: HIP kernels behind a C ABI, plus a thin ctypes binding."""
from .binding import (ALLOC_FN, FREE_FN, Index, IvftqError, declared_symbols, ivftq_build_codebook,  # noqa: F401
                      ivftq_build_refined_codebook, ivftq_build_coarsened_codebook,
                      ivftq_haar_from_gaussian, ivftq_haar_rotation, ivftq_measure_mfma_rate, ivftq_quantiser_grid, ivftq_rerank, ivftq_version,
                      load_library)

_KV = ("KVCache", "declared_kv_symbols", "kv_append", "kv_attend", "kv_compact", "kv_copy", "kv_fork", "kv_free", "kv_page_bytes", "kv_read",
       "kv_reserve", "kv_trim")


def __getattr__(name):
    """The key-value cache's calls take torch tensors and nothing else: torch is imported with the first of them."""
    if name in _KV:
        from . import kv
        globals().update({n: getattr(kv, n) for n in _KV})
        return globals()[name]
    raise AttributeError(f"module {__name__!r} has no attribute {name!r}")
