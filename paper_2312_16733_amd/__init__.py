"""MI355X-native SubNetAct forward path: Python binding over libsubnetact.so.

Argument marshalling only; every step of the path runs in the HIP kernels behind
the C ABI declared in include/subnetact.h.  Importing this package does not load
the library; the first call does, and fails loudly if it has not been built.
"""
from .binding import (ArchDesc, SubnetCfgC, Supernet, lib, library_path, arch_desc_from_spec,
                      tensor_infos, norm_infos, pack_weights, pack_stats, cfg_to_c,
                      supernet_load, subnet_forward, SnaError)

__all__ = ["ArchDesc", "SubnetCfgC", "Supernet", "lib", "library_path", "arch_desc_from_spec",
           "tensor_infos", "norm_infos", "pack_weights", "pack_stats", "cfg_to_c",
           "supernet_load", "subnet_forward", "SnaError"]

# Autoregressive serving: needs torch, which the rest of the package does not, and so comes when it is asked for by name
_SERVING = ("PagedCache", "PagedBatch", "kv_append", "paged_attention", "verify_draft")


def __getattr__(name):
    if name in _SERVING:
        from . import serving
        for n in _SERVING:
            globals()[n] = getattr(serving, n)
        return globals()[name]
    raise AttributeError(f"module {__name__!r} has no attribute {name!r}")


def __dir__():
    return sorted({*globals(), *_SERVING})
