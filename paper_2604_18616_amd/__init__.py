"""MI355X-native operators of language models: flash-attention forward, bf16 GEMM, FP8 MoE feed-forward, rotary positions and a
quantised paged cache with attention over it.  HIP kernels behind a C ABI plus a thin binding.

``attn_fwd``, ``gemm_bf16``, ``moe_ffn_fp8``, ``rope_bf16`` and ``kv_fp8_write``, ``kv_fp8_read``, ``attn_kv_fp8`` (from
:mod:`.binding`) marshal device pointers into the C-ABI library built from ``csrc/``; every step of the computation runs in the
HIP kernels.  :mod:`.inputs` generates the seeded synthetic workloads.
"""

import sys

__all__ = ["attn_fwd", "gemm_bf16", "moe_ffn_fp8", "rope_bf16", "rope_frequencies", "KvFp8Cache", "kv_fp8_cache", "kv_fp8_write", "kv_fp8_read", "attn_kv_fp8",
           "load_library", "build_library", "inputs"]

_OF_BINDING = ("attn_fwd", "gemm_bf16", "moe_ffn_fp8", "moe_workspace_bytes", "load_library", "attn_fwd_flops", "rope_bf16", "rope_frequencies",
               "KvFp8Cache", "kv_fp8_cache", "kv_fp8_write", "kv_fp8_read", "attn_kv_fp8", "strerror", "version", "AttnError")


class _Name:
    """A name of the binding, which is imported with the first one.  It is looked up there each time, so that what a program puts
    in a function's place is found through the package too.  (A descriptor, because a module's __getattr__ is only asked after
    the lookup has failed: 0.6 us in place of 0.2, where a small call takes 5.)"""

    def __init__(self, name):
        self.name = name

    def __get__(self, package, owner=None):
        try:
            return getattr(binding, self.name)
        except NameError:
            from . import binding as first_time             # (which makes it a name of this module)
            return getattr(first_time, self.name)


sys.modules[__name__].__class__ = type("_Package", (type(sys),), {name: _Name(name) for name in _OF_BINDING})


def __getattr__(name):
    if name == "build_library":
        from .build import build_library
        return build_library
    raise AttributeError(name)
