"""sdv: the verify path of retrieval-based greedy speculative decoding on one B200.

Python binding of the C-ABI library declared in include/sdv.h: argument marshalling only,
every step of the path runs in the library's CUDA kernels.  Beside the contexts (Sdv) stand operators on plain device
tensors: gemm_noalloc, and those on a cache kept in pages (paged.py).  PyTorch is used for device memory
and streams.  There is no CPU fallback: importing works without a GPU, creating a context
does not.
"""
from .binding import (SdvError, Sdv, SdvConfig, lib, load_library, EXPORTS, OK, EINVAL, ENOMEM, ECAPACITY,
                      ESTATE, ECUDA, ETIMEOUT, ETOOBIG, gemm_noalloc)
from .paged import paged_slots, rope_append, rope_frequencies, tree_attention, tree_attention_workspace, verify_sampled

__all__ = ["SdvError", "Sdv", "SdvConfig", "lib", "load_library", "EXPORTS", "OK", "EINVAL", "ENOMEM",
           "ECAPACITY", "ESTATE", "ECUDA", "ETIMEOUT", "ETOOBIG", "gemm_noalloc", "paged_slots", "rope_append", "rope_frequencies", "tree_attention",
           "tree_attention_workspace", "verify_sampled"]
