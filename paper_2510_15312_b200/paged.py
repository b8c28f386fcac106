"""Operators on a cache kept in pages, on torch tensors: slots, rotary append, tree attention and sampled verification
(include/sdv.h says what each computes).  Argument checks, allocation of outputs and the calls are csrc/paged_torch.cpp's; the work is queued on
the current stream, or on `stream`, and the calls return at once.  All tensors are on the current device; index arrays are int32.  What the tensors' shapes and types
do not allow raises ValueError, what the library refuses SdvError.  Outputs not passed in are allocated by torch, on the stream the
work is queued on; the vectors that one call returns share an allocation.  Results carry no gradients; given tensors that
a call writes to count as changed in place."""
from __future__ import annotations

import ctypes as C
import math
from typing import Optional

from . import binding
from .binding import EINVAL, SdvError
from .build import build_torch_calls

_calls = None   # the module of csrc/paged_torch.cpp, once it has the library's entry points


def _load():
    global _calls
    if _calls is None:
        import torch   # (contexts and the library do without)
        if not torch.cuda.is_available():
            raise SdvError(binding.ECUDA, "no CUDA device (there is no CPU fallback)")
        torch.cuda.init()
        library = binding.lib()
        build_torch_calls()
        from . import _paged
        _paged.bind(*(C.cast(getattr(library, "sdv_" + n), C.c_void_p).value for n in ("paged_slots", "rope_append", "tree_attention_workspace_bytes", "tree_attention", "tree_attention_fresh", "verify_sampled")))
        _calls = _paged
    return _calls


def _on(stream, name, *args):
    import torch
    with torch.cuda.stream(stream):
        return getattr(_calls, name)(*args)


def _fail(rc: int, where: str):
    raise SdvError(rc, where)


def paged_slots(kv_len, cu_rows, block_table, n_held, free_pages, free_state, page_size: int, n_rows: int, parent=None, out=None, stream=None):
    """Hands pages to the sequences that need more and gives every row its slot and position: (slots, positions, n_held, free_state) after the call;
    block_table [sequences][width] is updated in place.  free_state[0] is the first unused entry of free_pages; of the returned one, the second entry is the number of
    sequences that were refused for want of pages (their slots are -1).  With parent, at most 262144 rows.  out: the four tensors to write to."""
    calls = _calls or _load()
    args = (kv_len, cu_rows, block_table, n_held, free_pages, free_state, page_size, n_rows, parent, out if out is None else tuple(out))
    r = calls.paged_slots(*args) if stream is None else _on(stream, "paged_slots", *args)
    return r if type(r) is tuple else _fail(r, "sdv_paged_slots")


def rope_frequencies(rot_dim: int, theta: float = 1.0e4, scaling: Optional[str] = None, factor: float = 1.0, original_positions: int = 8192, low: float = 1.0, high: float = 4.0,
                     fast: float = 32.0, slow: float = 1.0):
    """(angles per position of the rot_dim / 2 pairs as a list of floats, factor on cosine and sine) for rope_append.
      None      theta^(-2i / rot_dim)
      "linear"  divided by `factor`
      "banded"  by the turns a pair makes within the original positions: up to `low` divided by `factor`, from `high` on kept, a straight line between
      "yarn"    Peng et al. 2023 (arXiv 2309.00071): the line is in the pair's number, between those that turn `fast` and `slow` times; cosine and
                sine grow by 0.1 ln(factor) + 1"""
    if rot_dim < 2 or rot_dim % 2 or not theta > 0 or not factor > 0 or original_positions < 1:
        raise ValueError("rope_frequencies: an even rot_dim, positive theta and factor expected")
    f = [theta ** (-2.0 * i / rot_dim) for i in range(rot_dim // 2)]
    if scaling is None:
        return f, 1.0
    if scaling == "linear":
        return [x / factor for x in f], 1.0
    if scaling == "banded":
        if not high > low:
            raise ValueError("rope_frequencies: high > low expected")
        keep = [min(1.0, max(0.0, (original_positions * x / (2 * math.pi) - low) / (high - low))) for x in f]
        return [x / factor * (1 - k) + x * k for x, k in zip(f, keep)], 1.0
    if scaling == "yarn":
        if theta == 1.0:
            raise ValueError("rope_frequencies: theta other than 1 expected")
        pair = lambda turns: rot_dim * math.log(original_positions / (turns * 2 * math.pi)) / (2 * math.log(theta))  # noqa: E731
        first, last = max(math.floor(pair(fast)), 0), min(math.ceil(pair(slow)), rot_dim - 1)
        gone = [min(1.0, max(0.0, (i - first) / max(last - first, 0.001))) for i in range(rot_dim // 2)]
        return [x / factor * g + x * (1 - g) for x, g in zip(f, gone)], (0.1 * math.log(factor) + 1.0 if factor > 1 else 1.0)
    raise ValueError(f"rope_frequencies: unknown scaling {scaling!r}")


def rope_append(positions, frequencies, q=None, k=None, v=None, k_pages=None, v_pages=None, slots=None, interleaved: bool = False, factor: float = 1.0, q_out=None,
                stream=None):
    """Rotates q [rows][query heads][head dim] and k [rows][KV heads][head dim] by positions [rows] (int32) times frequencies [rot_dim / 2] (float64); k and v go to their
    slots of the pages [pages][KV heads][page size][head dim] (any strides with contiguous head elements), a row whose slot is outside the pool is not written.  q, or k, v,
    the pages and slots, may be left out.  Returns the rotated q (q_out; may be q itself), None without q."""
    calls = _calls or _load()
    args = (positions, frequencies, q, k, v, k_pages, v_pages, slots, interleaved, factor, q_out)
    r = calls.rope_append(*args) if stream is None else _on(stream, "rope_append", *args)
    return r[0] if type(r) is tuple else _fail(r, "sdv_rope_append")


def tree_attention_workspace(n_seqs: int, head_dim: int):
    """A workspace for tree_attention on the current device, for up to n_seqs sequences."""
    import torch
    _load()
    n = binding.lib().sdv_tree_attention_workspace_bytes(n_seqs, head_dim)
    if n == 0:
        raise SdvError(EINVAL, "sdv_tree_attention_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device="cuda")


def tree_attention(q, k_pages, v_pages, block_table, kv_len, cu_rows, parent=None, scale: Optional[float] = None, out=None, workspace=None, status=None, stream=None):
    """Every row of q [rows][query heads][head dim] attends to the kv_len[b] committed tokens of its sequence and to the rows on its own path through
    the draft tree, whose keys and values were appended before.  scale: 1 / sqrt(head dim) unless given.  A sequence has at
    most 64 rows here.  out: like q; rows past the 64th of a sequence and rows of no sequence are left as they were; without one, the first are NaN and the others zeros.  workspace: see
    tree_attention_workspace; without one torch allocates it for the call.  status: int32 [1], set to 1 when a wait inside the kernel ran out."""
    calls = _calls or _load()
    args = (q, k_pages, v_pages, block_table, kv_len, cu_rows, parent, scale, out, workspace, status)
    r = calls.tree_attention(*args) if stream is None else _on(stream, "tree_attention", *args)
    return r[0] if type(r) is tuple else _fail(r, "sdv_tree_attention")


def verify_sampled(target_probs, tokens, cu_rows, uniforms, draft_probs=None, parent=None, slots=None, out=None, stream=None):
    """Accepts drafted tokens against the target's probabilities [rows][vocab] (float32) with the uniform random numbers uniforms [rows] and draws one
    token behind the accepted ones: (accept_len [sequences], tokens [rows], rows [rows], slots [rows] or None).  draft_probs [rows][vocab]: what each draft of a chain was sampled from; without, drafts
    count as certain (retrieved), and parent may make them trees.  slots: every row's slot, for the slots that accepted rows move to.  A sequence
    without rows has accept_len -1, also when no sequence has any.  out: the tensors to write to."""
    calls = _calls or _load()
    args = (target_probs, tokens, cu_rows, uniforms, draft_probs, parent, slots, out if out is None else tuple(out))
    r = calls.verify_sampled(*args) if stream is None else _on(stream, "verify_sampled", *args)
    return r if type(r) is tuple else _fail(r, "sdv_verify_sampled")
