"""Operators on a cache kept in pages, on torch tensors: slots, rotary append, tree attention and sampled verification
(include/sdv.h says what each computes).  Argument marshalling only; the work is queued on the current stream, or on `stream`,
and the calls return at once.  All tensors are on the current device; index arrays are int32.  What the tensors' shapes and types
do not allow raises ValueError, what the library refuses SdvError.  Outputs not passed in are allocated by torch, on the stream the
work is queued on."""
from __future__ import annotations

import contextlib
import ctypes as C
import math
from typing import Optional, Tuple

from . import binding
from .binding import EINVAL, OK, SdvError

_vp, _i, _ll, _f = C.c_void_p, C.c_int, C.c_longlong, C.c_float


class _Pages(C.Structure):
    _fields_ = [("k", _vp), ("v", _vp)] + [(n, _i) for n in ("dtype", "n_pages", "page_size", "n_kv_heads", "head_dim")] + \
               [(n, _ll) for n in ("page_stride", "head_stride", "token_stride")]


class _SlotsArgs(C.Structure):
    _fields_ = [(n, _vp) for n in ("kv_len", "cu_rows", "parent", "n_held", "free_pages", "free_state", "block_table", "slots", "positions",
                                   "n_held_out", "free_state_out")] + [("table_stride", _ll)] + \
               [(n, _i) for n in ("n_seqs", "n_rows", "page_size", "table_width", "n_free")]


class _RopeArgs(C.Structure):
    _fields_ = [(n, _vp) for n in ("q", "k", "v", "q_out", "positions", "slots", "frequencies")] + \
               [(n, _ll) for n in ("q_row_stride", "q_head_stride", "out_row_stride", "out_head_stride", "k_row_stride", "k_head_stride",
                                   "v_row_stride", "v_head_stride")] + \
               [(n, _i) for n in ("n_rows", "n_q_heads", "n_kv_heads", "head_dim", "rot_dim", "interleaved", "dtype")] + [("factor", _f)]


class _AttentionArgs(C.Structure):
    _fields_ = [(n, _vp) for n in ("q", "out", "block_table", "kv_len", "cu_rows", "parent", "workspace", "status")] + [("workspace_bytes", C.c_size_t)] + \
               [(n, _ll) for n in ("q_row_stride", "q_head_stride", "out_row_stride", "out_head_stride", "table_stride")] + \
               [(n, _i) for n in ("n_seqs", "n_rows", "n_q_heads", "table_width")] + [("scale", _f)]


class _VerifyArgs(C.Structure):
    _fields_ = [(n, _vp) for n in ("target", "draft", "tokens", "cu_rows", "parent", "slots", "uniforms", "accept_len", "out_tokens", "out_rows",
                                   "out_slots")] + [("target_stride", _ll), ("draft_stride", _ll)] + [(n, _i) for n in ("n_seqs", "n_rows", "vocab")]


_types = None   # torch dtype -> SDV_BF16 / SDV_FP16


def _dtype(t, what: str) -> int:
    global _types
    if _types is None:
        import torch
        _types = {torch.bfloat16: 0, torch.float16: 1}
    d = _types.get(t.dtype)
    if d is None:
        raise ValueError(f"{what}: bfloat16 or float16 expected, got {t.dtype}")
    return d


def _index(t, shape: Tuple[int, ...], what: str, device: int) -> int:
    """Address of a contiguous int32 tensor of this shape on the device."""
    import torch
    if t.dtype is not torch.int32 or t.get_device() != device or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{what}: contiguous int32 tensor of shape {tuple(shape)} on the current device expected")
    return t.data_ptr()


def _on(t, device: int, what: str):
    if t.get_device() != device:
        raise ValueError(f"{what}: not on the current CUDA device")


def _enter(stream):
    """(torch, current device, handle of the stream, context in which outputs are allocated)."""
    import torch
    if not torch.cuda.is_available():
        raise SdvError(binding.ECUDA, "no CUDA device (there is no CPU fallback)")
    device = torch.cuda.current_device()
    if stream is not None:
        return torch, device, stream.cuda_stream, torch.cuda.stream(stream)
    try:
        s = torch._C._cuda_getCurrentRawStream(device)
    except AttributeError:
        s = torch.cuda.current_stream().cuda_stream
    return torch, device, s, contextlib.nullcontext()


def _check(rc: int, where: str):
    if rc != OK:
        raise SdvError(rc, where)


def _pool(k_pages, v_pages, device: int) -> _Pages:
    """[pages][KV heads][tokens of a page][head dim], any strides with contiguous head elements (a pool that keeps the
    tokens outside the heads is passed as .transpose(1, 2))."""
    if k_pages.ndim != 4 or v_pages.shape != k_pages.shape or v_pages.dtype != k_pages.dtype or v_pages.stride() != k_pages.stride():
        raise ValueError("k_pages and v_pages: two tensors [pages][KV heads][page size][head dim] of the same shape, strides and type expected")
    _on(k_pages, device, "k_pages")
    _on(v_pages, device, "v_pages")
    n, heads, page, dim = k_pages.shape
    s0, s1, s2, s3 = k_pages.stride()
    if s3 != 1 and dim > 1:
        raise ValueError("k_pages: the elements of a head have to be contiguous")
    # the stride of a dimension of one says nothing
    return _Pages(k_pages.data_ptr(), v_pages.data_ptr(), _dtype(k_pages, "k_pages"), n, page, heads, dim, s0 if n > 1 else 0, s1 if heads > 1 else 0, s2 if page > 1 else 0)


def _rows(t, heads_dim, what: str, device: int):
    """Row and head stride of a tensor [rows][heads][head dim]."""
    if t.ndim != 3:
        raise ValueError(f"{what}: [rows][heads][head dim] expected")
    _on(t, device, what)
    if t.shape[2] > 1 and t.stride(2) != 1:
        raise ValueError(f"{what}: the elements of a head have to be contiguous")
    if heads_dim is not None and (t.shape != heads_dim[0] or t.dtype != heads_dim[1]):
        raise ValueError(f"{what}: shape {tuple(heads_dim[0])} of {heads_dim[1]} expected")
    return (t.stride(0) if t.shape[0] > 1 else 0), (t.stride(1) if t.shape[1] > 1 else 0)


def paged_slots(kv_len, cu_rows, block_table, n_held, free_pages, free_state, page_size: int, n_rows: int, parent=None, out=None, stream=None):
    """Hands pages to the sequences that need more and gives every row its slot and position: (slots, positions, n_held, free_state) after the call;
    block_table [sequences][width] is updated in place.  free_state[0] is the first unused entry of free_pages; of the returned one, the second entry is the number of
    sequences that were refused for want of pages (their slots are -1).  out: the four tensors to write to."""
    torch, dev, s, alloc = _enter(stream)
    n = kv_len.shape[0]
    if block_table.ndim != 2 or block_table.shape[0] != n or block_table.dtype is not torch.int32 or (block_table.shape[1] > 1 and block_table.stride(1) != 1):
        raise ValueError("block_table: int32 [sequences][width] with contiguous rows expected")
    _on(block_table, dev, "block_table")
    n_rows = int(n_rows)
    if n_rows < 0 or free_state.ndim != 1 or free_state.shape[0] < 1:
        raise ValueError("paged_slots: n_rows >= 0 and a free_state of at least one entry expected")
    if out is None:
        with alloc:
            both = torch.empty((2, n_rows), dtype=torch.int32, device=kv_len.device)
            held = torch.empty(n + 2, dtype=torch.int32, device=kv_len.device)
        out = (both[0], both[1], held[:n], held[n:])
    slots, positions, held, free = out
    a = _SlotsArgs(_index(kv_len, (n,), "kv_len", dev), _index(cu_rows, (n + 1,), "cu_rows", dev), None if parent is None else _index(parent, (n_rows,), "parent", dev),
                   _index(n_held, (n,), "n_held", dev), _index(free_pages, (free_pages.numel(),), "free_pages", dev), _index(free_state, free_state.shape, "free_state", dev),
                   block_table.data_ptr(), _index(slots, (n_rows,), "slots", dev), _index(positions, (n_rows,), "positions", dev), _index(held, (n,), "n_held (out)", dev),
                   _index(free, (2,), "free_state (out)", dev), block_table.stride(0) if n > 1 else block_table.shape[1], n, n_rows, page_size, block_table.shape[1],
                   free_pages.numel())
    _check(binding.lib().sdv_paged_slots(C.byref(a), s), "sdv_paged_slots")
    return slots, positions, held, free


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
    slots of the pages, a row whose slot is outside the pool is not written.  q, or k, v, the pages and slots, may be left out.  Returns the rotated q (q_out; may be q
    itself), None without q."""
    torch, dev, s, alloc = _enter(stream)
    n = positions.shape[0]
    if frequencies.dtype is not torch.float64 or frequencies.ndim != 1 or not frequencies.is_contiguous():
        raise ValueError("frequencies: contiguous float64 [rot_dim / 2] expected")
    _on(frequencies, dev, "frequencies")
    first = q if q is not None else k
    if first is None or (k is None) != (v is None):
        raise ValueError("rope_append: q, or k and v, expected")
    a = _RopeArgs(positions=_index(positions, (n,), "positions", dev), frequencies=frequencies.data_ptr(), n_rows=n, head_dim=first.shape[-1], rot_dim=2 * frequencies.shape[0],
                  interleaved=bool(interleaved), dtype=_dtype(first, "q" if q is not None else "k"), factor=factor)
    pages = None
    if q is not None:
        a.q_row_stride, a.q_head_stride = _rows(q, None, "q", dev)
        if q.shape[0] != n:
            raise ValueError("q: as many rows as positions expected")
        if q_out is None:
            with alloc:
                q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        a.out_row_stride, a.out_head_stride = _rows(q_out, (q.shape, q.dtype), "q_out", dev)
        a.q, a.q_out, a.n_q_heads = q.data_ptr(), q_out.data_ptr(), q.shape[1]
    if k is not None:
        if k_pages is None or v_pages is None or slots is None:
            raise ValueError("rope_append: k and v need k_pages, v_pages and slots")
        pages = _pool(k_pages, v_pages, dev)
        shape = torch.Size((n, pages.n_kv_heads, pages.head_dim))
        a.k_row_stride, a.k_head_stride = _rows(k, (shape, k_pages.dtype), "k", dev)
        a.v_row_stride, a.v_head_stride = _rows(v, (shape, k_pages.dtype), "v", dev)
        a.k, a.v, a.slots, a.n_kv_heads = k.data_ptr(), v.data_ptr(), _index(slots, (n,), "slots", dev), pages.n_kv_heads
        if q is not None and (q.dtype != k.dtype or q.shape[2] != k.shape[2]):
            raise ValueError("rope_append: q and k of one type and head dim expected")
    if n:
        _check(binding.lib().sdv_rope_append(C.byref(a), None if pages is None else C.byref(pages), s), "sdv_rope_append")
    return q_out if q is not None else None


def tree_attention_workspace(n_seqs: int, head_dim: int):
    """A workspace for tree_attention on the current device, for up to n_seqs sequences."""
    import torch
    _enter(None)
    n = binding.lib().sdv_tree_attention_workspace_bytes(n_seqs, head_dim)
    if n == 0:
        raise SdvError(EINVAL, "sdv_tree_attention_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device="cuda")


def tree_attention(q, k_pages, v_pages, block_table, kv_len, cu_rows, parent=None, scale: Optional[float] = None, out=None, workspace=None, status=None, stream=None):
    """Every row of q [rows][query heads][head dim] attends to the kv_len[b] committed tokens of its sequence and to the rows on its own path through
    the draft tree, whose keys and values were appended before.  scale: 1 / sqrt(head dim) unless given.  out: like q; rows of no sequence are left as they were.  workspace: see
    tree_attention_workspace; without one torch allocates it for the call.  status: int32 [1], set to 1 when a wait inside the kernel ran out."""
    torch, dev, s, alloc = _enter(stream)
    pages = _pool(k_pages, v_pages, dev)
    n, heads, dim = q.shape if q.ndim == 3 else (0, 0, 0)
    q_row, q_head = _rows(q, None, "q", dev)
    if q.dtype != k_pages.dtype or dim != pages.head_dim:
        raise ValueError("q: type and head dim of the pages expected")
    seqs = kv_len.shape[0]
    if block_table.ndim != 2 or block_table.shape[0] != seqs or block_table.dtype is not torch.int32 or (block_table.shape[1] > 1 and block_table.stride(1) != 1):
        raise ValueError("block_table: int32 [sequences][width] with contiguous rows expected")
    _on(block_table, dev, "block_table")
    lib = binding.lib()
    with alloc:
        if out is None:
            out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        if workspace is None:
            workspace = torch.empty(lib.sdv_tree_attention_workspace_bytes(seqs, dim), dtype=torch.uint8, device=q.device)
    out_row, out_head = _rows(out, (q.shape, q.dtype), "out", dev)
    _on(workspace, dev, "workspace")
    if n == 0 or seqs == 0:
        return out
    a = _AttentionArgs(q.data_ptr(), out.data_ptr(), block_table.data_ptr(), _index(kv_len, (seqs,), "kv_len", dev), _index(cu_rows, (seqs + 1,), "cu_rows", dev),
                       None if parent is None else _index(parent, (n,), "parent", dev), workspace.data_ptr(),
                       None if status is None else _index(status, (1,), "status", dev), workspace.numel() * workspace.element_size(), q_row, q_head, out_row, out_head,
                       block_table.stride(0) if seqs > 1 else block_table.shape[1], seqs, n, heads, block_table.shape[1], dim ** -0.5 if scale is None else scale)
    _check(lib.sdv_tree_attention(C.byref(a), C.byref(pages), s), "sdv_tree_attention")
    return out


def verify_sampled(target_probs, tokens, cu_rows, uniforms, draft_probs=None, parent=None, slots=None, out=None, stream=None):
    """Accepts drafted tokens against the target's probabilities [rows][vocab] (float32) with the uniform random numbers uniforms [rows] and draws one
    token behind the accepted ones: (accept_len [sequences], tokens [rows], rows [rows], slots [rows] or None).  draft_probs [rows][vocab]: what each draft of a chain was sampled from; without, drafts
    count as certain (retrieved), and parent may make them trees.  slots: every row's slot, for the slots that accepted rows move to.  out: the tensors to write to."""
    torch, dev, s, alloc = _enter(stream)
    n, seqs = tokens.shape[0], cu_rows.shape[0] - 1
    for t, what in ((target_probs, "target_probs"), (draft_probs, "draft_probs")):
        if t is None:
            continue
        if t.ndim != 2 or t.dtype is not torch.float32 or t.shape != (n, target_probs.shape[1]) or (t.shape[1] > 1 and t.stride(1) != 1):
            raise ValueError(f"{what}: float32 [rows][vocab] with contiguous rows expected")
        _on(t, dev, what)
    if uniforms.dtype is not torch.float32 or uniforms.shape != (n,) or not uniforms.is_contiguous() or uniforms.get_device() != dev:
        raise ValueError("uniforms: contiguous float32 [rows] on the current device expected")
    if draft_probs is not None and parent is not None:
        raise ValueError("verify_sampled: drafts with probabilities are chains")
    if out is None:
        with alloc:
            o = torch.empty(max(seqs, 0) + 3 * n, dtype=torch.int32, device=tokens.device)
        out = (o[:seqs], o[seqs:seqs + n], o[seqs + n:seqs + 2 * n], None if slots is None else o[seqs + 2 * n:])
    accept, out_tokens, out_rows, out_slots = out
    vocab = target_probs.shape[1]
    a = _VerifyArgs(target_probs.data_ptr(), None if draft_probs is None else draft_probs.data_ptr(), _index(tokens, (n,), "tokens", dev), _index(cu_rows, (seqs + 1,), "cu_rows", dev),
                    None if parent is None else _index(parent, (n,), "parent", dev), None if slots is None else _index(slots, (n,), "slots", dev), uniforms.data_ptr(),
                    _index(accept, (seqs,), "accept_len", dev), _index(out_tokens, (n,), "tokens (out)", dev), _index(out_rows, (n,), "rows (out)", dev),
                    None if slots is None else _index(out_slots, (n,), "slots (out)", dev), target_probs.stride(0) if n > 1 else vocab,
                    0 if draft_probs is None else draft_probs.stride(0) if n > 1 else vocab, seqs, n, vocab)
    if n and seqs:
        _check(binding.lib().sdv_verify_sampled(C.byref(a), s), "sdv_verify_sampled")
    return accept, out_tokens, out_rows, out_slots
