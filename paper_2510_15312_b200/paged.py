"""Operators on a cache kept in pages, on torch tensors: slots, rotary append, tree attention and sampled verification
(include/sdv.h says what each computes).  Argument marshalling only; the work is queued on the current stream, or on `stream`,
and the calls return at once.  All tensors are on the current device; index arrays are int32.  What the tensors' shapes and types
do not allow raises ValueError, what the library refuses SdvError.  Outputs not passed in are allocated by torch, on the stream the
work is queued on."""
from __future__ import annotations

import ctypes as C
import math
import struct
from typing import Optional

import torch

from . import binding
from .binding import EINVAL, SdvError

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


def _packer(structure):
    """Packs a structure's fields, in order, into bytes with the structure's layout (a fifth of the time that filling a ctypes structure takes)."""
    code = {_vp: "P", _i: "i", _ll: "q", _f: "f", C.c_size_t: "N"}
    s = struct.Struct("@" + "".join(code[t] for _, t in structure._fields_))
    assert s.size <= C.sizeof(structure) <= s.size + 7   # the padding at the end is nobody's field
    return struct.Struct(s.format + "0q").pack


_pack_pages, _pack_slots, _pack_rope, _pack_attention, _pack_verify = (_packer(t) for t in (_Pages, _SlotsArgs, _RopeArgs, _AttentionArgs, _VerifyArgs))
_i32, _f32, _f64, _u8 = torch.int32, torch.float32, torch.float64, torch.uint8
_types = {torch.bfloat16: 0, torch.float16: 1}   # SDV_BF16, SDV_FP16


def _empty_public(shape, strides, dtype):
    return torch.empty_strided(shape, strides, dtype=dtype, device="cuda")


try:   # the same in half the time (0.7 of 1.4 us), where torch has the function for it
    from torch._C._dynamo.guards import _empty_strided_cuda as _empty
except ImportError:
    _empty = _empty_public
_present = False                                 # whether a CUDA device has been seen


def _dtype(t, what: str) -> int:
    d = _types.get(t.dtype)
    if d is None:
        raise ValueError(f"{what}: bfloat16 or float16 expected, got {t.dtype}")
    return d


def _index(t, shape, device: int, what: str) -> int:
    """Address of a contiguous int32 tensor of this shape on the device."""
    if t.dtype is not _i32 or t.get_device() != device or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{what}: contiguous int32 tensor of shape {tuple(shape)} on the current device expected")
    return t.data_ptr()


def _table(t, n: int, device: int):
    """(address, width, distance of rows) of the block tables of n sequences."""
    if t.dtype is not _i32 or t.get_device() != device or t.dim() != 2:
        raise ValueError("block_table: int32 [sequences][width] on the current device expected")
    rows, width = t.shape
    row, column = t.stride()
    if rows != n or (column != 1 and width > 1):
        raise ValueError("block_table: a contiguous row for every sequence expected")
    return t.data_ptr(), width, row if n > 1 else width


def _enter(stream):
    """(current device, handle of the stream)."""
    global _present, _empty
    if not _present:
        if not torch.cuda.is_available():
            raise SdvError(binding.ECUDA, "no CUDA device (there is no CPU fallback)")
        try:   # not part of torch's documented interface: another version's may take other arguments
            _empty((1,), (1,), _i32)
        except Exception:
            _empty = _empty_public
        _present = True
    device = torch.cuda.current_device()
    if stream is not None:
        return device, stream.cuda_stream
    try:   # the current stream's handle without a Stream object around it, where torch has the function for it
        return device, torch._C._cuda_getCurrentRawStream(device)
    except AttributeError:
        return device, torch.cuda.current_stream().cuda_stream


def _vectors(stream, *lengths):
    """Fresh int32 vectors for outputs, allocated on the stream that writes them."""
    if stream is None:
        return [_empty((n,), (1,), _i32) for n in lengths]
    with torch.cuda.stream(stream):
        return [_empty((n,), (1,), _i32) for n in lengths]


def _check(rc: int, where: str):
    if rc:
        raise SdvError(rc, where)


def _pool(k_pages, v_pages, device: int):
    """(address of k, of v, type, pages, page size, KV heads, head dim, strides) of [pages][KV heads][tokens of a page][head dim], any strides with contiguous
    head elements (a pool that keeps the tokens outside the heads is passed as .transpose(1, 2))."""
    shape, strides, dtype = k_pages.shape, k_pages.stride(), k_pages.dtype
    if len(shape) != 4 or v_pages.shape != shape or v_pages.dtype is not dtype or v_pages.stride() != strides:
        raise ValueError("k_pages and v_pages: two tensors [pages][KV heads][page size][head dim] of the same shape, strides and type expected")
    if k_pages.get_device() != device or v_pages.get_device() != device:
        raise ValueError("k_pages, v_pages: not on the current CUDA device")
    n, heads, page, dim = shape
    s0, s1, s2, s3 = strides
    if s3 != 1 and dim > 1:
        raise ValueError("k_pages: the elements of a head have to be contiguous")
    # the stride of a dimension of one says nothing
    return (k_pages.data_ptr(), v_pages.data_ptr(), _dtype(k_pages, "k_pages"), n, page, heads, dim, s0 if n > 1 else 0, s1 if heads > 1 else 0, s2 if page > 1 else 0)


def _rows(t, device: int, what: str):
    """(shape, row stride, head stride) of a tensor [rows][heads][head dim]."""
    shape = t.shape
    if len(shape) != 3 or t.get_device() != device:
        raise ValueError(f"{what}: [rows][heads][head dim] on the current CUDA device expected")
    s0, s1, s2 = t.stride()
    if s2 != 1 and shape[2] > 1:
        raise ValueError(f"{what}: the elements of a head have to be contiguous")
    return shape, (s0 if shape[0] > 1 else 0), (s1 if shape[1] > 1 else 0)


def _fresh(stream, shape, dtype):
    """A contiguous tensor [rows][heads][head dim] for an output."""
    n, heads, dim = shape
    if stream is None:
        return _empty((n, heads, dim), (heads * dim, dim, 1), dtype)
    with torch.cuda.stream(stream):
        return _empty((n, heads, dim), (heads * dim, dim, 1), dtype)


def paged_slots(kv_len, cu_rows, block_table, n_held, free_pages, free_state, page_size: int, n_rows: int, parent=None, out=None, stream=None):
    """Hands pages to the sequences that need more and gives every row its slot and position: (slots, positions, n_held, free_state) after the call;
    block_table [sequences][width] is updated in place.  free_state[0] is the first unused entry of free_pages; of the returned one, the second entry is the number of
    sequences that were refused for want of pages (their slots are -1).  out: the four tensors to write to."""
    dev, s = _enter(stream)
    n, = per_seq = kv_len.shape
    per_row, listed, states = (n_rows,), free_pages.shape, free_state.shape
    table, width, table_stride = _table(block_table, n, dev)
    if n_rows < 0 or len(listed) != 1 or len(states) != 1 or states[0] < 1:
        raise ValueError("paged_slots: n_rows >= 0, a list of free pages and a free_state of at least one entry expected")
    if out is None:
        out = slots, positions, held, free = _vectors(stream, n_rows, n_rows, n, 2)
        to = (slots.data_ptr(), positions.data_ptr(), held.data_ptr(), free.data_ptr())
    else:
        slots, positions, held, free = out
        to = (_index(slots, per_row, dev, "slots"), _index(positions, per_row, dev, "positions"), _index(held, per_seq, dev, "n_held (out)"), _index(free, (2,), dev, "free_state (out)"))
    a = _pack_slots(_index(kv_len, per_seq, dev, "kv_len"), _index(cu_rows, (n + 1,), dev, "cu_rows"), 0 if parent is None else _index(parent, per_row, dev, "parent"),
                    _index(n_held, per_seq, dev, "n_held"), _index(free_pages, listed, dev, "free_pages"), _index(free_state, states, dev, "free_state"), table, *to, table_stride, n, n_rows,
                    page_size, width, listed[0])
    _check(binding.lib().sdv_paged_slots(a, s), "sdv_paged_slots")
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
    dev, s = _enter(stream)
    n, = per_row = positions.shape
    if frequencies.dtype is not _f64 or frequencies.dim() != 1 or not frequencies.is_contiguous() or frequencies.get_device() != dev:
        raise ValueError("frequencies: contiguous float64 [rot_dim / 2] on the current device expected")
    if (q is None and k is None) or (k is None) != (v is None):
        raise ValueError("rope_append: q, or k and v, expected")
    pages, q_ptr, out_ptr, k_ptr, v_ptr, slot_ptr = None, 0, 0, 0, 0, 0
    q_row = q_head = out_row = out_head = k_row = k_head = v_row = v_head = heads = kv_heads = 0
    if k is not None:
        if k_pages is None or v_pages is None or slots is None:
            raise ValueError("rope_append: k and v need k_pages, v_pages and slots")
        pages = _pool(k_pages, v_pages, dev)
        dtype, kv_heads, dim = pages[2], pages[5], pages[6]
        shape, k_row, k_head = _rows(k, dev, "k")
        v_shape, v_row, v_head = _rows(v, dev, "v")
        if shape != (n, kv_heads, dim) or v_shape != shape or k.dtype is not k_pages.dtype or v.dtype is not k_pages.dtype:
            raise ValueError("k, v: [rows][KV heads][head dim] of the pages' type expected")
        k_ptr, v_ptr, slot_ptr = k.data_ptr(), v.data_ptr(), _index(slots, per_row, dev, "slots")
    if q is not None:
        shape, q_row, q_head = _rows(q, dev, "q")
        if shape[0] != n or (k is not None and (shape[2] != dim or q.dtype is not k.dtype)):
            raise ValueError("q: a row for every position, with the head dim and type of k, expected")
        dtype, heads, dim = _dtype(q, "q"), shape[1], shape[2]
        if q_out is None:
            q_out, out_row, out_head = _fresh(stream, shape, q.dtype), heads * dim, dim
        else:
            out_shape, out_row, out_head = _rows(q_out, dev, "q_out")
            if out_shape != shape or q_out.dtype is not q.dtype:
                raise ValueError("q_out: shape and type of q expected")
        q_ptr, out_ptr = q.data_ptr(), q_out.data_ptr()
    half = frequencies.shape[0]
    a = _pack_rope(q_ptr, k_ptr, v_ptr, out_ptr, _index(positions, per_row, dev, "positions"), slot_ptr, frequencies.data_ptr(), q_row, q_head, out_row, out_head, k_row, k_head,
                   v_row, v_head, n, heads, kv_heads, dim, 2 * half, 1 if interleaved else 0, dtype, factor)
    if n:
        _check(binding.lib().sdv_rope_append(a, None if pages is None else _pack_pages(*pages), s), "sdv_rope_append")
    return q_out if q is not None else None


def tree_attention_workspace(n_seqs: int, head_dim: int):
    """A workspace for tree_attention on the current device, for up to n_seqs sequences."""
    _enter(None)
    n = binding.lib().sdv_tree_attention_workspace_bytes(n_seqs, head_dim)
    if n == 0:
        raise SdvError(EINVAL, "sdv_tree_attention_workspace_bytes")
    return torch.empty(n, dtype=_u8, device="cuda")


def tree_attention(q, k_pages, v_pages, block_table, kv_len, cu_rows, parent=None, scale: Optional[float] = None, out=None, workspace=None, status=None, stream=None):
    """Every row of q [rows][query heads][head dim] attends to the kv_len[b] committed tokens of its sequence and to the rows on its own path through
    the draft tree, whose keys and values were appended before.  scale: 1 / sqrt(head dim) unless given.  out: like q; rows of no sequence are left as they were.  workspace: see
    tree_attention_workspace; without one torch allocates it for the call.  status: int32 [1], set to 1 when a wait inside the kernel ran out."""
    dev, s = _enter(stream)
    pages = _pool(k_pages, v_pages, dev)
    shape, q_row, q_head = _rows(q, dev, "q")
    n, heads, dim = shape
    dtype = q.dtype
    if dtype is not k_pages.dtype or dim != pages[6]:
        raise ValueError("q: type and head dim of the pages expected")
    seqs, = per_seq = kv_len.shape
    table, width, table_stride = _table(block_table, seqs, dev)
    lib = binding.lib()
    if out is None:
        out, out_row, out_head = _fresh(stream, shape, dtype), heads * dim, dim
    else:
        out_shape, out_row, out_head = _rows(out, dev, "out")
        if out_shape != shape or out.dtype is not dtype:
            raise ValueError("out: shape and type of q expected")
    if workspace is None:
        size = lib.sdv_tree_attention_workspace_bytes(seqs, dim)
        if stream is None:
            workspace = _empty((size,), (1,), _u8)
        else:
            with torch.cuda.stream(stream):
                workspace = _empty((size,), (1,), _u8)
    else:
        size = workspace.numel() * workspace.element_size()
        if workspace.get_device() != dev or not workspace.is_contiguous():
            raise ValueError("workspace: contiguous memory of the current device expected")
    a = _pack_attention(q.data_ptr(), out.data_ptr(), table, _index(kv_len, per_seq, dev, "kv_len"), _index(cu_rows, (seqs + 1,), dev, "cu_rows"),
                        0 if parent is None else _index(parent, (n,), dev, "parent"), workspace.data_ptr(), 0 if status is None else _index(status, (1,), dev, "status"),
                        size, q_row, q_head, out_row, out_head, table_stride, seqs, n, heads, width, dim ** -0.5 if scale is None else scale)
    if n and seqs:
        _check(lib.sdv_tree_attention(a, _pack_pages(*pages), s), "sdv_tree_attention")
    return out


def _probs(t, n: int, vocab: int, device: int, what: str):
    """(address, distance of rows) of float32 [rows][vocab]."""
    if t.dtype is not _f32 or t.get_device() != device or t.shape != (n, vocab):
        raise ValueError(f"{what}: float32 [rows][vocab] on the current device expected")
    row, column = t.stride()
    if column != 1 and vocab > 1:
        raise ValueError(f"{what}: contiguous rows expected")
    return t.data_ptr(), row if n > 1 else vocab


def verify_sampled(target_probs, tokens, cu_rows, uniforms, draft_probs=None, parent=None, slots=None, out=None, stream=None):
    """Accepts drafted tokens against the target's probabilities [rows][vocab] (float32) with the uniform random numbers uniforms [rows] and draws one
    token behind the accepted ones: (accept_len [sequences], tokens [rows], rows [rows], slots [rows] or None).  draft_probs [rows][vocab]: what each draft of a chain was sampled from; without, drafts
    count as certain (retrieved), and parent may make them trees.  slots: every row's slot, for the slots that accepted rows move to.  out: the tensors to write to."""
    dev, s = _enter(stream)
    n, = per_row = tokens.shape
    edges, = bounds = cu_rows.shape
    seqs = edges - 1
    if target_probs.dim() != 2 or seqs < 0:
        raise ValueError("verify_sampled: target_probs [rows][vocab] and cu_rows [sequences + 1] expected")
    vocab = target_probs.shape[1]
    target, target_stride = _probs(target_probs, n, vocab, dev, "target_probs")
    draft, draft_stride = (0, 0) if draft_probs is None else _probs(draft_probs, n, vocab, dev, "draft_probs")
    if draft_probs is not None and parent is not None:
        raise ValueError("verify_sampled: drafts with probabilities are chains")
    if uniforms.dtype is not _f32 or uniforms.shape != per_row or not uniforms.is_contiguous() or uniforms.get_device() != dev:
        raise ValueError("uniforms: contiguous float32 [rows] on the current device expected")
    if out is None:
        if slots is None:
            (accept, out_tokens, out_rows), out_slots = _vectors(stream, seqs, n, n), None
        else:
            accept, out_tokens, out_rows, out_slots = _vectors(stream, seqs, n, n, n)
        to = (accept.data_ptr(), out_tokens.data_ptr(), out_rows.data_ptr(), 0 if slots is None else out_slots.data_ptr())
    else:
        accept, out_tokens, out_rows, out_slots = out
        to = (_index(accept, (seqs,), dev, "accept_len"), _index(out_tokens, per_row, dev, "tokens (out)"), _index(out_rows, per_row, dev, "rows (out)"),
              0 if slots is None else _index(out_slots, per_row, dev, "slots (out)"))
    a = _pack_verify(target, draft, _index(tokens, per_row, dev, "tokens"), _index(cu_rows, bounds, dev, "cu_rows"), 0 if parent is None else _index(parent, per_row, dev, "parent"),
                     0 if slots is None else _index(slots, per_row, dev, "slots"), uniforms.data_ptr(), *to, target_stride, draft_stride, seqs, n, vocab)
    if n and seqs:
        _check(binding.lib().sdv_verify_sampled(a, s), "sdv_verify_sampled")
    return accept, out_tokens, out_rows, out_slots
