"""The argument structures of include/sdv.h for the operators on a cache kept in pages, to call the C entry points directly."""
import ctypes as C

_vp, _i, _ll, _f = C.c_void_p, C.c_int, C.c_longlong, C.c_float


class Pages(C.Structure):
    _fields_ = [("k", _vp), ("v", _vp)] + [(n, _i) for n in ("dtype", "n_pages", "page_size", "n_kv_heads", "head_dim")] + \
               [(n, _ll) for n in ("page_stride", "head_stride", "token_stride")]


class SlotsArgs(C.Structure):
    _fields_ = [(n, _vp) for n in ("kv_len", "cu_rows", "parent", "n_held", "free_pages", "free_state", "block_table", "slots", "positions",
                                   "n_held_out", "free_state_out")] + [("table_stride", _ll)] + \
               [(n, _i) for n in ("n_seqs", "n_rows", "page_size", "table_width", "n_free")]


class RopeArgs(C.Structure):
    _fields_ = [(n, _vp) for n in ("q", "k", "v", "q_out", "positions", "slots", "frequencies")] + \
               [(n, _ll) for n in ("q_row_stride", "q_head_stride", "out_row_stride", "out_head_stride", "k_row_stride", "k_head_stride",
                                   "v_row_stride", "v_head_stride")] + \
               [(n, _i) for n in ("n_rows", "n_q_heads", "n_kv_heads", "head_dim", "rot_dim", "interleaved", "dtype")] + [("factor", _f)]


class AttentionArgs(C.Structure):
    _fields_ = [(n, _vp) for n in ("q", "out", "block_table", "kv_len", "cu_rows", "parent", "workspace", "status")] + [("workspace_bytes", C.c_size_t)] + \
               [(n, _ll) for n in ("q_row_stride", "q_head_stride", "out_row_stride", "out_head_stride", "table_stride")] + \
               [(n, _i) for n in ("n_seqs", "n_rows", "n_q_heads", "table_width")] + [("scale", _f)]


class VerifyArgs(C.Structure):
    _fields_ = [(n, _vp) for n in ("target", "draft", "tokens", "cu_rows", "parent", "slots", "uniforms", "accept_len", "out_tokens", "out_rows",
                                   "out_slots")] + [("target_stride", _ll), ("draft_stride", _ll)] + [(n, _i) for n in ("n_seqs", "n_rows", "vocab")]
