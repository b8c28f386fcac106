"""Refusals of the operators on a cache kept in pages that come before any device is touched, and the frequencies of scaled rotary embeddings."""
import ctypes as C
import math

import pytest

import paged_structs as paged
import paper_2510_15312_b200 as pkg

P = 256   # an address that is never read here


def good_pages(**kw):
    return paged.Pages(**{**dict(k=8 * P, v=9 * P, dtype=0, n_pages=4, page_size=16, n_kv_heads=2, head_dim=64, page_stride=2048, head_stride=1024, token_stride=64), **kw})


def good_slots(**kw):
    f = dict(kv_len=P, cu_rows=P, parent=None, n_held=P, free_pages=P, free_state=P, block_table=6 * P, slots=3 * P, positions=4 * P, n_held_out=2 * P, free_state_out=5 * P,
             table_stride=8, n_seqs=2, n_rows=5, page_size=16, table_width=8, n_free=9)
    return paged.SlotsArgs(**{**f, **kw})


def good_rope(**kw):
    f = dict(q=7 * P, k=P, v=P, q_out=7 * P, positions=P, slots=P, frequencies=P, q_row_stride=256, q_head_stride=64, out_row_stride=256, out_head_stride=64, k_row_stride=128,
             k_head_stride=64, v_row_stride=128, v_head_stride=64, n_rows=5, n_q_heads=4, n_kv_heads=2, head_dim=64, rot_dim=64, interleaved=0, dtype=0, factor=1.0)
    return paged.RopeArgs(**{**f, **kw})


def good_attention(**kw):
    f = dict(q=P, out=2 * P, block_table=P, kv_len=P, cu_rows=P, parent=None, workspace=3 * P, status=None, workspace_bytes=1 << 30, q_row_stride=256, q_head_stride=64,
             out_row_stride=256, out_head_stride=64, table_stride=8, n_seqs=2, n_rows=5, n_q_heads=4, table_width=8, scale=0.125)
    return paged.AttentionArgs(**{**f, **kw})


def good_verify(**kw):
    f = dict(target=P, draft=None, tokens=P, cu_rows=P, parent=None, slots=None, uniforms=P, accept_len=4 * P, out_tokens=2 * P, out_rows=3 * P, out_slots=None, target_stride=100,
             draft_stride=100, n_seqs=2, n_rows=5, vocab=100)
    return paged.VerifyArgs(**{**f, **kw})


def slots(**kw):
    return pkg.lib().sdv_paged_slots(C.byref(good_slots(**kw)), None)


def rope(pages=None, **kw):
    return pkg.lib().sdv_rope_append(C.byref(good_rope(**kw)), C.byref(good_pages(**(pages or {}))), None)


def attention(pages=None, **kw):
    return pkg.lib().sdv_tree_attention(C.byref(good_attention(**kw)), C.byref(good_pages(**(pages or {}))), None)


def verify(**kw):
    return pkg.lib().sdv_verify_sampled(C.byref(good_verify(**kw)), None)


@pytest.mark.parametrize("kw", [dict(n_seqs=-1), dict(n_seqs=4097), dict(n_rows=-1), dict(page_size=0), dict(table_width=-1), dict(n_free=-1), dict(table_stride=7),
                                dict(n_seqs=4096, table_width=1 << 20, table_stride=1 << 20),
                                dict(slots=P), dict(slots=4 * P), dict(n_held_out=P), dict(free_state_out=P), dict(block_table=P), dict(positions=6 * P), dict(parent=4 * P)])
def test_slots_refuses(kw):
    assert slots(**kw) == pkg.EINVAL


@pytest.mark.parametrize("kw", [dict(n_rows=-1), dict(dtype=2), dict(head_dim=63), dict(head_dim=258, rot_dim=64), dict(rot_dim=0), dict(rot_dim=66), dict(rot_dim=7), dict(k=None),
                                dict(v=None), dict(q=None, k=None, v=None), dict(n_q_heads=0), dict(n_kv_heads=0), dict(out_row_stride=0), dict(out_head_stride=-64), dict(q_out=P), dict(out_row_stride=512), dict(q_head_stride=128, q_row_stride=512), dict(k=8 * P), dict(v=8 * P),
                                dict(q_out=9 * P), dict(pages=dict(v=8 * P))])
def test_rope_refuses(kw):
    assert rope(**kw) == pkg.EINVAL


@pytest.mark.parametrize("kw", [dict(n_seqs=-1), dict(n_seqs=4097), dict(n_rows=-1), dict(n_q_heads=3), dict(n_q_heads=0), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf),
                                dict(scale=math.nan), dict(table_stride=7), dict(q_row_stride=4), dict(q_head_stride=65), dict(out_row_stride=9), dict(out_head_stride=2),
                                dict(table_width=-1), dict(out_row_stride=0), dict(out_head_stride=0), dict(n_q_heads=258), dict(pages=dict(head_dim=96)), dict(pages=dict(page_size=24)), dict(pages=dict(page_size=4)), dict(pages=dict(n_kv_heads=0)),
                                dict(out=P), dict(workspace=2 * P), dict(status=P), dict(status=3 * P), dict(out=8 * P), dict(out=9 * P)])
def test_attention_refuses(kw):
    assert attention(**kw) == pkg.EINVAL


@pytest.mark.parametrize("kw", [dict(n_seqs=-1), dict(n_seqs=4097), dict(n_rows=-1), dict(vocab=0), dict(vocab=(1 << 21) + 1, target_stride=1 << 22), dict(target_stride=99),
                                dict(draft=P, draft_stride=99), dict(draft=P, parent=P), dict(slots=P), dict(out_slots=P), dict(out_tokens=P), dict(out_rows=P), dict(out_rows=2 * P),
                                dict(slots=5 * P, out_slots=5 * P), dict(slots=5 * P, out_slots=P), dict(accept_len=P), dict(accept_len=2 * P), dict(parent=4 * P)])
def test_verify_refuses(kw):
    assert verify(**kw) == pkg.EINVAL


def test_null_arguments():
    L = pkg.lib()
    assert L.sdv_paged_slots(None, None) == pkg.EINVAL and L.sdv_rope_append(None, None, None) == pkg.EINVAL
    assert L.sdv_tree_attention(None, None, None) == pkg.EINVAL and L.sdv_verify_sampled(None, None) == pkg.EINVAL
    assert L.sdv_tree_attention(C.byref(good_attention()), None, None) == pkg.EINVAL
    assert L.sdv_tree_attention_workspace_bytes(-1, 64) == 0 and L.sdv_tree_attention_workspace_bytes(4, 96) == 0


def test_calls_without_work_do_nothing():
    assert rope(n_rows=0) == pkg.OK
    assert attention(n_rows=0) == pkg.OK and attention(n_seqs=0) == pkg.OK and attention(table_width=0) == pkg.OK
    assert verify(n_rows=0) == pkg.OK and verify(n_seqs=0) == pkg.OK


def test_no_cpu_fallback():
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    # well-formed calls reach the device, which is not there
    assert slots() == pkg.ECUDA and rope() == pkg.ECUDA and attention() == pkg.ECUDA and verify() == pkg.ECUDA
    t = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(pkg.SdvError):
        pkg.paged_slots(t, torch.zeros(5, dtype=torch.int32), t[:, None], t, t, t, 16, 0)
    with pytest.raises(pkg.SdvError):
        pkg.rope_append(t, torch.zeros(2, dtype=torch.float64), q=torch.zeros(4, 1, 4, dtype=torch.bfloat16))


def test_frequencies():
    f, a = pkg.rope_frequencies(8, theta=100.0)
    assert a == 1.0 and f == pytest.approx([1.0, 100 ** -0.25, 0.1, 100 ** -0.75], rel=1e-15)
    assert pkg.rope_frequencies(8, 100.0, "linear", factor=4.0)[0] == pytest.approx([x / 4 for x in f], rel=1e-15)
    # banded: a pair that turns `high` times or more within the original positions keeps its frequency, one that turns `low` times or less has it divided
    b, a = pkg.rope_frequencies(64, 1.0e4, "banded", factor=8.0, original_positions=1000, low=1.0, high=4.0)
    base = pkg.rope_frequencies(64, 1.0e4)[0]
    for x, y in zip(base, b):
        turns = 1000 * x / (2 * math.pi)
        if turns >= 4:
            assert y == x
        elif turns <= 1:
            assert y == pytest.approx(x / 8, rel=1e-15)
        else:
            assert x / 8 < y < x
    assert a == 1.0 and any(x / 8 < y < x for x, y in zip(base, b))
    # yarn: the fastest pairs are kept, the slowest divided, in between monotone; the factor grows with the logarithm
    y, a = pkg.rope_frequencies(64, 1.0e4, "yarn", factor=8.0, original_positions=1000)
    assert a == pytest.approx(0.1 * math.log(8) + 1, rel=1e-15)
    ratio = [p / q for p, q in zip(y, base)]
    assert ratio[0] == 1.0 and ratio[-1] == pytest.approx(1 / 8, rel=1e-12) and all(p >= q - 1e-12 for p, q in zip(ratio, ratio[1:]))
    # the two ends of the line, worked out by hand: pairs that turn 32 times and once within 1000 positions
    at = [64 * math.log(1000 / (t * 2 * math.pi)) / (2 * math.log(1.0e4)) for t in (32.0, 1.0)]
    first, last = math.floor(at[0]), math.ceil(at[1])
    assert ratio[first] == 1.0 and ratio[last] == pytest.approx(1 / 8, rel=1e-12) and ratio[last - 1] > 1 / 8 + 1e-3
    for bad in (dict(rot_dim=7), dict(rot_dim=0), dict(rot_dim=8, theta=0.0), dict(rot_dim=8, factor=0.0), dict(rot_dim=8, scaling="other"), dict(rot_dim=8, scaling="banded", low=4.0)):
        with pytest.raises(ValueError):
            pkg.rope_frequencies(**bad)
