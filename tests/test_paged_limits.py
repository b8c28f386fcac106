"""Sizes that the operators on pages refuse because their kernels count in 32 bits (the fake addresses are never read: a call that passes ends at the device)."""
import pytest

import paper_2510_15312_b200 as pkg
from test_paged_refusals import rope, slots, verify

MOST = 1 << 30


def taken(rc):
    import torch
    return rc == (pkg.EINVAL if torch.cuda.is_available() else pkg.ECUDA)   # with a device, the fake addresses are what is refused


@pytest.mark.parametrize("call", [slots, rope, verify])
def test_rows(call):
    assert call(n_rows=MOST + 1) == pkg.EINVAL and call(n_rows=2 ** 31 - 1) == pkg.EINVAL
    assert taken(call(n_rows=MOST))


@pytest.mark.parametrize("kw", [dict(n_q_heads=2 ** 31 - 1), dict(n_q_heads=(MOST >> 6) - 3), dict(n_kv_heads=2 ** 31 - 1), dict(q=None, n_kv_heads=(MOST >> 7) + 1)])
def test_elements_of_a_row(kw):
    assert rope(**kw, k_row_stride=2 ** 34, v_row_stride=2 ** 34, out_row_stride=2 ** 34, q_row_stride=2 ** 34) == pkg.EINVAL


def test_the_longest_rows():
    assert taken(rope(n_q_heads=(MOST >> 6) - 4, out_row_stride=2 ** 34, q_row_stride=2 ** 34))


def test_rows_with_parents():
    """A row's depth is walked step by step: a chain of n rows takes n^2 / 2 of them in all, so n is bounded."""
    assert slots(parent=7 * 256, n_rows=4096 * 64 + 1) == pkg.EINVAL
    assert taken(slots(parent=7 * 256, n_rows=4096 * 64)) and taken(slots(n_rows=4096 * 64 + 1))
