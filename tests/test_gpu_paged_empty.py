"""Calls of the operators on pages in which nothing, or not everything, is to be computed: their results say so."""
import pytest

import paper_2510_15312_b200 as pkg
from test_gpu_paged import i32

pytestmark = pytest.mark.gpu


def dirty():
    """Fills what the allocator will hand out next with something that is no result."""
    import torch
    x = [torch.full((1 << n,), 0x5a5a5a5a, dtype=torch.int32, device="cuda") for n in (6, 8, 10, 12, 14)]
    del x


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("slots", [False, True])
@pytest.mark.parametrize("drafts", [False, True])
def test_verify_of_idle_sequences(drafts, slots, given):
    """An idle step: every sequence is without rows."""
    import torch
    t, e = torch.empty((0, 11), device="cuda"), i32([])
    out = (i32([5, 6, 7]), i32([]), i32([]), i32([])) if given else None
    dirty()
    acc, words, rows, moved = pkg.verify_sampled(t, e, i32([0, 0, 0, 0]), torch.empty(0, device="cuda"), draft_probs=t if drafts else None, slots=e if slots else None, out=out)
    assert acc.tolist() == [-1, -1, -1] and words.numel() == rows.numel() == 0
    assert (moved is None) == (not slots)
    if given:
        assert acc is out[0]


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("slots", [False, True])
def test_verify_of_rows_without_sequences(slots, given):
    import torch
    n = 5
    out = (i32([]), i32([9] * n), i32([9] * n), i32([9] * n)) if given else None
    dirty()
    acc, words, rows, moved = pkg.verify_sampled(torch.rand(n, 7, device="cuda"), i32(range(n)), i32([0]), torch.rand(n, device="cuda"), slots=i32(range(n)) if slots else None, out=out)
    assert acc.numel() == 0 and words.tolist() == rows.tolist() == [-1] * n
    assert moved.tolist() == [-1] * n if slots else moved is None


def test_verify_of_idle_sequences_in_a_graph():
    import torch
    t, e, u, cu = torch.empty((0, 11), device="cuda"), i32([]), torch.empty(0, device="cuda"), i32([0, 0, 0])
    pkg.verify_sampled(t, e, cu, u)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        acc = pkg.verify_sampled(t, e, cu, u)[0]
    acc.fill_(3)
    g.replay()
    assert acc.tolist() == [-1, -1]
