"""Slots of sequences with more rows than a draft tree has, whose parents are given as well."""
import numpy as np
import pytest

import paged_reference as R
import paper_2510_15312_b200 as pkg
from test_gpu_paged import forest, i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [[9000], [20, 3000, 64, 0, 700], [65, 129]])
@pytest.mark.parametrize("kind", ["chain", "tree"])
def test_slots(rows, kind):
    import torch
    rng = np.random.default_rng(len(rows))
    parent = np.concatenate([np.arange(n) - 1 for n in rows]).astype(np.int32) if kind == "chain" else forest(rng, rows, 7)
    cu = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    length, page, width = rng.integers(0, 50, len(rows)).astype(np.int32), 16, 600
    held = -(-length // 16)
    order = rng.permutation(2000).astype(np.int32)
    table, at = np.full((len(rows), width), -1, np.int32), 0
    for b, h in enumerate(held):
        table[b, :h] = order[at:at + h]
        at += h
    # depths from the definition row by row, each from its parent's
    pos = np.zeros(cu[-1], np.int64)
    for b, (r0, r1) in enumerate(R.spans(cu)):
        for i in range(r1 - r0):
            pos[r0 + i] = length[b] if i == 0 else pos[r0 + parent[r0 + i]] + 1
    exp = R.slots(length, cu, table, held, order[at:], 0, page, int(cu[-1]))
    dev = i32(table)
    got = pkg.paged_slots(i32(length), i32(cu), dev, i32(held), i32(order[at:]), i32([0]), page, int(cu[-1]), parent=i32(parent))
    np.testing.assert_array_equal(got[0].cpu().numpy(), exp[0])
    np.testing.assert_array_equal(got[1].cpu().numpy(), pos)
    np.testing.assert_array_equal(dev.cpu().numpy(), exp[2])
    assert torch.equal(got[2].cpu(), torch.tensor(exp[3], dtype=torch.int32))
