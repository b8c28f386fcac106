"""Attention of draft trees over pages whose keys and values do not arrive: its waits run out, it says so, and nothing of it stays behind."""
import ctypes as C

import pytest

import paper_2510_15312_b200 as pkg
from paged_structs import AttentionArgs, Pages
from test_gpu_paged import i32
from test_gpu_tree_attention import Case

pytestmark = pytest.mark.gpu

CASES = {
    "parts": ([9], [5000], 12, 2, 128),                         # one item over many blocks, merged; a tile a block
    "long": ([9], [50000], 12, 2, 128),
    "items": ([40, 3, 1, 64], [200, 300, 90, 150], 28, 4, 64),  # blocks with several whole items
    "whole": ([5] * 10, [400] * 10, 4, 4, 64),                  # a short table: whole items a block
    "shares": ([17] * 40, [40 * i for i in range(40)], 6, 2, 128),
}


def share(c):
    """Tiles of the block that has most (csrc/tree_plan.h: equal shares of all tiles, or of all items where tables are short)."""
    import torch
    blocks, g = 2 * torch.cuda.get_device_properties(0).multi_processor_count, c.hq // c.hkv
    chunks, keys = [-(-n // (128 // g)) for n in c.rows], c.table.shape[1] * c.page
    tiles = [-(-(a + b) // 64) for a, b in zip(c.rows, c.lengths)]
    if -(-keys // 64) <= (8 if len(c.rows) >= 8 else 4):
        assert sum(chunks) * c.hkv <= blocks
        return max(tiles)
    return -(-sum(a * b for a, b in zip(chunks, tiles)) * c.hkv // blocks)


def call(c, out, status, wait_ns, tiles):
    import torch
    ws = pkg.tree_attention_workspace(len(c.rows), c.hd)
    table, lengths, cu, parent = i32(c.table), i32(c.lengths), i32(c.cu), None if c.parent is None else i32(c.parent)
    pages = Pages(c.k.data_ptr(), c.v.data_ptr(), 0, c.k.shape[0], c.page, c.hkv, c.hd, *c.k.stride()[:3])
    args = AttentionArgs(q=c.q.data_ptr(), out=out.data_ptr(), block_table=table.data_ptr(), kv_len=lengths.data_ptr(), cu_rows=cu.data_ptr(), parent=parent.data_ptr(),
                         workspace=ws.data_ptr(), status=status.data_ptr(), workspace_bytes=ws.numel(), q_row_stride=c.q.stride(0), q_head_stride=c.q.stride(1),
                         out_row_stride=out.stride(0), out_head_stride=out.stride(1), table_stride=table.stride(0), n_seqs=len(c.rows), n_rows=c.n, n_q_heads=c.hq,
                         table_width=table.shape[1], scale=c.hd ** -0.5)
    rc = pkg.lib().sdv_debug_tree_attention(C.byref(args), C.byref(pages), wait_ns, tiles, C.c_void_p(torch.cuda.current_stream().cuda_stream))
    torch.cuda.synchronize()
    return rc


@pytest.mark.parametrize("name", list(CASES))
@pytest.mark.parametrize("tiles", [0, 1, 2, 3])
def test_copies_that_do_not_arrive(name, tiles):
    import torch
    rows, lengths, hq, hkv, hd = CASES[name]
    c = Case(rows, lengths, hq, hkv, hd, 16, tree=True, seed=5)
    want = c.run()
    out, status = torch.full_like(want, 77.0), torch.zeros(1, dtype=torch.int32, device="cuda")
    some = share(c) > tiles
    assert call(c, out, status, 20_000_000, tiles) == pkg.OK and int(status[0]) == int(some)
    n = int(c.cu[-1])
    lost = torch.isnan(out)
    assert bool(lost[:n].any()) == some and bool(((out == want) | lost)[:n].all()) and bool((out[n:] == 77.0).all())   # right, or NaN
    if tiles == 0:
        assert bool(lost[:n].all())
    assert torch.equal(c.run(), want)                           # (checks its own status too)
    assert int(status[0]) == int(some)


@pytest.mark.parametrize("name", list(CASES))
def test_a_wait_given_up_while_copies_and_products_are_under_way(name):
    """A limit of a microsecond: some waits run out, the copies and products of others are still to come when their blocks end."""
    import torch
    rows, lengths, hq, hkv, hd = CASES[name]
    c = Case(rows, lengths, hq, hkv, hd, 16, tree=True, seed=6)
    want = c.run()
    n = int(c.cu[-1])
    for wait_ns in (0, 100, 1000, 3000):
        out, status = torch.full_like(want, 77.0), torch.zeros(1, dtype=torch.int32, device="cuda")
        assert call(c, out, status, wait_ns, 1 << 20) == pkg.OK
        lost = torch.isnan(out)
        assert bool(((out == want) | lost)[:n].all()) and bool(lost.any()) <= bool(status[0])
        assert torch.equal(c.run(), want)


def test_refuses():
    import torch
    c = Case([2], [20], 4, 2, 64, tree=True)
    out, status = torch.zeros_like(c.q), torch.zeros(1, dtype=torch.int32, device="cuda")
    assert call(c, out, status, 1000, -1) == pkg.EINVAL
    assert call(c, out, status, 10 ** 9, 1 << 20) == pkg.OK and int(status[0]) == 0
    assert torch.equal(out[:2], c.run()[:2])
