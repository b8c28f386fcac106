"""Calls of the operators on pages in which nothing, or not everything, is to be computed: their results say so."""
import numpy as np
import pytest

import paper_2510_15312_b200 as pkg
from test_gpu_paged import i32
from test_gpu_tree_attention import Case

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


def fresh(c, **kw):
    """An attention without `out`, in memory that held something else."""
    import torch
    dirt = torch.full_like(c.q, 55.0)
    del dirt
    return pkg.tree_attention(c.q, c.k, c.v, kw.pop("table", i32(c.table)), i32(c.lengths), i32(c.cu), parent=None if c.parent is None else i32(c.parent), **kw)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("hq,hkv,hd", [(14, 2, 64), (24, 8, 128), (1, 1, 64)])
@pytest.mark.parametrize("rows,lengths,pad,before", [([3], [5], 6, 0), ([70, 2], [100, 5], 3, 0), ([1, 64, 65, 0, 200], [700, 3, 90, 8, 0], 1, 0), ([2, 90], [10, 10], 400, 7), ([0, 0], [3, 4], 4, 0),
                                                     ([1] * 100 + [300] + [2] * 50, [9] * 151, 2, 1)])
def test_attention_without_an_output_to_write_to(rows, lengths, pad, before, hq, hkv, hd, dtype):
    """Rows of no sequence are zeros, rows past the limit NaN, the others as with a given output."""
    import torch
    c = Case(rows, lengths, hq, hkv, hd, 16, dtype, True, seed=2, pad=pad)
    if before:   # the first rows belong to nobody
        c.cu = (c.cu + before).astype(np.int32)
        c.q = torch.cat([c.q[:before], c.q])[:c.n]
        c.parent = np.concatenate([c.parent[:before], c.parent])[:c.n]
    want = c.run()
    kind = np.zeros(c.n, np.int64)
    for a, b in zip(c.cu[:-1], c.cu[1:]):
        kind[a:b] = 1
        kind[a + 64:b] = 2
    kind = torch.tensor(kind, device="cuda")
    got = fresh(c)
    assert torch.equal(got[kind == 1], want[kind == 1])
    assert bool((got[kind == 0] == 0).all()) and bool(torch.isnan(got[kind == 2]).all())
    assert bool((want[kind != 1] == 77.0).all())               # a given one: left as they were


def test_attention_without_sequences_or_columns():
    import torch
    c = Case([2], [20], 4, 2, 64)
    none = torch.empty((1, 0), dtype=torch.int32, device="cuda")
    assert bool((fresh(c, table=none) == 0).all())
    out = torch.full_like(c.q, 77.0)
    assert bool((fresh(c, table=none, out=out) == 77.0).all())
    c.lengths, c.cu = [], np.array([0], np.int32)
    assert bool((fresh(c, table=none[:0]) == 0).all())


def test_attention_without_an_output_in_a_graph():
    """Replayed with other numbers of rows in the same buffers."""
    import torch
    c = Case([64, 10], [90, 30], 6, 2, 64, tree=True, pad=0)
    q, table, kv, cu, parent = c.q, i32(c.table), i32(c.lengths), i32(c.cu), i32(c.parent)
    call = lambda: pkg.tree_attention(q, c.k, c.v, table, kv, cu, parent=parent)  # noqa: E731
    call()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = call()
    for bounds in ([0, 64, 74], [0, 5, 7], [0, 70, 74], [3, 3, 3], [0, 0, 66]):
        cu.copy_(i32(bounds))
        got.fill_(55.0)
        g.replay()
        given = pkg.tree_attention(q, c.k, c.v, table, kv, cu, parent=parent, out=torch.full_like(q, 77.0))
        kind = np.zeros(c.n, np.int64)
        for a, b in zip(bounds[:-1], bounds[1:]):
            kind[a:b] = 1
            kind[a + 64:b] = 2
        kind = torch.tensor(kind, device="cuda")
        whole = lambda x: torch.nan_to_num(x, nan=-9.0)  # noqa: E731  (a row over tokens that were never appended is anything)
        assert torch.equal(whole(got[kind == 1]), whole(given[kind == 1]))
        assert bool((got[kind == 0] == 0).all()) and bool(torch.isnan(got[kind == 2]).all()) and bool((given[kind != 1] == 77.0).all())


@pytest.mark.parametrize("inside", [False, True])
def test_idle_calls_in_and_behind_inference_mode(inside):
    """Outputs made in inference mode are taken outside of it too, as by calls that have something to do, and ordinary ones inside."""
    import torch
    with torch.inference_mode(not inside):
        out = (i32([5, 6]), i32([]), i32([]), None)
    t, u, cu, e = torch.empty((0, 11), device="cuda"), torch.empty(0, device="cuda"), i32([0, 0, 0]), i32([])
    with torch.inference_mode(inside):
        version = None if out[0].is_inference() else out[0]._version
        acc = pkg.verify_sampled(t, e, cu, u, out=out)[0]
    assert acc.tolist() == [-1, -1] and (version is None or out[0]._version > version)


def test_the_bytes_behind_the_last_field_of_the_arguments_say_nothing():
    """The C call leaves rows that nobody computes as they were, whatever lies in the padding of its structure."""
    import ctypes as C
    import torch
    from paged_structs import AttentionArgs, Pages
    c = Case([2], [20], 4, 2, 64)
    out, ws = torch.full_like(c.q, 77.0), pkg.tree_attention_workspace(1, 64)
    table, lengths, cu = i32(c.table), i32(c.lengths), i32(c.cu)
    pages = Pages(c.k.data_ptr(), c.v.data_ptr(), 0, c.k.shape[0], 16, 2, 64, *c.k.stride()[:3])
    args = AttentionArgs(q=c.q.data_ptr(), out=out.data_ptr(), block_table=table.data_ptr(), kv_len=lengths.data_ptr(), cu_rows=cu.data_ptr(), workspace=ws.data_ptr(),
                         workspace_bytes=ws.numel(), q_row_stride=256, q_head_stride=64, out_row_stride=256, out_head_stride=64, table_stride=table.stride(0), n_seqs=1, n_rows=c.n,
                         n_q_heads=4, table_width=table.shape[1], scale=0.125)
    end = AttentionArgs.scale.offset + 4
    C.memset(C.addressof(args) + end, 0xff, C.sizeof(args) - end)
    stream = C.c_void_p(torch.cuda.current_stream().cuda_stream)
    for call, rest in ((pkg.lib().sdv_tree_attention, 77.0), (pkg.lib().sdv_tree_attention_fresh, 0.0)):
        assert call(C.byref(args), C.byref(pages), stream) == pkg.OK
        torch.cuda.synchronize()
        assert bool((out[2:] == rest).all()) and torch.equal(out[:2], c.run()[:2])
