"""Outputs of the operators on pages that begin inside an input or another output are refused; neighbours and arrays in each other's gaps are not."""
import pytest

import paper_2510_15312_b200 as pkg
from test_gpu_paged import i32, rope_case

pytestmark = pytest.mark.gpu


def refused(f, *a, **kw):
    with pytest.raises(pkg.SdvError) as e:
        f(*a, **kw)
    assert e.value.code == pkg.EINVAL


def test_slots():
    import torch
    n, held, free, state, cu = i32([3, 9]), i32([1, 1]), i32([2, 3, 4, 5]), i32([0, 0]), i32([0, 3, 8])
    mem = torch.zeros(200, dtype=torch.int32, device="cuda")
    table = mem[:20].view(2, 10)
    table[:, 0] = i32([0, 1])
    good = (mem[20:28], mem[28:36], mem[36:38], mem[38:40])      # one behind the other
    want = pkg.paged_slots(n, cu, table.clone()[:, :6], held, free, state, 8, 8)
    got = pkg.paged_slots(n, cu, table[:, :6], held, free, state, 8, 8, out=good)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    gap = (mem[20:28], mem[28:36], mem[6:8], mem[16:18])           # behind the columns that the table has
    got = pkg.paged_slots(n, cu, table[:, :6], i32([1, 1]), free, state, 8, 8, out=gap)
    assert torch.equal(got[2], want[2])
    for out in ((mem[20:28], mem[27:35], mem[36:38], mem[38:40]), (mem[19:27], *good[1:]), (good[0], good[1], mem[5:7], good[3]), (*good[:3], mem[37:39]), (*good[:3], mem[35:37])):
        refused(pkg.paged_slots, n, cu, table[:, :6 if out[2].data_ptr() == mem[5:7].data_ptr() else 10], held, free, state, 8, 8, out=out)
    for name in ("kv_len", "cu_rows", "n_held", "free_pages", "parent"):
        a = dict(kv_len=n, cu_rows=cu, block_table=table, n_held=held, free_pages=free, free_state=state, page_size=8, n_rows=8, out=good)
        x = {"kv_len": n, "cu_rows": cu, "n_held": held, "free_pages": free, "parent": i32([-1, 0, 1, -1, 0, 1, 2, 3])}[name]
        mem[50:50 + x.numel()] = x
        last = 50 + x.numel() - 1
        refused(pkg.paged_slots, **{**a, name: mem[50:50 + x.numel()], "out": (mem[last:last + 8], *good[1:])})
        pkg.paged_slots(**{**a, name: mem[50:50 + x.numel()], "out": (mem[last + 1:last + 9], *good[1:]), "n_held": mem[50:52] if name == "n_held" else i32([1, 1])})


def test_rope():
    import torch
    q, k, v, kp, vp, pos, slot = rope_case("bfloat16", 6, 4, 2, 64, 64, False, 8, False, qkv=False)
    f, p, s = torch.tensor(pkg.rope_frequencies(64)[0], dtype=torch.float64, device="cuda"), i32(pos), i32(slot)
    want = pkg.rope_append(p, f, q=q)
    mem = torch.zeros(40, 4, 64, dtype=q.dtype, device="cuda")
    mem[:6] = q
    refused(pkg.rope_append, p, f, q=mem[:6], q_out=mem[1:7])                       # a row further on
    refused(pkg.rope_append, p, f, q=mem[1:7], q_out=mem[:6])
    assert torch.equal(pkg.rope_append(p, f, q=mem[:6], q_out=mem[6:12]), want)
    assert torch.equal(pkg.rope_append(p, f, q=mem[:6], q_out=mem[:6]), want)       # in place
    wide = torch.zeros(6, 12, 64, dtype=q.dtype, device="cuda")
    wide[:, 1:9:2] = q
    assert torch.equal(pkg.rope_append(p, f, q=wide[:, 1:9:2], q_out=wide[:, 0:8:2]), want)     # heads in turn
    refused(pkg.rope_append, p, f, q=wide[:, 1:9:2], q_out=wide[:, 3:11:2])
    refused(pkg.rope_append, p, f, q=wide[:, 1:5], q_out=wide[:, 4:8])
    pool = torch.zeros(2, 2, 2, 8, 64, dtype=q.dtype, device="cuda")               # pages of keys and values in turn
    pkg.rope_append(p, f, k=k, v=v, k_pages=pool[:, 0], v_pages=pool[:, 1], slots=s % 16)
    flat = torch.zeros(5000, dtype=q.dtype, device="cuda")
    view = lambda at: flat[at:at + 2 * 2 * 8 * 64].view(2, 2, 8, 64)               # noqa: E731
    refused(pkg.rope_append, p, f, k=k, v=v, k_pages=view(0), v_pages=view(64), slots=s % 16)
    pkg.rope_append(p, f, k=k, v=v, k_pages=view(0), v_pages=view(2048), slots=s % 16)
    inside = flat[128:128 + 6 * 2 * 64].view(6, 2, 64)                             # rows to be appended in the pages themselves
    refused(pkg.rope_append, p, f, k=inside, v=v, k_pages=view(0), v_pages=view(2048), slots=s % 16)
    refused(pkg.rope_append, p, f, k=k, v=inside, k_pages=view(2048), v_pages=view(0), slots=s % 16)
    refused(pkg.rope_append, p, f, q=inside, k=k, v=v, k_pages=view(0), v_pages=view(2048), slots=s % 16)


def test_attention():
    import torch
    q, k, v, kp, vp, pos, slot = rope_case("bfloat16", 6, 4, 2, 64, 64, False, 8, False, qkv=False)
    table, kv, cu = i32([[0, 1, 2]]), i32([9]), i32([0, 6])
    want = pkg.tree_attention(q, kp, vp, table, kv, cu)
    mem = torch.zeros(40, 4, 64, dtype=q.dtype, device="cuda")
    mem[:6] = q
    refused(pkg.tree_attention, mem[:6], kp, vp, table, kv, cu, out=mem[5:11])
    assert torch.equal(pkg.tree_attention(mem[:6], kp, vp, table, kv, cu, out=mem[6:12]), want)
    pool = torch.cat([kp.flatten(), torch.zeros(6 * 256, dtype=q.dtype, device="cuda")])
    inside, keys = pool[kp.numel() - 64:kp.numel() - 64 + 6 * 256].view(6, 4, 64), pool[:kp.numel()].view(kp.shape)
    refused(pkg.tree_attention, q, keys, vp, table, kv, cu, out=inside)
    assert torch.equal(pkg.tree_attention(q, keys, vp, table, kv, cu, out=pool[kp.numel():].view(6, 4, 64)), want)
    ws = pkg.tree_attention_workspace(1, 64)
    refused(pkg.tree_attention, q, kp, vp, table, kv, cu, workspace=ws, out=ws[512:512 + 6 * 512].view(q.dtype).view(6, 4, 64))
    refused(pkg.tree_attention, q, kp, vp, table, kv, cu, workspace=ws, status=ws[512:516].view(torch.int32))


def test_verify():
    import torch
    n, vocab = 4, 10
    mem = torch.zeros(100, dtype=torch.int32, device="cuda")
    t, tok, cu, u = torch.rand(n, vocab, device="cuda"), i32(range(n)), i32([0, 1, 4]), torch.rand(n, device="cuda")
    want = pkg.verify_sampled(t, tok, cu, u)
    got = pkg.verify_sampled(t, tok, cu, u, out=(mem[:2], mem[2:6], mem[6:10], None))
    assert all(torch.equal(a, b) for a, b in zip(got[:3], want[:3]))
    for out in ((mem[:2], mem[1:5], mem[6:10], None), (mem[:2], mem[2:6], mem[5:9], None)):
        refused(pkg.verify_sampled, t, tok, cu, u, out=out)
    mem[50:54] = tok
    refused(pkg.verify_sampled, t, mem[50:54], cu, u, out=(mem[:2], mem[53:57], mem[6:10], None))
    wide = torch.rand(n, vocab + 6, device="cuda")
    wide[:, :vocab] = t
    hole = wide.view(torch.int32)[1, vocab:vocab + 4]                              # behind the columns of a row
    got = pkg.verify_sampled(wide[:, :vocab], tok, cu, u, out=(mem[:2], hole, mem[6:10], None))
    assert torch.equal(got[1], want[1])
    refused(pkg.verify_sampled, wide[:, :vocab], tok, cu, u, out=(mem[:2], wide.view(torch.int32)[1, vocab - 1:vocab + 3], mem[6:10], None))
