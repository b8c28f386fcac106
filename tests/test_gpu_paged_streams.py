"""The operators on pages in a step that runs over several streams, called and captured."""
import numpy as np
import pytest

import paged_reference as R
import paper_2510_15312_b200 as pkg
from test_gpu_paged import forest, i32, spread

pytestmark = pytest.mark.gpu


def test_a_step_over_two_streams():
    """Slots on one stream; keys and values appended on another while queries are turned on the first; attention where both meet, the verification of other rows beside it."""
    import torch
    rng = np.random.default_rng(2)
    hq, hkv, hd, page, rows, length = 6, 2, 64, 16, [9, 20, 1, 33], [700, 30, 0, 1500]
    cu = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    n, f = int(cu[-1]), torch.tensor(pkg.rope_frequencies(hd)[0], dtype=torch.float64, device="cuda")
    parent, dcu, kv = i32(forest(rng, rows, 4)), i32(cu), i32(length)
    order = rng.permutation(300).astype(np.int32)
    held = -(-np.array(length) // page)
    table0, at = np.full((4, 120), -1, np.int32), 0
    for b, h in enumerate(held):
        table0[b, :h] = order[at:at + h]
        at += h
    table, dheld, free, state = i32(table0), i32(held), i32(order[at:]), i32([0])
    q, k, v = (torch.zeros(n, h, hd, dtype=torch.bfloat16, device="cuda") for h in (hq, hkv, hkv))
    kp, vp = (torch.tensor(rng.standard_normal((300, hkv, page, hd)), device="cuda").bfloat16() for _ in range(2))
    p = spread(rng, n, 3000)
    target, tokens, u = torch.tensor(p, device="cuda"), i32(p.argmax(1)).roll(1), torch.tensor(rng.random(n).astype(np.float32), device="cuda")
    side = torch.cuda.Stream()

    def step(apart):
        main = torch.cuda.current_stream()
        slots, pos, h, s = pkg.paged_slots(kv, dcu, table, dheld, free, state, page, n, parent=parent)
        if apart:
            side.wait_stream(main)
        other = side if apart else main
        pkg.rope_append(pos, f, k=k, v=v, k_pages=kp, v_pages=vp, slots=slots, stream=other)
        verified = pkg.verify_sampled(target, tokens, dcu, u, parent=parent, slots=slots, stream=other)
        qr = pkg.rope_append(pos, f, q=q)
        if apart:
            main.wait_stream(side)
        return (slots, pos, h, s, qr, pkg.tree_attention(qr, kp, vp, table, kv, dcu, parent=parent), *verified)

    def fill(seed):
        r = np.random.default_rng(seed)
        for x in (q, k, v):
            x.copy_(torch.tensor(r.standard_normal(tuple(x.shape))).bfloat16())
        u.copy_(torch.tensor(r.random(n).astype(np.float32)))

    fill(0)
    step(True)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step(True)
    for seed in range(1, 12):
        fill(seed)
        want = [x.clone() for x in step(False)]
        torch.cuda.synchronize()
        apart = step(True)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(apart, want))
        for x in got:
            x.zero_()
        table.copy_(i32(table0))
        g.replay()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    exp = R.verify(p, tokens.cpu().numpy(), cu, u.cpu().numpy(), None, parent.cpu().numpy(), got[0].cpu().numpy())
    for a, b in zip(got[6:], exp):
        np.testing.assert_array_equal(a.cpu().numpy(), b)
