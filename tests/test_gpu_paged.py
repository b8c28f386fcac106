"""Slots, rotary append and sampled verification on a cache kept in pages, against their definitions in 64 bits."""
import numpy as np
import pytest

import paged_reference as R
import paper_2510_15312_b200 as pkg

pytestmark = pytest.mark.gpu


def i32(x):
    import torch
    return torch.tensor(np.asarray(x, dtype=np.int32), device="cuda")


def forest(rng, rows, back=5):
    out = []
    for n in rows:
        out += [-1] * min(n, 1) + [int(rng.integers(max(0, i - back), i)) for i in range(1, n)]
    return np.array(out, dtype=np.int32)


# ------------------------------------------------------------------------------------------ slots
SLOTS = {
    # (rows, committed tokens, held pages or None: those of the committed tokens, page size, table width, spare pages of the list)
    "one row": ([1], [0], None, 16, 4, 3),
    "page borders": ([1, 1, 3, 16, 17], [15, 16, 14, 0, 32], None, 16, 8, 2),
    "page of one": ([3, 2], [5, 0], None, 1, 16, 1),
    "odd page": ([4, 9, 1], [13, 6, 7], None, 7, 8, 0),
    "without rows": ([0, 4, 0, 0, 2, 0], [9, 3, 0, 100, 1, 5], None, 8, 4, 0),
    "nothing held": ([2, 5, 1], [70, 0, 33], [0, 0, 0], 16, 8, 1),
    "more held than needed": ([2, 2], [3, 3], [3, 1], 8, 5, 0),
    "list runs out": ([9, 9, 9, 1], [0, 8, 0, 4], None, 8, 4, -3),
    "list is empty": ([1, 1], [8, 3], None, 8, 4, -100),
    "table too narrow": ([40, 1, 3], [0, 2, 8], None, 8, 3, 4),
    "many": ([int(x) for x in np.random.default_rng(3).integers(0, 30, 700)], [int(x) for x in np.random.default_rng(4).integers(0, 900, 700)], None, 32, 32, 5),
    "most": ([1] * 4096, [7] * 4096, None, 8, 2, 0),
    "prompt": ([9000], [0], [0], 64, 150, 2),
}


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("name", list(SLOTS))
def test_slots(name, tree):
    import torch
    rows, length, held, page, width, spare = SLOTS[name]
    if tree and max(rows) > 64:
        rows = [min(r, 64) for r in rows]
    rng = np.random.default_rng(11)
    held = np.array([-(-x // page) for x in length] if held is None else held, dtype=np.int32)
    want = [-(-(a + b) // page) if a else 0 for a, b in zip(rows, length)]
    n_free = max(0, 4 + sum(max(0, w - h) for w, h in zip(want, held)) + spare)
    order = rng.permutation(int(held.sum()) + n_free).astype(np.int32)
    table, at = np.full((len(rows), width), -7, dtype=np.int32), 0
    for b, h in enumerate(held):
        h = min(int(h), width)
        held[b] = h
        table[b, :h] = order[at:at + h]
        at += h
    free, head = order[at:at + n_free], min(4, n_free)
    cu = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    n_rows = int(cu[-1]) + 3                          # three rows of padding
    parent = np.concatenate([forest(rng, rows), [-1] * 3]).astype(np.int32) if tree else None
    exp = R.slots(np.array(length), cu, table, held, free, head, page, n_rows, parent)
    wide = torch.full((len(rows), width + 3), -9, dtype=torch.int32, device="cuda")   # a table that is part of a wider one
    wide[:, :width] = i32(table)
    kv, h0 = i32(length), i32(held)
    got = pkg.paged_slots(kv, i32(cu), wide[:, :width], h0, i32(free), i32([head, 55]), page, n_rows, parent=None if parent is None else i32(parent))
    np.testing.assert_array_equal(got[0].cpu().numpy(), exp[0])
    np.testing.assert_array_equal(got[1].cpu().numpy(), exp[1])
    np.testing.assert_array_equal(wide[:, :width].cpu().numpy(), exp[2])
    assert int((wide[:, width:] != -9).sum()) == 0
    np.testing.assert_array_equal(got[2].cpu().numpy(), exp[3])
    assert got[3].tolist() == list(exp[4])
    np.testing.assert_array_equal(h0.cpu().numpy(), held)                            # inputs stay


def test_slots_of_arrays_that_hold_anything():
    """Nothing outside the buffers, -1 where there is no slot (csrc bounds: lengths and rows are clamped, negative pages have no slot)."""
    import torch
    table = torch.full((3, 4), -5, dtype=torch.int32, device="cuda")
    slots, pos, held, free = pkg.paged_slots(i32([-9, 2 ** 31 - 1, 5]), i32([0, 2, 7, 4]), table, i32([0, 0, 3]), i32([1, 2, 3]), i32([-4]), 8, 9)
    s = slots.cpu().numpy()
    assert s[:2].tolist() == [8, 9] and (s[2:] == -1).all()                        # a negative length is 0; the second sequence does not fit; rows descend
    assert held.tolist() == [1, 0, 3] and free.tolist() == [1, 1]
    slots, *_ = pkg.paged_slots(i32([3]), i32([0, 2]), i32([[-1, 2 ** 31 - 1]]), i32([2]), i32([0]), i32([0]), 4, 2)
    assert slots.tolist() == [-1, -1]                                               # pages -1 and one beyond 32 bits


def test_slots_without_sequences():
    import torch
    e = torch.empty(0, dtype=torch.int32, device="cuda")
    slots, pos, held, free = pkg.paged_slots(e, i32([0]), torch.empty((0, 4), dtype=torch.int32, device="cuda"), e, i32([5]), i32([1]), 8, 2)
    assert slots.tolist() == [-1, -1] and pos.tolist() == [0, 0] and held.numel() == 0 and free.tolist() == [1, 0]


def test_slots_refuses():
    import torch
    t, cu = i32([3]), i32([0, 1])
    table, free, state = i32([[0, 1]]), i32([2, 3]), i32([0, 0])
    out = [torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(3)] + [torch.zeros(2, dtype=torch.int32, device="cuda")]
    for bad in (dict(out=(out[0], out[1], t, out[3])), dict(out=(out[0], out[1], out[2], state))):   # outputs over inputs
        with pytest.raises(pkg.SdvError):
            pkg.paged_slots(t, cu, table, t, free, state, 8, 1, **bad)
    for args in ((t.long(), cu, table, t, free, state, 8, 1), (t, cu[:1], table, t, free, state, 8, 1), (t, cu, table.t(), t, free, state, 8, 1),
                 (t, cu, table, t, free, state, 8, -1), (t.cpu(), cu, table, t, free, state, 8, 1), (t, cu, table.cpu(), t, free, state, 8, 1)):
        with pytest.raises(ValueError):
            pkg.paged_slots(*args)
    with pytest.raises(pkg.SdvError):
        pkg.paged_slots(t, cu, table, t, free, state, 0, 1)


# ------------------------------------------------------------------------------------------ rotary embedding and append
def rope_case(dtype, n, hq, hkv, hd, rot, interleaved, page, tokens_first, seed=0, far=5000, qkv=True, offset=0):
    import torch
    rng = np.random.default_rng(seed)
    t = getattr(torch, dtype)
    if qkv:   # the three side by side in one row, `offset` elements in
        wide = torch.tensor(rng.standard_normal((n, offset + (hq + 2 * hkv) * hd)), device="cuda").to(t)[:, offset:]
        q, k, v = (x.unflatten(1, (-1, hd)) for x in wide.split([hq * hd, hkv * hd, hkv * hd], 1))
    else:
        q, k, v = (torch.tensor(rng.standard_normal((n, h, hd)), device="cuda").to(t) for h in (hq, hkv, hkv))
    pages = -(-n // page) + 2
    shape = (pages, page, hkv, hd) if tokens_first else (pages, hkv, page, hd)
    kp, vp = (torch.tensor(rng.standard_normal(shape), device="cuda").to(t) for _ in range(2))
    if tokens_first:
        kp, vp = kp.transpose(1, 2), vp.transpose(1, 2)
    pos = rng.integers(-far, far, n).astype(np.int32)
    slot = rng.permutation(pages * page)[:n].astype(np.int32)
    return q, k, v, kp, vp, pos, slot


def check_rope(got, x, pos, f, factor, interleaved, what):
    """Half a step of the type for the rounding; cosine and sine in fp32 from an exact angle: 2^-22 each, products and sums three roundings of 2^-24."""
    import torch
    exp, size = R.rope(x.double().cpu().numpy(), pos, f, factor, interleaved)
    u = torch.finfo(got.dtype).eps / 2
    err = np.abs(got.double().cpu().numpy() - exp)
    tiny = 2.0 ** -25 if got.dtype == torch.float16 else 0.0   # half a step of the smallest numbers
    assert (err <= u * np.abs(exp) + (1 + u) * (2.0 ** -22 + 3 * 2.0 ** -24) * size + tiny).all(), (what, err.max())
    rot = 2 * len(f)
    assert torch.equal(got[..., rot:], x[..., rot:])


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype,n,hq,hkv,hd,rot,page,tokens_first,offset", [
    ("bfloat16", 1, 4, 4, 64, 64, 16, False, 0),
    ("float16", 9, 12, 2, 128, 128, 16, True, 0),
    ("bfloat16", 33, 14, 2, 64, 32, 8, False, 0),
    ("bfloat16", 130, 6, 2, 128, 34, 32, True, 0),     # 17 pairs: one element at a time
    ("float16", 77, 10, 2, 64, 24, 64, False, 8),
    ("bfloat16", 50, 3, 1, 64, 64, 7, False, 3),       # rows on odd boundaries, an odd page
    ("float16", 41, 2, 2, 80, 20, 16, True, 4),
    ("bfloat16", 1300, 5, 1, 256, 256, 128, False, 2),
    ("bfloat16", 3000, 4, 2, 64, 64, 32, True, 0),
    ("float16", 20, 1, 1, 2, 2, 8, False, 0),
    ("bfloat16", 3, 66, 4, 256, 102, 16, False, 0),    # more heads than shared memory takes at a time
    ("float16", 2500, 7, 1, 96, 90, 16, True, 0),
    ("bfloat16", 40, 3, 3, 72, 64, 8, False, 0),       # heads that are no multiple of sixteen
    ("float16", 30, 2, 1, 88, 86, 16, False, 8),
])
def test_rope_append(dtype, n, hq, hkv, hd, rot, page, tokens_first, offset, interleaved):
    import torch
    q, k, v, kp, vp, pos, slot = rope_case(dtype, n, hq, hkv, hd, rot, interleaved, page, tokens_first, seed=n, offset=offset)
    f = np.array(pkg.rope_frequencies(rot, 1.0e4)[0])
    slot[::5] = np.where(np.arange(len(slot[::5])) % 3 == 0, -1, slot[::5])
    kp0, vp0 = kp.clone(), vp.clone()
    if hd < 8:   # strides of pages are multiples of eight
        with pytest.raises(pkg.SdvError):
            pkg.rope_append(i32(pos), torch.tensor(f, device="cuda"), q=q, k=k, v=v, k_pages=kp, v_pages=vp, slots=i32(slot), interleaved=interleaved, factor=1.25)
        got = pkg.rope_append(i32(pos), torch.tensor(f, device="cuda"), q=q, interleaved=interleaved, factor=1.25)
        return check_rope(got, q, pos, f, 1.25, interleaved, "q")
    before = q.clone()
    got = pkg.rope_append(i32(pos), torch.tensor(f, device="cuda"), q=q, k=k, v=v, k_pages=kp, v_pages=vp, slots=i32(slot), interleaved=interleaved, factor=1.25)
    assert torch.equal(before, q)
    check_rope(got, q, pos, f, 1.25, interleaved, "q")
    row = np.nonzero(slot >= 0)[0]
    at = (torch.tensor(slot[row] // page, device="cuda").long()[:, None], torch.arange(hkv, device="cuda")[None], torch.tensor(slot[row] % page, device="cuda").long()[:, None])
    check_rope(kp[at], k[torch.tensor(row, device="cuda")], pos[row], f, 1.25, interleaved, "k")
    assert torch.equal(vp[at], v[torch.tensor(row, device="cuda")])
    kp[at], vp[at] = kp0[at], vp0[at]                                               # all else is as it was
    assert torch.equal(kp, kp0) and torch.equal(vp, vp0)


def test_rope_in_place_and_alone():
    import torch
    q, k, v, kp, vp, pos, slot = rope_case("bfloat16", 19, 4, 2, 64, 64, False, 16, False, qkv=False)
    f = torch.tensor(pkg.rope_frequencies(64, 1.0e6)[0], dtype=torch.float64, device="cuda")
    a = pkg.rope_append(i32(pos), f, q=q)
    q2, kp2 = q.clone(), kp.clone()
    assert pkg.rope_append(i32(pos), f, q=q2, q_out=q2) is q2 and torch.equal(a, q2)
    assert pkg.rope_append(i32(pos), f, k=k, v=v, k_pages=kp, v_pages=vp, slots=i32(slot)) is None
    assert not torch.equal(kp, kp2)
    none = torch.empty((0, 4, 64), dtype=torch.bfloat16, device="cuda")
    assert pkg.rope_append(i32([]), f, q=none).shape == (0, 4, 64)


@pytest.mark.parametrize("position", [0, 1, 999983, 2 ** 31 - 1, -2 ** 31])
def test_rope_at_far_positions(position):
    """The angle is exact to 2^-22 of a radian at any position."""
    import torch
    x = torch.randn(1, 2, 64, device="cuda").half()
    f = np.array(pkg.rope_frequencies(64, 1.0e4, "yarn", factor=32.0)[0])
    pos = np.array([position])
    check_rope(pkg.rope_append(i32(pos), torch.tensor(f, device="cuda"), q=x), x, pos, f, 1.0, False, position)


def test_rope_does_not_write_outside_the_pool():
    """Slots outside the pool are left out: the bounds are the kernel's own comparison with pages times page size."""
    import torch
    q, k, v, kp, vp, pos, slot = rope_case("bfloat16", 6, 2, 1, 64, 64, False, 8, False)
    around = torch.full((kp.numel() * 2,), 3.0, dtype=torch.bfloat16, device="cuda")
    pool = around[kp.numel() // 2:kp.numel() // 2 + kp.numel()].view(kp.shape)       # a pool within a larger tensor
    whole = kp.shape[0] * 8
    pkg.rope_append(i32(pos), torch.tensor(pkg.rope_frequencies(64)[0], dtype=torch.float64, device="cuda"), k=k, v=v, k_pages=pool, v_pages=vp,
                    slots=i32([-1, whole, whole + 5, 2 ** 31 - 1, -2 ** 31, 0]))
    pool[0, :, 0] = 3.0
    assert bool((around == 3.0).all())


def test_rope_refuses():
    import torch
    q, k, v, kp, vp, pos, slot = rope_case("bfloat16", 6, 4, 2, 64, 64, False, 8, False, qkv=False)
    f, p, s = torch.tensor(pkg.rope_frequencies(64)[0], dtype=torch.float64, device="cuda"), i32(pos), i32(slot)
    good = dict(q=q, k=k, v=v, k_pages=kp, v_pages=vp, slots=s)
    for bad in (dict(v=None), dict(slots=None), dict(k_pages=None), dict(q=q[:5]), dict(k=k[:, :1]), dict(v=v.half()), dict(q=q.half()), dict(q=q.float()),
                dict(v_pages=vp[:1]), dict(v_pages=vp.half()), dict(slots=s.long()), dict(slots=s.cpu()), dict(q=q.cpu()), dict(q=q.transpose(1, 2)), dict(q_out=q[:, :2]),
                dict(k_pages=kp.transpose(2, 3), v_pages=vp.transpose(2, 3))):
        with pytest.raises(ValueError):
            pkg.rope_append(p, f, **{**good, **bad})
    with pytest.raises(ValueError):
        pkg.rope_append(p, f.float(), **good)
    with pytest.raises(ValueError):
        pkg.rope_append(p, f)
    with pytest.raises(pkg.SdvError):   # pairs beyond the head
        pkg.rope_append(p, torch.zeros(33, dtype=torch.float64, device="cuda"), q=q)


# ------------------------------------------------------------------------------------------ sampled verification
def spread(rng, n, vocab, sharp=3.0):
    x = rng.standard_normal((n, vocab)) * sharp
    p = np.exp(x - x.max(1, keepdims=True))
    return (p / p.sum(1, keepdims=True)).astype(np.float32)


def verify_case(rng, rows, vocab, tree, drafts, pad=2):
    n = sum(rows) + pad
    cu = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    target = spread(rng, n, vocab)
    parent = np.concatenate([forest(rng, rows, 3), [-1] * pad]).astype(np.int32) if tree else None
    tokens = rng.integers(0, vocab, n).astype(np.int32)
    draft = spread(rng, n, vocab) if drafts else None
    for r0, r1 in R.spans(cu):
        for i in range(1, r1 - r0):
            before = r0 + R.up(parent, r0, i)
            if drafts:
                mix = 0.7 * target[before].astype(np.float64) + 0.3 * draft[r0 + i]
                draft[r0 + i] = (mix / mix.sum()).astype(np.float32)
                tokens[r0 + i] = min(int(np.searchsorted(np.cumsum(draft[r0 + i].astype(np.float64)), rng.random())), vocab - 1)
            elif rng.random() < 0.8:      # likely tokens, siblings with the same one among them
                tokens[r0 + i] = np.argsort(target[before])[-1 - int(rng.integers(0, min(3, vocab)))]
    return target, tokens, cu, rng.random(n).astype(np.float32), draft, parent


def check_verify(target, tokens, cu, u, draft, parent, slots=None, stride=None):
    import torch
    dev = lambda x: None if x is None else torch.tensor(x, device="cuda")  # noqa: E731
    t, d = dev(target), dev(draft)
    if stride:
        w = torch.full((target.shape[0], stride), float("nan"), device="cuda")
        w[:, 1:1 + target.shape[1]] = t
        t = w[:, 1:1 + target.shape[1]]    # rows on 4-byte boundaries
    got = pkg.verify_sampled(t, dev(tokens), dev(cu), dev(u), draft_probs=d, parent=dev(parent), slots=dev(slots))
    exp = R.verify(target, tokens, cu, u, draft, parent, slots)
    for g, e, what in zip(got, exp, ("accept_len", "tokens", "rows", "slots")):
        if g is not None:
            np.testing.assert_array_equal(g.cpu().numpy(), e, err_msg=what)
    return exp


@pytest.mark.parametrize("kind", ["chain", "tree", "sampled"])
@pytest.mark.parametrize("rows,vocab", [([1], 1), ([2], 5), ([9], 2016), ([3, 0, 64, 1], 513), ([64], 1000), ([7] * 40, 4099), ([5, 2, 17], 151936), ([1] * 300, 777), ([33, 20], 40000)])
def test_verify(rows, vocab, kind):
    rng = np.random.default_rng(len(rows) * 1000 + vocab)
    for round in range(3):
        case = verify_case(rng, rows, vocab, kind == "tree", kind == "sampled")
        check_verify(*case, slots=rng.permutation(5000)[:case[0].shape[0]].astype(np.int32), stride=vocab + 5 if round == 2 else None)


def test_verify_reaches_every_outcome():
    """The cases above do take every way: none, some and all accepted, later siblings among them."""
    rng = np.random.default_rng(5)
    seen, sibling = set(), False
    for _ in range(40):
        case = verify_case(rng, [6] * 8, 50, True, False)
        acc, _, rows, moved = check_verify(*case, slots=np.arange(50, dtype=np.int32))
        seen |= set(int(a) for a in acc)
        sibling |= bool((moved >= 0).any())
    assert {0, 1, 2, 3} <= seen and sibling


def test_verify_of_certain_predictions_is_the_greedy_scan():
    """A target with one certain token per row: exactly the matching prefix is accepted, the model's token follows (as sdv_verify does it)."""
    rng = np.random.default_rng(9)
    y = rng.integers(0, 300, 20)
    target = np.zeros((20, 300), np.float32)
    target[np.arange(20), y] = 1.0
    tokens = np.concatenate([[0], y[:-1]]).astype(np.int32)
    for e in range(1, 20):
        wrong = tokens.copy()
        wrong[e] = (wrong[e] + 1) % 300
        acc, words, _, _ = check_verify(target, wrong, np.array([0, 20], np.int32), rng.random(20).astype(np.float32), None, None)
        assert acc[0] == e - 1 and words[:e].tolist() == y[:e].tolist()


def test_verify_at_the_borders():
    """Shares of powers of two and random numbers on their sums: every comparison is exact."""
    p = np.array([[0.25, 0.0, 0.5, 0.25], [0.125, 0.125, 0.25, 0.5], [0.5, 0.5, 0.0, 0.0]], np.float32)
    cu = np.array([0, 3], np.int32)
    for x in range(4):
        for ux in (0.0, 0.125, 0.25, 0.5, 0.75):
            for u0 in (0.0, 0.25, 0.5, 0.75, 1 - 2.0 ** -24):
                check_verify(p, np.array([0, x, 3], np.int32), cu, np.array([u0, ux, ux], np.float32), None, None)
    q = np.array([[0, 0, 0, 0], [0.5, 0.0, 0.5, 0.0], [0.0, 0.0, 0.0, 1.0]], np.float32)
    for x, x2 in ((0, 3), (2, 3), (2, 1)):
        for ux in (0.0, 0.25, 0.5, 0.75):
            for u0 in (0.0, 0.25, 0.5, 1 - 2.0 ** -24):
                check_verify(p, np.array([0, x, x2], np.int32), cu, np.array([u0, ux, 0.999], np.float32), q, None)


def test_verify_siblings():
    """Children of one row: shares of rejected ones leave, a token that comes twice has none the second time, the first accepted one is followed."""
    p = np.zeros((6, 8), np.float32)
    p[0] = [0.5, 0.25, 0.125, 0.125, 0, 0, 0, 0]
    p[1:] = 0.125
    parent, cu = np.array([-1, 0, 0, 0, 0, 2], np.int32), np.array([0, 6], np.int32)
    for toks in ([0, 0, 1, 2, 3, 5], [0, 0, 0, 0, 0, 5], [0, 4, 5, 6, 7, 1], [0, 3, 2, 1, 0, 7], [0, 1, 1, 0, 0, 2]):
        for us in ([0.9] * 6, [0.0] * 6, [0.3, 0.6, 0.6, 0.4, 0.999, 0.5], [0.5, 0.49, 0.51, 0.2, 0.9, 0.99]):
            check_verify(p, np.array(toks, np.int32), cu, np.array(us, np.float32), None, parent, slots=np.arange(10, 16, dtype=np.int32))


def test_verify_where_nothing_is_left():
    cu = np.array([0, 2], np.int32)
    u = np.array([0.5, 0.9999], np.float32)
    p = np.array([[0.0, 0.9, 0.0], [0.2, 0.3, 0.5]], np.float32)       # shares that do not add up to one: the only token is rejected, then drawn all the same
    acc, words, _, _ = check_verify(p, np.array([0, 1], np.int32), cu, u, None, None)
    assert acc[0] == 0 and words[0] == 1
    q = np.array([[0, 0, 0], [0.0, 0.95, 0.05]], np.float32)             # the draft gives every token more than the target
    assert check_verify(p, np.array([0, 1], np.int32), cu, u, q, None)[1][0] == 1
    acc, words, _, _ = check_verify(np.zeros((2, 3), np.float32), np.array([0, 1], np.int32), cu, u, None, None)
    assert acc[0] == 0 and words[0] == -1                                # a distribution without any share
    acc, words, _, _ = check_verify(np.full((2, 700), np.nan, np.float32), np.array([0, 1], np.int32), cu, u, None, None)
    assert acc[0] == 0 and words[0] == -1
    mixed = np.full((1, 1100), np.nan, np.float32)
    mixed[0, [3, 600, 1099]] = [0.25, 0.5, 0.25]
    mixed[0, 7] = -4.0
    for x, word in ((0.0, 3), (0.25, 600), (0.75, 1099), (0.9999999, 1099)):
        assert check_verify(mixed, np.array([0], np.int32), np.array([0, 1], np.int32), np.array([x], np.float32), None, None)[1][0] == word


def test_verify_tokens_outside_the_vocabulary_are_rejected():
    rng = np.random.default_rng(2)
    for bad in (-1, 600, 2 ** 31 - 1, -2 ** 31):
        target, tokens, cu, u, draft, parent = verify_case(rng, [4, 3], 600, False, False)
        tokens[[1, 5]] = bad
        u[[1, 5]] = 0.0
        acc = check_verify(target, tokens, cu, u, None, None)[0]
        assert acc.tolist() == [0, 0]
        check_verify(target, tokens, cu, u, spread(rng, 9, 600), None)


def test_verify_rows_past_the_limit_and_bad_parents():
    rng = np.random.default_rng(6)
    target, tokens, cu, u, _, _ = verify_case(rng, [90, 2], 64, False, False)
    u[:] = 0.0                                                           # everything is accepted, as far as it is looked at
    tokens[1:90] = target[0:89].argmax(1)
    acc, words, _, _ = check_verify(target, tokens, cu, u, None, None)
    assert acc[0] == 63 and (words[64:90] == -1).all()
    parent = rng.integers(-5, 200, 92).astype(np.int32)                  # most of them not an earlier row: those continue row 0
    case = verify_case(rng, [60, 30], 64, False, False)
    check_verify(case[0], case[1], case[2], case[3], None, parent)


def test_verify_refuses():
    import torch
    t = torch.rand(4, 10, device="cuda")
    tok, cu, u = i32([0, 1, 2, 3]), i32([0, 4]), torch.rand(4, device="cuda")
    for a, kw in (((t.half(), tok, cu, u), {}), ((t[:3], tok, cu, u), {}), ((t.t().contiguous().t(), tok, cu, u), {}), ((t, tok.long(), cu, u), {}), ((t, tok, cu, u.double()), {}),
                  ((t, tok, cu, u), dict(draft_probs=t, parent=tok)), ((t, tok, cu, u), dict(draft_probs=t[:, :9])), ((t.cpu(), tok, cu, u), {}), ((t, tok, cu, u), dict(slots=tok[:3]))):
        with pytest.raises(ValueError):
            pkg.verify_sampled(*a, **kw)
    out = [torch.zeros(n, dtype=torch.int32, device="cuda") for n in (1, 4, 4)] + [None]
    for bad in ((t, tok, cu, u, dict(out=(out[0], tok, out[2], None))), (t[:1].expand(4, 10), tok, cu, u, {})):   # outputs over inputs, rows on top of each other
        with pytest.raises(pkg.SdvError):
            pkg.verify_sampled(*bad[:4], **bad[4])
    accepted, words, rows, slots = pkg.verify_sampled(t[:0], tok[:0], i32([0]), u[:0])
    assert accepted.numel() == 0 and words.numel() == 0 and slots is None


# ------------------------------------------------------------------------------------------ the calls themselves
def calls():
    """A call of each operator (without the stream) and the tensors it is given."""
    import torch
    q, k, v, kp, vp, pos, slot = rope_case("bfloat16", 6, 4, 2, 64, 64, False, 8, False, qkv=False)
    f, t = torch.tensor(pkg.rope_frequencies(64)[0], dtype=torch.float64, device="cuda"), torch.rand(6, 10, device="cuda")
    pos, slot, u, cu, length, tok = i32(pos), i32(slot), torch.rand(6, device="cuda"), i32([0, 6]), i32([2]), i32([0, 1, 2, 3, 4, 5])
    table, held, free, state = i32([[0, 1, 2, 3]]), i32([1]), i32([1, 2, 3]), i32([0])
    return [("paged_slots", (length, cu, table, held, free, state, 8, 6), {}),
            ("rope_append", (pos, f, q, k, v, kp, vp, slot), {}),
            ("rope_append", (pos, f), dict(k=k, v=v, k_pages=kp, v_pages=vp, slots=slot)),
            ("tree_attention", (q, kp, vp, table, length, cu), {}),
            ("verify_sampled", (t, tok, cu, u), {}),
            ("verify_sampled", (t, tok, cu, u), dict(draft_probs=t, slots=slot))]


def test_calls_keep_no_references():
    """Neither the arguments nor the results outlive a call, refused or not."""
    import sys
    import torch
    for name, a, kw in calls():
        given = [x for x in (*a, *kw.values()) if torch.is_tensor(x)]
        count = lambda: [sys.getrefcount(x) for x in given] + [sys.getrefcount(None)]  # noqa: E731
        getattr(pkg, name)(*a, **kw)
        torch.cuda.synchronize()
        before, memory = count(), torch.cuda.memory_allocated()
        for _ in range(50):
            r = getattr(pkg, name)(*a, **kw)
            with pytest.raises(ValueError):
                getattr(pkg, name)(a[0][:, None], *a[1:], **kw)
        del r
        after = count()
        assert after[:-1] == before[:-1] and abs(after[-1] - before[-1]) < 25 and torch.cuda.memory_allocated() == memory, name   # None's own count moves a little by itself


def test_calls_refuse_what_is_no_tensor():
    for name, a, kw in calls():
        for i in range(len(a)):
            if not isinstance(a[i], int):
                with pytest.raises(ValueError):
                    getattr(pkg, name)(*a[:i], "no tensor", *a[i + 1:], **kw)
    name, a, kw = calls()[0]
    for out in ((), (a[0],) * 3, (a[0],) * 5, (None,) * 4):
        with pytest.raises(ValueError):
            pkg.paged_slots(*a, out=out)
    for bad in ((*a[:6], 8, -1), (*a[:7], 2 ** 40)):
        with pytest.raises(ValueError):
            pkg.paged_slots(*bad)
    for size in (0, -8, 2 ** 40):
        with pytest.raises(pkg.SdvError):
            pkg.paged_slots(*a[:6], size, 6)
    with pytest.raises(ValueError):
        pkg.verify_sampled(*calls()[4][1], out=(a[0], a[0]))


def test_calls_from_several_threads():
    """Each thread has its own current stream; the answers are those of one thread."""
    import threading
    import torch
    todo = calls()[3:]
    want = [getattr(pkg, n)(*a, **kw) for n, a, kw in todo]
    torch.cuda.synchronize()
    wrong = []

    def work():
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(100):
                    got = [getattr(pkg, n)(*a, **kw) for n, a, kw in todo]
                torch.cuda.current_stream().synchronize()
            same = lambda x, y: torch.equal(x, y) if torch.is_tensor(x) else x is y  # noqa: E731
            for g, w in zip(got, want):
                if not all(same(x, y) for x, y in zip(g, w)):
                    wrong.append(g)
        except Exception as e:   # seen by the test, not by the thread
            wrong.append(e)
    threads = [threading.Thread(target=work) for _ in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_a_failed_launch_is_not_reported_by_another_call():
    """Into a stream whose capture the host has made invalid nothing can be queued; a context that is made afterwards knows nothing of it."""
    import ctypes as C
    import torch
    from paper_2510_15312_b200.binding import Sdv, config_from
    from sdv_inputs import get_config
    todo = calls()
    torch.cuda.synchronize()
    cudart, s, graph = C.CDLL("libcudart.so.12"), C.c_void_p(), C.c_void_p()
    assert cudart.cudaStreamCreate(C.byref(s)) == 0 and cudart.cudaStreamBeginCapture(s, 1) == 0
    assert cudart.cudaStreamSynchronize(s) != 0     # not allowed while capturing
    cudart.cudaGetLastError()                       # torch's runtime keeps its own, the library has another
    a = todo[1][1]
    with pytest.raises(pkg.SdvError):               # (into the pages alone: no output to allocate)
        pkg.rope_append(*a[:2], k=a[3], v=a[4], k_pages=a[5], v_pages=a[6], slots=a[7], stream=torch.cuda.ExternalStream(s.value))
    assert cudart.cudaStreamEndCapture(s, C.byref(graph)) != 0 and cudart.cudaStreamDestroy(s) == 0
    cudart.cudaGetLastError()
    Sdv(config_from(get_config("tiny"), k_max=8)).close()
    for name, a, kw in todo:
        getattr(pkg, name)(*a, **kw)
    torch.cuda.synchronize()
