"""Attention of draft trees over a cache kept in pages, against its definition in 64 bits, and a whole step of the operators together."""
import numpy as np
import pytest

import paged_reference as R
import paper_2510_15312_b200 as pkg
from test_gpu_paged import forest, i32, spread

pytestmark = pytest.mark.gpu


class Case:
    """Sequences with rows and committed tokens in a pool whose unused places hold `junk`."""

    def __init__(self, rows, lengths, hq, hkv, hd, page=16, dtype="bfloat16", tree=False, tokens_first=False, seed=0, junk=float("nan"), pad=2, spare=2, sharp=1.5):
        import torch
        rng = np.random.default_rng(seed)
        self.rng, self.rows, self.lengths, self.hq, self.hkv, self.hd, self.page = rng, rows, lengths, hq, hkv, hd, page
        self.t = getattr(torch, dtype)
        self.cu = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        self.n = int(self.cu[-1]) + pad
        need = [-(-(a + b) // page) for a, b in zip(rows, lengths)]
        pages = sum(need) + spare
        order = rng.permutation(pages).astype(np.int32)
        self.table = np.full((len(rows), max(need) + 1), -3, dtype=np.int32)
        at = 0
        for b, k in enumerate(need):
            self.table[b, :k] = order[at:at + k]
            at += k
        shape = (pages, page, hkv, hd) if tokens_first else (pages, hkv, page, hd)
        k, v = (torch.full(shape, junk, dtype=self.t, device="cuda") for _ in range(2))
        self.k, self.v = (x.transpose(1, 2) if tokens_first else x for x in (k, v))
        for b, (n, length) in enumerate(zip(rows, lengths)):
            for i in range(need[b]):
                m = min(page, n + length - i * page)
                for x in (self.k, self.v):
                    x[int(self.table[b, i]), :, :m] = torch.tensor(rng.standard_normal((hkv, m, hd)), device="cuda").to(self.t)
        self.q = torch.tensor(rng.standard_normal((self.n, hq, hd)) * sharp, device="cuda").to(self.t)
        self.parent = np.concatenate([forest(rng, rows), [-1] * pad]).astype(np.int32) if tree else None

    def run(self, **kw):
        import torch
        out = kw.pop("out", None)
        if out is None:
            out = torch.full(self.q.shape, 77.0, dtype=self.t, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        a = dict(parent=None if self.parent is None else i32(self.parent), out=out, status=status)
        got = pkg.tree_attention(kw.pop("q", self.q), self.k, self.v, i32(self.table), i32(self.lengths), i32(self.cu), **{**a, **kw})
        assert int(status[0]) == 0
        return got

    def tokens(self, b):
        """Keys and values of a sequence, [KV heads][tokens][dim], in 64 bits."""
        n = self.lengths[b] + self.rows[b]
        pages = self.table[b, :-(-n // self.page)]
        return [np.concatenate([x[int(p)].double().cpu().numpy() for p in pages], 1)[:, :n] if len(pages) else np.zeros((self.hkv, 0, self.hd)) for x in (self.k, self.v)]

    def check(self, got, scale=None, only=None, rows=64):
        """The probabilities' rounding to the 16-bit type is off by at most u of each, the result's by u of it; a score's products and sums in fp32 by at most
        hd 2^-24 of the sum of their magnitudes, twice (numerator and denominator), and 2^-21 for the exponentials and sums."""
        import torch
        got = got.double().cpu().numpy()
        scale = self.hd ** -0.5 if scale is None else scale
        u = torch.finfo(self.t).eps / 2
        for b in range(len(self.rows)) if only is None else only:
            r0, n, length = int(self.cu[b]), min(self.rows[b], rows), self.lengths[b]
            if n == 0:
                continue
            k, v = self.tokens(b)
            allowed = np.zeros((n, k.shape[1]), bool)
            allowed[:, :length] = True
            for i in range(n):
                allowed[i, [length + e for e in R.path(self.parent, r0, i)]] = True
            q = self.q[r0:r0 + n].double().cpu().numpy()
            with np.errstate(invalid="ignore", over="ignore"):
                exp, mass, size = R.attention(q, k, v, allowed, scale)
                err = np.abs(got[r0:r0 + n] - exp)
                eps = 2 * self.hd * 2.0 ** -24 * size[..., None] + 2.0 ** -21
                tiny = 2.0 ** -25 if self.t == torch.float16 else 0.0
                # probabilities below fp16's normal range: half a step of 2^-24 each, against a largest of at least one
                low = (2.0 ** -25 * np.abs(v).sum(1).max() if self.t == torch.float16 else 0.0)
                ok = (err <= u * np.abs(exp) + (1 + u) * (u + eps) * mass + tiny + low) | (got[r0:r0 + n] == exp) | (np.isnan(got[r0:r0 + n]) & np.isnan(exp))
            assert ok.all(), (b, np.argwhere(~ok)[:5].tolist(), float(np.nanmax(np.where(ok, 0, err))))
        return self


SHAPES = [(4, 4, 64), (14, 2, 64), (12, 2, 128), (24, 8, 128), (28, 4, 128), (8, 1, 64), (9, 1, 128)]


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("hq,hkv,hd", SHAPES)
@pytest.mark.parametrize("rows,lengths,page,tree", [
    ([1], [0], 16, False),                                   # nothing but itself
    ([1], [1], 8, False),
    ([1, 1, 1], [63, 64, 65], 32, False),                    # around a tile's end
    ([2, 17, 1], [127, 111, 300], 64, True),
    ([9], [700], 128, False),
    ([64, 1, 33], [5, 260, 0], 16, True),                    # trees as wide as they come, from nothing on
    ([0, 5, 0, 0, 3, 0], [40, 12, 0, 9, 129, 50], 8, True),  # sequences without rows
    ([64], [64], 256, False),
])
def test_attention(hq, hkv, hd, dtype, rows, lengths, page, tree):
    import torch
    c = Case(rows, lengths, hq, hkv, hd, page, dtype, tree, tokens_first=(page == 32 or page == 64), seed=page + len(rows))
    got = c.run()
    c.check(got)
    assert bool((got[int(c.cu[-1]):] == 77.0).all())          # rows of no sequence
    assert torch.equal(c.run(), got)                          # the same again, to the bit


@pytest.mark.parametrize("rows,lengths,hq,hkv,hd", [([3] * 50, [37 * i % 900 for i in range(50)], 12, 2, 128), ([1] * 300, [i % 130 for i in range(300)], 4, 4, 64),
                                                    ([5, 1], [9000, 20], 6, 2, 128), ([20, 40, 1, 64], [3000, 2100, 4000, 129], 14, 2, 64), ([17], [20000], 8, 1, 64)])
def test_attention_over_many_shares(rows, lengths, hq, hkv, hd):
    """Sequences of all lengths: shares that hold several of them, sequences that take one, a few, or most of the blocks."""
    Case(rows, lengths, hq, hkv, hd, 32, "float16", True, seed=8).check(Case(rows, lengths, hq, hkv, hd, 32, "float16", True, seed=8).run())


@pytest.mark.parametrize("hq,hkv,hd,rows", [(32, 1, 64, 9), (128, 1, 64, 3), (128, 2, 128, 5), (100, 1, 64, 2), (43, 1, 128, 40), (5, 5, 64, 64)])
def test_groups_of_many_heads(hq, hkv, hd, rows):
    """All heads of a group of as many rows as fit 128 tile rows: one row, two, all of them; tiles that stay partly empty."""
    c = Case([rows, 1, rows], [90, 0, 333], hq, hkv, hd, 16, "float16", True, seed=hq)
    c.check(c.run())


def test_as_many_sequences_as_there_may_be():
    c = Case([1] * 4096, [i % 7 for i in range(4096)], 2, 1, 64, 8, "bfloat16")
    c.check(c.run(), only=range(0, 4096, 97))
    import torch
    d = Case([1] * 2000 + [30] + [1] * 2000, [3] * 2000 + [5000] + [i % 90 for i in range(2000)], 2, 1, 64, 32, "bfloat16")   # a long one among them
    d.check(d.run(), only=[0, 1, 1999, 2000, 2001, 3999, 4000])
    with pytest.raises(pkg.SdvError):
        e = torch.zeros(4097, dtype=torch.int32, device="cuda")
        pkg.tree_attention(c.q, c.k, c.v, e[:, None], e, torch.zeros(4098, dtype=torch.int32, device="cuda"))


def test_maxima_that_keep_growing():
    """Keys sorted so that every tile brings larger scores: the output is rescaled again and again."""
    import torch
    c = Case([6], [1500], 4, 2, 64, 16, sharp=1.0)
    for h in range(2):
        for i, p in enumerate(c.table[0, :-(-1506 // 16)]):
            for t in range(16):
                if i * 16 + t < 1506:
                    c.k[int(p), h, t] = c.k[int(p), h, t] * 0.05 + (c.q[0, h * 2] * (0.0009 * (i * 16 + t))).to(c.t)
    c.check(c.run(scale=3.0), scale=3.0)
    d = Case([3], [400], 2, 1, 128, 16, "float16", sharp=30.0)      # scores of hundreds
    d.check(d.run())
    assert torch.isfinite(d.run()[:3]).all()


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("length", [0, 30, 64, 100, 200])
def test_what_a_row_does_not_see_does_not_reach_it(length, hd, dtype):
    """Infinities, NaN and the type's lowest value in rows of the tree: those who do not see them are as if they were not there, those who do see them."""
    import torch
    c = Case([20, 4], [length, 77], 6, 2, hd, 16, dtype, True, seed=3, junk=float("inf"))
    clean = c.run()
    low = torch.finfo(c.t).min

    def put(x, i, value):
        t = length + i
        x[int(c.table[0, t // 16]), :, t % 16, 5:9] = value
    for i, (kv, vv) in {7: (float("nan"), 1.0), 11: (float("inf"), float("inf")), 13: (low, low), 16: (0.5, float("nan")), 19: (1.0, -float("inf"))}.items():
        put(c.k, i, kv)
        put(c.v, i, vv)
    got = c.run()
    touched = [i for i in range(20) if set(R.path(c.parent, 0, i)) & {7, 11, 13, 16, 19}]
    rest = [i for i in range(20) if i not in touched] + list(range(20, 24))
    assert touched and len(rest) > 6
    assert torch.equal(got[rest], clean[rest])
    c.check(got, only=[1])
    # a row that sees an infinite value behind a finite score has it in its output, in these columns only
    alone = [i for i in touched if set(R.path(c.parent, 0, i)) & {7, 11, 13, 16, 19} == {19}]
    for i in alone:
        assert bool((got[i, :, 5:9] == -float("inf")).all()) and bool(torch.isfinite(got[i, :, 9:]).all())
    assert bool(torch.isnan(got[16, :, 5:9]).all()) and (set(R.path(c.parent, 0, 16)) & {7, 11, 13} or bool(torch.isfinite(got[16, :, 9:]).all()))
    assert bool(torch.isnan(got[7]).all())                     # a NaN among its keys: the whole row


def test_values_of_committed_tokens_reach_everybody():
    import torch
    c = Case([5], [150], 4, 2, 64, 16, tree=True, seed=1)
    c.v[int(c.table[0, 4]), 1, 3, 10] = float("inf")
    got = c.run()
    assert bool((got[:5, 2:, 10] == float("inf")).all()) and int((~torch.isfinite(got[:5])).sum()) == 5 * 2


def test_strides_of_queries_and_outputs():
    import torch
    c = Case([7, 3], [90, 10], 6, 2, 64, tree=True)
    plain = c.run()
    wide = torch.zeros(c.n, 3, 10, 64, dtype=c.t, device="cuda")      # queries between other heads, outputs with the heads outside
    wide[:, 1, 2:8] = c.q
    out = torch.full((6, c.n + 4, 64), 77.0, dtype=c.t, device="cuda").transpose(0, 1)[2:2 + c.n]
    got = c.run(q=wide[:, 1, 2:8], out=out)
    assert got is out and torch.equal(got, plain)
    c.check(plain)


def test_rows_past_the_limit_are_left_alone():
    import torch
    c = Case([70, 2], [100, 5], 4, 2, 64, 16)
    got = c.run()
    c.check(got, rows=64)
    assert bool((got[64:70] == 77.0).all()) and not bool((got[70:72] == 77.0).any())


def test_block_tables_and_lengths_that_hold_anything():
    """Pages outside the pool read as zeros (as the copies fill them: the kernel gives page numbers to the copies only, and compares them before any other read), lengths
    are cut to the table."""
    import torch
    c = Case([3], [40], 4, 2, 64, 16, junk=0.0, spare=6)
    zeros = int(sorted(set(range(c.k.shape[0])) - set(c.table[0, :3].tolist()))[0])
    want = c.table.copy()
    want[0, 1] = zeros
    c.table[0, 1] = 2 ** 31 - 1
    got = c.run()
    c.table = want
    assert torch.equal(got, c.run())
    c.table[0, 1] = -2 ** 31
    assert torch.equal(got, c.run())
    # more tokens than the table has room for: the first ones count
    d = Case([2], [30], 4, 4, 64, 16, junk=0.0)
    d.table = d.table[:, :2].copy()
    d.lengths = [2 ** 31 - 1]
    full = d.run()
    d.lengths, d.rows, d.cu = [30], [2], d.cu
    k, v = d.tokens(0)
    exp, mass, _ = R.attention(d.q[:2].double().cpu().numpy(), k, v, np.ones((2, 32), bool), 64 ** -0.5)
    assert (np.abs(full[:2].double().cpu().numpy() - exp) <= 2.0 ** -8 * np.abs(exp) + (2.0 ** -8 + 1e-4) * mass * (1 + 2.0 ** -8)).all()
    # nothing to see at all: a length of less than nothing and a sequence whose rows descend
    e = Case([2, 2], [0, 0], 4, 4, 64, 16)
    e.lengths, e.cu = [-5, 3], np.array([0, 2, 1], np.int32)
    e.run()


def test_a_long_cache_beyond_32_bit_offsets():
    """A pool of more than 2^31 elements, the sequence's pages at its far end."""
    import torch
    pages, page, hkv, hd = 4100, 64, 64, 128
    k = torch.zeros(pages, hkv, page, hd, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    assert k.numel() > 2 ** 31
    rng = np.random.default_rng(1)
    use = [pages - 1, 3, pages - 2, pages - 3]
    for p in use:
        for x in (k, v):
            x[p] = torch.tensor(rng.standard_normal((hkv, page, hd)), device="cuda").to(x.dtype)
    q = torch.tensor(rng.standard_normal((2, hkv, hd)) * 1.5, device="cuda").to(k.dtype)
    got = pkg.tree_attention(q, k, v, i32([use]), i32([250]), i32([0, 2])).double().cpu().numpy()
    kk, vv = (np.concatenate([x[p].double().cpu().numpy() for p in use], 1)[:, :252] for x in (k, v))
    allowed = np.ones((2, 252), bool)
    allowed[0, 251] = False
    exp, mass, size = R.attention(q.double().cpu().numpy(), kk, vv, allowed, hd ** -0.5)
    assert (np.abs(got - exp) <= 2.0 ** -8 * np.abs(exp) + (1 + 2.0 ** -8) * (2.0 ** -8 + 2 * hd * 2.0 ** -24 * size[..., None] + 2.0 ** -21) * mass).all()
    # and the append, at the pool's last slot
    f = torch.tensor(pkg.rope_frequencies(128)[0], dtype=torch.float64, device="cuda")
    row = torch.tensor(rng.standard_normal((1, hkv, hd)), device="cuda").to(k.dtype)
    pkg.rope_append(i32([0]), f, k=row, v=row, k_pages=k, v_pages=v, slots=i32([pages * page - 1]))
    assert torch.equal(v[pages - 1, :, page - 1], row[0]) and torch.equal(k[pages - 1, :, page - 1], row[0])   # position 0: not rotated


def test_streams_workspaces_and_graphs():
    import torch
    cases = [Case([9, 30], [1000, 333], 12, 2, 128, 16, tree=True, seed=s) for s in range(3)]
    want = [c.run() for c in cases]
    ws = [pkg.tree_attention_workspace(2, 128) for _ in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    outs = []
    for _ in range(5):
        outs = [c.run(stream=s, workspace=w) for c, s, w in zip(cases, streams, ws)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
    # one workspace for calls that follow one another, whatever it holds
    ws[0].fill_(255)
    for c, w in zip(cases, want):
        assert torch.equal(c.run(workspace=ws[0]), w)
    # captured once, replayed on other lengths, tables and values in the same buffers
    c = cases[0]
    q, table, kv, cu, parent = c.q.clone(), i32(c.table), i32(c.lengths), i32(c.cu), i32(c.parent)
    k, v, out = c.k.clone(), c.v.clone(), torch.zeros_like(c.q)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        pkg.tree_attention(q, k, v, table, kv, cu, parent=parent, out=out, workspace=ws[1])
    for c, w in zip(cases, want):
        for dst, src in ((q, c.q), (table, i32(c.table)), (kv, i32(c.lengths)), (cu, i32(c.cu)), (parent, i32(c.parent)), (k, c.k), (v, c.v)):
            dst.copy_(src)
        for _ in range(2):
            out.fill_(77.0)
            g.replay()
            assert torch.equal(out, w)
    kv.copy_(i32([500, 3]))
    c.lengths = [500, 3]
    g.replay()
    assert torch.equal(out[:39], c.run()[:39])


def test_two_graphs_with_one_workspace():
    """Replayed one after the other on one stream they may share it."""
    import torch
    a, b = Case([9], [3000], 12, 2, 128, 16, seed=1), Case([4, 4], [500, 1200], 12, 2, 128, 16, tree=True, seed=2)
    want = [a.run(), b.run()]
    ws = pkg.tree_attention_workspace(2, 128)
    outs, graphs, held = [], [], []
    for c in (a, b):
        args = dict(block_table=i32(c.table), kv_len=i32(c.lengths), cu_rows=i32(c.cu), parent=None if c.parent is None else i32(c.parent))
        out = torch.full_like(c.q, 77.0)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            pkg.tree_attention(c.q, c.k, c.v, out=out, workspace=ws, **args)
        outs.append(out)
        graphs.append(g)
        held.append(args)
    for order in ((0, 1), (1, 0), (0, 0), (1, 1)):
        for k in order:
            outs[k].fill_(77.0)
            graphs[k].replay()
        assert all(torch.equal(outs[k], want[k]) for k in order)


def test_a_captured_step():
    """All four operators in one graph, replayed on other inputs in the same buffers: as called one by one."""
    import torch
    rng = np.random.default_rng(4)
    hq, hkv, hd, page, vocab, rows = 6, 2, 128, 16, 3000, [9, 5, 20]
    cu, n = i32([0, 9, 14, 34]), 34
    parent, f = i32(forest(rng, rows, 4)), torch.tensor(pkg.rope_frequencies(hd)[0], dtype=torch.float64, device="cuda")
    kv, held, state, table = i32([200, 0, 90]), i32([13, 0, 6]), i32([0, 0]), torch.full((3, 30), -1, dtype=torch.int32, device="cuda")
    pages = rng.permutation(60).astype(np.int32)
    table[0, :13], table[2, :6] = i32(pages[:13]), i32(pages[13:19])
    free = i32(pages[19:])
    q, k, v = (torch.zeros(n, h, hd, dtype=torch.bfloat16, device="cuda") for h in (hq, hkv, hkv))
    kp, vp = (torch.tensor(rng.standard_normal((60, hkv, page, hd)), device="cuda").bfloat16() for _ in range(2))
    target, tokens, u = torch.zeros(n, vocab, device="cuda"), i32(np.zeros(n)), torch.zeros(n, device="cuda")

    def fill(seed):
        r = np.random.default_rng(seed)
        for x in (q, k, v):
            x.copy_(torch.tensor(r.standard_normal(tuple(x.shape))).bfloat16())
        p = spread(r, n, vocab)
        target.copy_(torch.tensor(p))
        tokens.copy_(torch.tensor(p.argmax(1).astype(np.int32)).roll(1))
        u.copy_(torch.tensor(r.random(n).astype(np.float32)))
        kv.copy_(torch.tensor([200 - seed, 0, 90 + seed], dtype=torch.int32))

    def step():
        slots, pos, h, s = pkg.paged_slots(kv, cu, table, held, free, state, page, n, parent=parent)
        qr = pkg.rope_append(pos, f, q=q, k=k, v=v, k_pages=kp, v_pages=vp, slots=slots)
        out = pkg.tree_attention(qr, kp, vp, table, kv, cu, parent=parent)
        return (slots, pos, h, s, qr, out) + tuple(pkg.verify_sampled(target, tokens, cu, u, parent=parent, slots=slots))

    fill(0)
    step()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step()
    for seed in (1, 2, 3):
        fill(seed)
        want = [x.clone() for x in step()]
        for x in got:
            x.zero_()
        g.replay()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_attention_refuses():
    import torch
    c = Case([2], [20], 4, 2, 64)
    a = dict(q=c.q, k_pages=c.k, v_pages=c.v, block_table=i32(c.table), kv_len=i32([20]), cu_rows=i32([0, 2]))
    for bad in (dict(q=c.q.float()), dict(q=c.q.half()), dict(q=c.q[..., :32]), dict(k_pages=c.k[:1]), dict(v_pages=c.v.half()), dict(v_pages=c.v.transpose(2, 3)), dict(kv_len=i32([20, 1])),
                dict(cu_rows=i32([0, 1, 2])), dict(cu_rows=i32([0, 2]).long()), dict(block_table=a["block_table"].long()), dict(block_table=a["block_table"][0]), dict(q=c.q.cpu()),
                dict(kv_len=i32([20]).cpu()), dict(parent=i32([0])), dict(out=c.q.half()), dict(out=c.q[:1]), dict(k_pages=c.k.float(), v_pages=c.v.float(), q=c.q.float())):
        with pytest.raises(ValueError):
            pkg.tree_attention(**{**a, **bad})
    for bad in (dict(q=c.q[:, :1].expand(c.n, 4, 64)), dict(q=c.q[:1].expand(c.n, 4, 64)), dict(out=torch.empty(c.n, 1, 64, dtype=c.t, device="cuda").expand(c.n, 4, 64)),
                dict(k_pages=c.k[:, :1].expand_as(c.k), v_pages=c.v[:, :1].expand_as(c.v)), dict(scale=0.0), dict(scale=float("nan")), dict(workspace=torch.empty(1 << 10, dtype=torch.uint8, device="cuda")), dict(q=c.q[:, :3]), dict(q=c.q.view(-1)[4:4 + 4 * 64].view(1, 4, 64)),
                dict(out=torch.empty(c.n * 256 + 1, dtype=c.t, device="cuda")[1:].view(c.n, 4, 64))):
        with pytest.raises(pkg.SdvError):
            pkg.tree_attention(**{**a, **bad})
    with pytest.raises(pkg.SdvError) as e:
        pkg.tree_attention(**a, workspace=torch.empty(1 << 10, dtype=torch.uint8, device="cuda"))
    assert e.value.code == pkg.ENOMEM
    host = torch.empty(1 << 12, dtype=torch.uint8).pin_memory()
    import ctypes as C
    from paged_structs import AttentionArgs, Pages
    pages = Pages(c.k.data_ptr(), c.v.data_ptr(), 0, c.k.shape[0], 16, 2, 64, *c.k.stride()[:3])
    args = AttentionArgs(q=host.data_ptr() + 256 - host.data_ptr() % 256, out=c.q.data_ptr(), block_table=a["block_table"].data_ptr(), kv_len=a["kv_len"].data_ptr(),
                         cu_rows=a["cu_rows"].data_ptr(), workspace=c.q.data_ptr(), workspace_bytes=1 << 30, q_row_stride=256, q_head_stride=64, out_row_stride=256, out_head_stride=64,
                         table_stride=8, n_seqs=1, n_rows=2, n_q_heads=4, table_width=2, scale=1.0)
    assert pkg.lib().sdv_tree_attention(C.byref(args), C.byref(pages), None) == pkg.EINVAL     # host memory
    with pytest.raises(pkg.SdvError):
        pkg.tree_attention_workspace(5000, 64)


@pytest.mark.parametrize("tree", [False, True])
def test_steps_of_all_operators_together(tree):
    """Three sequences through several steps: pages handed out, rows rotated and appended, attention over cache and trees, drafts verified, accepted rows moved to their places. After
    every step the cache holds the rotated keys and the values of the accepted tokens, in order, and the next step's attention is the definition's over them."""
    import torch
    hq, hkv, hd, page, vocab = 6, 2, 64, 8, 60
    rng = np.random.default_rng(17 + tree)
    f = np.array(pkg.rope_frequencies(hd, 1.0e4)[0])
    fd = torch.tensor(f, device="cuda")
    k_pages, v_pages = (torch.full((60, hkv, page, hd), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.full((3, 16), -1, dtype=torch.int32, device="cuda")
    kv, held, free, state = i32([0, 0, 0]), i32([0, 0, 0]), i32(rng.permutation(60)), i32([0, 0])
    cache = [[np.zeros((hkv, 0, hd)), np.zeros((hkv, 0, hd))] for _ in range(3)]      # what should be there, as the 16-bit type holds it
    accepted_in_all = moved_in_all = 0
    for step in range(6):
        rows = [int(rng.integers(1, 14)) for _ in range(3)] if step else [13, 5, 9]
        cu = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        n = int(cu[-1])
        parent = forest(rng, rows, 3) if tree and step else None
        q, k, v = (torch.tensor(rng.standard_normal((n, h, hd)), device="cuda").bfloat16() for h in (hq, hkv, hkv))
        dparent = None if parent is None else i32(parent)
        slots, pos, held, state = pkg.paged_slots(kv, i32(cu), table, held, free, state, page, n, parent=dparent)
        assert int(state[1]) == 0
        qr = pkg.rope_append(pos, fd, q=q, k=k, v=v, k_pages=k_pages, v_pages=v_pages, slots=slots)
        out = pkg.tree_attention(qr, k_pages, v_pages, table, kv, i32(cu), parent=dparent)
        kr, _ = R.rope(k.double().cpu().numpy(), pos.cpu().numpy(), f, 1.0, False)
        kr = torch.tensor(kr).bfloat16().double().numpy()
        vr, qn = v.double().cpu().numpy(), qr.double().cpu().numpy()
        for b, (r0, r1) in enumerate(R.spans(cu)):
            length = cache[b][0].shape[1]
            assert int(kv[b]) == length
            kk, vv = np.concatenate([cache[b][0], kr[r0:r1].transpose(1, 0, 2)], 1), np.concatenate([cache[b][1], vr[r0:r1].transpose(1, 0, 2)], 1)
            allowed = np.zeros((r1 - r0, kk.shape[1]), bool)
            allowed[:, :length] = True
            for i in range(r1 - r0):
                allowed[i, [length + e for e in R.path(parent, r0, i)]] = True
            exp, mass, size = R.attention(qn[r0:r1], kk, vv, allowed, hd ** -0.5)
            # as in Case.check, and the keys' last bit: rotation in 32 and in 64 bits may round an element to either side, u of it in a score
            eps = (2 * hd * 2.0 ** -24 + 2 * 2.0 ** -8) * size[..., None] + 2.0 ** -21
            assert (np.abs(out[r0:r1].double().cpu().numpy() - exp) <= 2.0 ** -8 * np.abs(exp) + (1 + 2.0 ** -8) * (2.0 ** -8 + eps) * mass).all()
        if step == 0:      # the first step is the prompts: all rows are kept
            keep = [list(range(r)) for r in rows]
            kv = i32([len(x) for x in keep])
        else:
            target = spread(rng, n, vocab)
            tokens = np.array([np.argsort(target[r0 + max(R.up(parent, r0, i), 0)])[-1 - int(rng.integers(0, 2))] for r0, r1 in R.spans(cu) for i in range(r1 - r0)], np.int32)
            u = rng.random(n).astype(np.float32)
            acc, words, kept, moved = pkg.verify_sampled(torch.tensor(target, device="cuda"), i32(tokens), i32(cu), torch.tensor(u, device="cuda"), parent=dparent, slots=slots)
            e = R.verify(target, tokens, cu, u, None, parent, slots.cpu().numpy())
            for g, x in zip((acc, words, kept, moved), e):
                np.testing.assert_array_equal(g.cpu().numpy(), x)
            pkg.rope_append(pos, fd, k=k, v=v, k_pages=k_pages, v_pages=v_pages, slots=moved)
            keep = [[int(x) for x in kept[r0:r0 + int(acc[b]) + 1]] for b, (r0, r1) in enumerate(R.spans(cu))]
            kv = kv + acc + 1
            accepted_in_all += int(acc.sum())
            moved_in_all += int((moved >= 0).sum())
        for b, (r0, r1) in enumerate(R.spans(cu)):
            rows_kept = [r0 + i for i in keep[b]]
            cache[b] = [np.concatenate([cache[b][0], kr[rows_kept].transpose(1, 0, 2)], 1), np.concatenate([cache[b][1], vr[rows_kept].transpose(1, 0, 2)], 1)]
            m = cache[b][0].shape[1]
            pages = table[b, :-(-m // page)].tolist()
            kk, vv = (np.concatenate([x[p].double().cpu().numpy() for p in pages], 1)[:, :m] for x in (k_pages, v_pages))
            assert np.array_equal(vv, cache[b][1])
            assert (np.abs(kk - cache[b][0]) <= 2.0 ** -7 * np.abs(cache[b][0]) + 2.0 ** -20).all()
            cache[b][0] = kk
    assert accepted_in_all > 5 and (moved_in_all > 0 or not tree)
    assert len(set(int(p) for row in table.tolist() for p in row if p >= 0)) == int(held.sum()) == int(state[0])    # no page twice
