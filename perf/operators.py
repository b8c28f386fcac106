"""Operators of a batched speculative step on a cache kept in pages, as timed cases.

A serving program that verifies drafted tokens for several requests at once does four things with them besides the
dense layers, in this order:

  slots   pages are handed to the requests that need more, every drafted row gets its position and its place in the cache
  rope    queries and keys are turned by their positions, keys and values are written to their places
  attend  every drafted row attends to its request's cache and to the rows on its own path through the draft tree
  verify  drafts are accepted against the target model's probabilities, one token is sampled behind the accepted ones

A request's rows are row 0, the committed token, and its drafts; rows of all requests lie one behind the other, request b
has rows cu_rows[b] .. cu_rows[b + 1].  A cache of `page` tokens a page is [pages][KV heads][page][head dim], whatever its
strides; slot s of the cache is token s % page of page s // page.
"""
from __future__ import annotations

import math
from types import SimpleNamespace

import numpy as np
import torch

own = False

# Head layouts (query heads, KV heads, head dim) of the configurations in sdv_inputs/configs.py, and one KV head for eight queries.
HEADS = ((4, 4, 64), (14, 2, 64), (12, 2, 128), (24, 8, 128), (28, 4, 128), (10, 2, 64), (6, 2, 128), (8, 1, 64))
VOCABS = (2016, 3024, 4096, 128256, 151936, 152064)
# No attention case moves more bytes or computes more than these, no other case is larger than its kind's largest listed one.
ATTEND_BYTES, ATTEND_FLOPS = 6.0e8, 1.8e10
ROPE_ELEMENTS, VERIFY_ELEMENTS, SLOT_ROWS, SLOT_PAGES = 8191 * 32 * 128, 64 * 9 * 152064, 24000, 32000


def listed():
    return [
        # a few requests with tree drafts: a single launch's latency
        dict(name="slots 5 trees", kind="slots", batch=5, rows=20, ctx=1500, page=16, tree=True, ragged=False, fresh=False),
        # a full server: many requests, from one row to whole prompts, pages for all of it
        dict(name="slots 1000 requests", kind="slots", batch=1000, rows=47, ctx=2048, page=32, tree=False, ragged=True, fresh=True),
        # the rows of one chain of drafts at the 1.5B shape
        dict(name="rope 9 rows", kind="rope", rows=9, hq=12, hkv=2, hd=128, rot=128, interleaved=False, scaling="none", dtype="bfloat16", page=16, ctx=2048, tokens_first=False),
        # a batch of draft trees at the 0.5B shape, far positions, frequencies in three bands
        dict(name="rope 517 rows banded fp16", kind="rope", rows=517, hq=14, hkv=2, hd=64, rot=64, interleaved=False, scaling="banded", dtype="float16", page=64, ctx=100000, tokens_first=True),
        # a prompt at the 3B shape, half of every head turned, neighbours paired
        dict(name="rope prompt 8191 rows", kind="rope", rows=8191, hq=24, hkv=8, hd=128, rot=64, interleaved=True, scaling="yarn", dtype="bfloat16", page=32, ctx=40000, tokens_first=False),
        # one token of one short request at the smallest shape: latency
        dict(name="attend 1 token tiny", kind="attend", batch=1, rows=1, hq=4, hkv=4, hd=64, ctx=511, page=16, tree=False, ragged=False, dtype="bfloat16", tokens_first=False),
        # one request's chain of drafts behind a long context: the work has to be split along the cache
        dict(name="attend chain 17 of 65536", kind="attend", batch=1, rows=17, hq=12, hkv=2, hd=128, ctx=65535, page=64, tree=False, ragged=False, dtype="bfloat16", tokens_first=True),
        # draft trees of requests of all lengths, wide trees whose rows fill several tiles
        dict(name="attend 24 trees of 40", kind="attend", batch=24, rows=40, hq=24, hkv=8, hd=128, ctx=4096, page=16, tree=True, ragged=True, dtype="bfloat16", tokens_first=False),
        # plain decoding of a full batch at the 7B shape, one token each: the cache is read once
        dict(name="attend 64 tokens of 8192", kind="attend", batch=64, rows=1, hq=28, hkv=4, hd=128, ctx=8192, page=32, tree=False, ragged=True, dtype="float16", tokens_first=False),
        # one request, eight retrieved drafts (no draft distribution)
        dict(name="verify chain 9", kind="verify", batch=1, rows=9, vocab=151936, tree=False, drafts=False),
        # requests with draft trees
        dict(name="verify 12 trees of 21", kind="verify", batch=12, rows=21, vocab=128256, tree=True, drafts=False),
        # a full batch whose drafts a small model sampled
        dict(name="verify 64 sampled chains", kind="verify", batch=64, rows=9, vocab=152064, tree=False, drafts=True),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("slots", "rope", "attend", "attend", "verify"))
    flip = lambda: rng.random() < 0.5  # noqa: E731
    page = rng.choice((8, 16, 32, 64, 128))
    if kind == "slots":
        tree = flip()
        batch = _log(rng, 1, 1000)
        rows = _log(rng, 1, min(64 if tree else SLOT_ROWS, max(1, SLOT_ROWS // batch)))
        return dict(kind=kind, batch=batch, rows=rows, ctx=min(_log(rng, 1, 2048), max(1, SLOT_PAGES * page // batch)), page=page, tree=tree, ragged=flip(), fresh=flip())
    hq, hkv, hd = rng.choice(HEADS)
    dtype, tokens_first = rng.choice(("bfloat16", "float16")), flip()
    if kind == "rope":
        rows = min(_log(rng, 1, 8191), ROPE_ELEMENTS // ((hq + 2 * hkv) * hd))
        return dict(kind=kind, rows=rows, hq=hq, hkv=hkv, hd=hd, rot=2 * rng.randint(hd // 8, hd // 2), interleaved=flip(), scaling=rng.choice(("none", "linear", "banded", "yarn")),
                    dtype=dtype, page=page, ctx=_log(rng, 1, 1000000), tokens_first=tokens_first)
    if kind == "attend":
        case = dict(kind=kind, batch=_log(rng, 1, 64), rows=_log(rng, 1, 64), hq=hq, hkv=hkv, hd=hd, ctx=_log(rng, 1, 65536), page=page, tree=flip(), ragged=flip(), dtype=dtype,
                    tokens_first=tokens_first)
        while case["batch"] * case["ctx"] * hkv * hd * 4 > ATTEND_BYTES or case["batch"] * case["ctx"] * case["rows"] * hq * hd * 4 > ATTEND_FLOPS:
            case["batch" if case["batch"] > 1 and flip() else "ctx"] //= 2
        return case
    vocab, rows, tree = rng.choice(VOCABS), _log(rng, 1, 64), flip()
    batch = _log(rng, 1, min(64, max(1, VERIFY_ELEMENTS // (vocab * rows))))
    return dict(kind=kind, batch=batch, rows=rows, vocab=vocab + rng.choice((0, 0, 1, 7)), tree=tree, drafts=not tree and flip())


# ------------------------------------------------------------------------------------------ inputs
def _spread(most, n, least):
    """n numbers between `least` and `most`, spread evenly in no order, the largest among them; the same ones every time."""
    if n == 1:
        return [most]
    return [most] + [least + int((most - least + 1) * ((i * 0.6180339887498949) % 1.0)) for i in range(1, n)]


def _lengths(case):
    """(rows, committed tokens) of every request."""
    n = case["batch"]
    if not case["ragged"]:
        return [case["rows"]] * n, [case["ctx"]] * n
    return _spread(case["rows"], n, 1), _spread(case["ctx"], n, 0 if case["kind"] == "slots" else min(case["ctx"], 1 + case["ctx"] // 8))


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _cu(rows):
    return _i32([0] + np.cumsum(rows).tolist())


def _trees(rng, rows):
    """Parents of every request's rows: mostly the row before, else an earlier one."""
    out = []
    for n in rows:
        out += [-1] + [i - 1 if rng.random() < 0.55 else int(rng.integers(max(0, i - 6), i)) for i in range(1, n)]
    return _i32(out)


def _pool(gen, case, pages):
    """Keys and values in pages, [pages][KV heads][page][head dim]; tokens_first: the tokens of a page are the outer of the two in memory."""
    shape = (pages, case["page"], case["hkv"], case["hd"]) if case["tokens_first"] else (pages, case["hkv"], case["page"], case["hd"])
    pair = [torch.randn(shape, generator=gen, device="cuda", dtype=getattr(torch, case["dtype"])) for _ in range(2)]
    return [p.transpose(1, 2) if case["tokens_first"] else p for p in pair]


def _frequencies(case):
    """Angles per position of the turned pairs in 64 bits and the factor on cosine and sine."""
    rot, theta, factor, before = case["rot"], 1.0e6, 8.0, 8192
    f = theta ** (-np.arange(rot // 2, dtype=np.float64) * 2 / rot)
    if case["scaling"] == "linear":
        return f / factor, 1.0
    if case["scaling"] == "banded":   # long waves slowed down, short ones kept, a straight line between them
        keep = np.clip((before * f / (2 * math.pi) - 1.0) / (4.0 - 1.0), 0.0, 1.0)
        return f / factor * (1 - keep) + f * keep, 1.0
    if case["scaling"] == "yarn":     # the line in the pair's number
        at = lambda turns: rot * math.log(before / (turns * 2 * math.pi)) / (2 * math.log(theta))  # noqa: E731
        lo, hi = max(math.floor(at(32.0)), 0), min(math.ceil(at(1.0)), rot - 1)
        slow = np.clip((np.arange(rot // 2) - lo) / max(hi - lo, 0.001), 0.0, 1.0)
        return f / factor * slow + f * (1 - slow), 0.1 * math.log(factor) + 1.0
    return f, 1.0


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    st = SimpleNamespace(case=case)
    if case["kind"] == "rope":
        n, total = case["rows"], case["rows"] + case["page"] * 3
        dtype = getattr(torch, case["dtype"])
        # one product gives queries, keys and values side by side
        qkv = torch.randn((n, (case["hq"] + 2 * case["hkv"]) * case["hd"]), generator=gen, device="cuda").to(dtype)
        st.q, st.k, st.v = (t.unflatten(1, (-1, case["hd"])) for t in qkv.split([h * case["hd"] for h in (case["hq"], case["hkv"], case["hkv"])], 1))
        st.k_pages, st.v_pages = _pool(gen, case, -(-total // case["page"]))
        first = int(rng.integers(0, case["ctx"]))
        st.positions = _i32(first + np.arange(n) - (rng.random(n) < 0.3) * np.minimum(np.arange(n), 1))
        slots = rng.permutation(st.k_pages.shape[0] * case["page"])[:n]
        slots[rng.random(n) < 0.03] = -1      # rows of padding are not written
        st.slots = _i32(slots)
        f, st.factor = _frequencies(case)
        st.frequencies = torch.tensor(f, dtype=torch.float64, device="cuda")
        return st
    if case["kind"] == "verify":
        n, v = case["batch"] * case["rows"], case["vocab"]
        st.cu_rows, st.most_rows = _cu([case["rows"]] * case["batch"]), case["rows"]
        st.parent = _trees(rng, [case["rows"]] * case["batch"]) if case["tree"] else None
        st.target = torch.empty((n, v), device="cuda")
        st.draft = torch.empty((n, v), device="cuda") if case["drafts"] else None
        st.tokens = torch.zeros(n, dtype=torch.int32, device="cuda")
        local = np.arange(n) % case["rows"]
        before = np.arange(n) - 1 if not case["tree"] else np.arange(n) - local + st.parent.cpu().numpy()
        best = torch.empty((n, 4), dtype=torch.int64, device="cuda")
        for at in range(0, n, 64):            # a model's predictions: a few likely tokens, a long tail
            logits = torch.randn((min(64, n - at), v), generator=gen, device="cuda") * 2.0
            st.target[at:at + 64] = torch.softmax(logits * 1.4, 1)
            best[at:at + 64] = st.target[at:at + 64].topk(4, 1).indices
            st.target[at:at + 64].scatter_add_(1, best[at:at + 64], torch.tensor([[0.5, 0.2, 0.1, 0.05]], device="cuda").expand(logits.shape[0], 4) * 2)
            st.target[at:at + 64] /= st.target[at:at + 64].sum(1, keepdim=True)
        pick = torch.tensor(rng.integers(0, 4, n), device="cuda")
        held = torch.tensor(np.maximum(before, 0), device="cuda")
        st.tokens[:] = best[held, pick].to(torch.int32)   # retrieved drafts: mostly what the model finds likely
        if case["drafts"]:                    # a small model's distribution: the target's for the row before, blurred; the draft is a sample of it
            for at in range(0, n, 64):
                p = st.target[held[at:at + 64]]
                noise = torch.rand(p.shape, generator=gen, device="cuda") * 1.5 + 0.25
                q = p * noise
                st.draft[at:at + 64] = q / q.sum(1, keepdim=True)
            u = torch.tensor(rng.random((n, 1)), device="cuda")
            for at in range(0, n, 64):
                c = st.draft[at:at + 64].double().cumsum(1)
                st.tokens[at:at + 64] = torch.searchsorted(c, u[at:at + 64] * c[:, -1:], right=True).clamp(max=v - 1).squeeze(1).to(torch.int32)
        st.uniforms = torch.tensor(rng.random(n), device="cuda").float().clamp(max=1 - 2.0 ** -24)
        # where each row lies in the cache, as the pages were handed out
        st.slots = _i32(rng.permutation(4 * n)[:n])
        return st

    rows, lengths = _lengths(case)
    page, n = case["page"], sum(rows)
    st.cu_rows, st.kv_len, st.most_rows, st.most_keys = _cu(rows), _i32(lengths), max(rows), max(a + b for a, b in zip(rows, lengths))
    st.parent = _trees(rng, rows) if case["tree"] else None
    needed = [-(-(a + b) // page) for a, b in zip(rows, lengths)]
    width = max(needed) + 2
    if case["kind"] == "slots":
        # fresh: no request has a page yet; otherwise those of its committed tokens
        held = [0 if case["fresh"] else -(-b // page) for b in lengths]
        order = rng.permutation(sum(needed) + 7).astype(np.int32)
        table, at = np.full((case["batch"], width), -1, dtype=np.int32), 0
        for b, h in enumerate(held):
            table[b, :h] = order[at:at + h]
            at += h
        st.rows, st.n_held, st.block_table, st.free_pages = n, _i32(held), torch.tensor(table, device="cuda"), torch.tensor(order[at:], device="cuda")
        st.free_state = _i32([3, 0])          # three of the list's pages were given away before
        return st
    dtype = getattr(torch, case["dtype"])
    pages = sum(needed) + 3
    order, at = rng.permutation(pages).astype(np.int32), 0
    table = np.full((case["batch"], width), -1, dtype=np.int32)
    for b, k in enumerate(needed):
        table[b, :k] = order[at:at + k]
        at += k
    st.block_table = torch.tensor(table, device="cuda")
    st.k_pages, st.v_pages = _pool(gen, case, pages)
    # scores with a spread of a few units, as trained heads have them
    st.q = (torch.randn((n, case["hq"], case["hd"]), generator=gen, device="cuda") * 1.7).to(dtype)
    st.scale = case["hd"] ** -0.5
    return st


# ------------------------------------------------------------------------------------------ one pass
def run(state):
    return {"slots": _slots, "rope": _rope, "attend": _attend, "verify": _verify}[state.case["kind"]](state)


def _requests(cu_rows, n):
    """(request, row within it) of rows 0 .. n - 1."""
    row = torch.arange(n, device="cuda")
    b = torch.searchsorted(cu_rows, row, right=True) - 1
    return b, row - cu_rows[b]


def _paths(parent, b, local, batch, most):
    """[request][row][row]: whether the second is the first or one of those it continues."""
    step = torch.zeros((batch, most, most), device="cuda")
    step[b, local, local] = 1.0
    step[b, local, parent.clamp(min=0).long()] = 1.0
    return torch.linalg.matrix_power(step, 64) > 0 if most > 1 else step > 0   # at most 64 rows: every path in 63 steps


def _slots(st):
    page = st.case["page"]
    if own:
        import paper_2510_15312_b200 as sdv
        slots, positions, held, free = sdv.paged_slots(st.kv_len, st.cu_rows, st.block_table, st.n_held, st.free_pages, st.free_state, page, st.rows, parent=st.parent)
        return dict(slots=slots, positions=positions, held=held, free=free, table=st.block_table)
    batch, width = st.block_table.shape
    rows = st.cu_rows[1:] - st.cu_rows[:-1]
    want = torch.where(rows > 0, (st.kv_len + rows + page - 1) // page, 0)
    need = torch.where(want <= width, (want - st.n_held).clamp(min=0), 0)
    end = st.free_state[0] + need.cumsum(0)
    fits = (want <= width) & ((need == 0) | (end <= st.free_pages.numel()))
    held = torch.where(fits, st.n_held + need, st.n_held).to(torch.int32)
    column = torch.arange(width, device="cuda")[None]
    new = (column >= st.n_held[:, None]) & (column < held[:, None])
    source = ((end - need)[:, None] + column - st.n_held[:, None]).clamp(0, st.free_pages.numel() - 1)
    st.block_table.copy_(torch.where(new, st.free_pages[source], st.block_table))
    b, local = _requests(st.cu_rows, st.rows)
    depth = local if st.parent is None else _paths(st.parent, b, local, batch, st.most_rows).sum(2)[b, local] - 1
    at = st.kv_len[b] + local
    slots = torch.where(fits[b], st.block_table[b, (at // page).clamp(max=width - 1)] * page + at % page, -1).to(torch.int32)
    free = torch.stack([torch.where(fits, end, st.free_state[0]).max(), (~fits).sum()]).to(torch.int32)
    return dict(slots=slots, positions=(st.kv_len[b] + depth).to(torch.int32), held=held, free=free, table=st.block_table)


def _turn(x, cosine, sine, rot, interleaved):
    x = x.float()
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    y, z = a * cosine - b * sine, b * cosine + a * sine
    turned = torch.stack((y, z), -1).flatten(-2) if interleaved else torch.cat((y, z), -1)
    return torch.cat((turned, x[..., rot:]), -1)


def _rope(st):
    c = st.case
    if own:
        import paper_2510_15312_b200 as sdv
        q = sdv.rope_append(st.positions, st.frequencies, q=st.q, k=st.k, v=st.v, k_pages=st.k_pages, v_pages=st.v_pages, slots=st.slots, interleaved=c["interleaved"],
                            factor=st.factor)
        return dict(q=q, k_pages=st.k_pages, v_pages=st.v_pages)
    angle = st.positions.double()[:, None] * st.frequencies[None]
    cosine, sine = ((t * st.factor).float()[:, None] for t in (angle.cos(), angle.sin()))
    q = _turn(st.q, cosine, sine, c["rot"], c["interleaved"]).to(st.q.dtype)
    k = _turn(st.k, cosine, sine, c["rot"], c["interleaved"]).to(st.q.dtype)
    written = (st.slots >= 0)[:, None, None]
    page, token = st.slots.clamp(min=0) // c["page"], st.slots.clamp(min=0) % c["page"]
    keep = torch.arange(st.slots.shape[0], device="cuda")
    # rows of padding repeat a written one
    some = torch.where(st.slots >= 0, keep, torch.argmax((st.slots >= 0).int()))
    page, token = page[some], token[some]
    any_written = written.any()
    at = (page[:, None], torch.arange(c["hkv"], device="cuda")[None], token[:, None])
    st.k_pages.index_put_(at, torch.where(any_written, k[some], st.k_pages[at]))
    st.v_pages.index_put_(at, torch.where(any_written, st.v[some], st.v_pages[at]))
    return dict(q=q, k_pages=st.k_pages, v_pages=st.v_pages)


def _attend(st):
    c = st.case
    if own:
        import paper_2510_15312_b200 as sdv
        return sdv.tree_attention(st.q, st.k_pages, st.v_pages, st.block_table, st.kv_len, st.cu_rows, parent=st.parent, scale=st.scale)
    n, batch, most = st.q.shape[0], st.kv_len.shape[0], st.most_rows
    b, local = _requests(st.cu_rows, n)
    columns = -(-st.most_keys // c["page"])
    table = st.block_table[:, :columns].clamp(min=0).long()
    keys, values = (p[table].transpose(1, 2).flatten(2, 3).float() for p in (st.k_pages, st.v_pages))     # [request][KV head][token][dim]
    key = torch.arange(columns * c["page"], device="cuda")
    inside = key[None] < (st.kv_len + st.cu_rows[1:] - st.cu_rows[:-1])[:, None]
    values = values * inside[:, None, :, None]                                                           # behind a request's end lies anything
    q = torch.zeros((batch, most, c["hq"], c["hd"]), device="cuda")
    q[b, local] = st.q.float()
    q = q.view(batch, most, c["hkv"], -1, c["hd"]).permute(0, 2, 1, 3, 4).flatten(2, 3)                   # [request][KV head][row, head][dim]
    if st.parent is None:
        path = torch.ones((most, most), device="cuda").tril().bool().expand(batch, most, most)
    else:
        path = _paths(st.parent, b, local, batch, most)
    # a row sees the cache and its own path
    new = key[None] - st.kv_len[:, None]                                                                 # which row of the request a key is
    sees = (new < 0)[:, None] | ((new >= 0) & (new < most))[:, None] & path.gather(2, new.clamp(0, most - 1)[:, None].expand(batch, most, -1))
    sees = sees & inside[:, None]
    scores = (q @ keys.transpose(2, 3)) * st.scale
    scores = scores.masked_fill(~sees[:, None].repeat_interleave(c["hq"] // c["hkv"], 2), -math.inf)
    top = scores.amax(3, keepdim=True)
    weights = (scores - torch.where(top == -math.inf, 0.0, top)).exp()
    out = (weights @ values) / weights.sum(3, keepdim=True)
    out = out.view(batch, c["hkv"], most, -1, c["hd"]).permute(0, 2, 1, 3, 4).flatten(2, 3)
    return out[b, local].to(st.q.dtype)


def _verify(st):
    if own:
        import paper_2510_15312_b200 as sdv
        accepted, tokens, rows, slots = sdv.verify_sampled(st.target, st.tokens, st.cu_rows, st.uniforms, draft_probs=st.draft, parent=st.parent, slots=st.slots)
        return dict(accepted=accepted, tokens=tokens, rows=rows, slots=slots)
    n, batch, most = st.tokens.shape[0], st.cu_rows.shape[0] - 1, st.most_rows
    b, local = _requests(st.cu_rows, n)
    first = st.cu_rows[b].long()
    parent = (local - 1 if st.parent is None else st.parent).clamp(min=0).long()
    token = st.tokens.long()
    p = st.target[first + parent, token].double()
    if st.draft is not None:
        take = st.uniforms.double() * st.draft[torch.arange(n, device="cuda"), token].double() < p
    else:
        # a retrieved draft is certain: accepted with the probability that the target gives it among what its rejected siblings left
        at = torch.full((batch, most), -1, dtype=torch.int64, device="cuda")
        at[b, local] = torch.where(local > 0, parent, -1)
        words = torch.full((batch, most), -1, dtype=torch.int64, device="cuda")
        words[b, local] = token
        earlier = torch.ones((most, most), device="cuda", dtype=torch.bool).tril(-1)[None] & (at[:, :, None] == at[:, None, :]) & (at[:, :, None] >= 0)
        again = (earlier & (words[:, :, None] == words[:, None, :])).any(2)                               # an earlier sibling carries the same token
        grid = torch.zeros((batch, most), dtype=torch.float64, device="cuda")
        grid[b, local] = p
        grid = torch.where(again, 0.0, grid)
        left = 1.0 - (earlier.double() @ grid[:, :, None])[:, :, 0]
        take = st.uniforms.double() * left[b, local] < grid[b, local]
    take = take & (local > 0)
    # a row's first accepted child is the one that is followed
    takes = torch.zeros((batch, most), dtype=torch.bool, device="cuda")
    takes[b, local] = take
    up = torch.full((batch, most), -1, dtype=torch.int64, device="cuda")
    up[b, local] = torch.where(local > 0, parent, -1)
    same = (up[:, :, None] == up[:, None, :]) & (up[:, :, None] >= 0)
    before = torch.ones((most, most), device="cuda", dtype=torch.bool).tril(-1)
    follows = takes & ~(same & before & takes[:, None, :]).any(2)
    follows[:, 0] = True
    paths = _paths(parent.int(), b, local, batch, most)
    on = (paths & ~follows[:, None, :]).sum(2) == 0                                                       # every row of the path is followed
    alive = torch.zeros((batch, most), dtype=torch.bool, device="cuda")
    alive[b, local] = True
    on = on & alive
    accepted = on.sum(1) - 1
    last = torch.where(on, torch.arange(most, device="cuda")[None], -1).amax(1)                            # rows of a path ascend
    # what the last accepted row's distribution leaves
    left = st.target[st.cu_rows[:-1].long() + last.clamp(min=0)].double().clamp(min=0)
    rejected = (up == last[:, None]) & (up >= 0)
    if st.draft is not None:
        row = st.cu_rows[:-1].long() + torch.where(rejected.any(1), rejected.int().argmax(1), 0)
        rest = torch.where(rejected.any(1)[:, None], (left - st.draft[row].double()).clamp(min=0), left)
    else:
        tall = torch.zeros((batch, most), dtype=torch.int64, device="cuda")
        tall[b, local] = token
        hit = torch.zeros_like(left).scatter_add_(1, tall, rejected.double())
        rest = torch.where(hit > 0, 0.0, left)
    rest = torch.where(rest.sum(1, keepdim=True) > 0, rest, left)
    total = rest.cumsum(1)
    draw = torch.searchsorted(total, st.uniforms[st.cu_rows[:-1].long()].double()[:, None] * total[:, -1:], right=True)[:, 0]
    final = torch.where(rest > 0, torch.arange(rest.shape[1], device="cuda")[None], -1).amax(1)            # the last token that has a share
    draw = torch.minimum(draw, final)
    # behind one another: the accepted rows, their tokens, and the sampled token at the end
    place = (on.cumsum(1) - 1)[b, local]
    keep = on[b, local]
    rows = torch.full((n + 1,), -1, dtype=torch.int64, device="cuda")
    rows[torch.where(keep, first + place, n)] = local
    tokens = torch.full((n + 1,), -1, dtype=torch.int64, device="cuda")
    tokens[torch.where(keep & (local > 0), first + place - 1, n)] = token
    tokens[st.cu_rows[:-1].long() + accepted] = draw
    moved = torch.where(keep & (place != local), st.slots[(first + place).clamp(max=n - 1)], -1)
    return dict(accepted=accepted.to(torch.int32), tokens=tokens[:n].to(torch.int32), rows=rows[:n].to(torch.int32), slots=moved.to(torch.int32))


# ------------------------------------------------------------------------------------------ from the definitions, in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    return {"slots": _exact_slots, "rope": _exact_rope, "attend": _exact_attend, "verify": _exact_verify}[case["kind"]](st)


def _exact_slots(st):
    page, table, free = st.case["page"], st.block_table.cpu().numpy().copy(), st.free_pages.cpu().numpy()
    cu, length, held, head = st.cu_rows.tolist(), st.kv_len.tolist(), st.n_held.tolist(), st.free_state.tolist()[0]
    parent = None if st.parent is None else st.parent.tolist()
    slots, positions, short, at = [], [], 0, head
    for b in range(len(length)):
        n = cu[b + 1] - cu[b]
        want = -(-(length[b] + n) // page) if n else 0
        need = max(0, want - held[b]) if want <= table.shape[1] else 0
        fits = want <= table.shape[1] and (need == 0 or at + need <= len(free))
        if fits:
            table[b, held[b]:held[b] + need] = free[at:at + need]
            held[b] += need
            head = max(head, at + need)
        at += need
        short += not fits
        depth = []
        for i in range(n):
            depth.append(i if parent is None else 0 if i == 0 else depth[parent[cu[b] + i]] + 1)
            t = length[b] + i
            slots.append(int(table[b, t // page]) * page + t % page if fits else -1)
            positions.append(length[b] + depth[i])
    whole = lambda v: torch.tensor(np.asarray(v, dtype=np.int32))  # noqa: E731
    return dict(slots=whole(slots), positions=whole(positions), held=whole(held), free=whole([head, short]), table=whole(table))


def _exact_rope(st):
    c = st.case
    angle = np.exp(1j * np.outer(st.positions.cpu().numpy().astype(np.float64), st.frequencies.cpu().numpy())) * st.factor

    def turned(x):
        x = x.double().cpu().numpy().copy()
        pairs = (slice(0, c["rot"], 2), slice(1, c["rot"], 2)) if c["interleaved"] else (slice(0, c["rot"] // 2), slice(c["rot"] // 2, c["rot"]))
        z = (x[..., pairs[0]] + 1j * x[..., pairs[1]]) * angle[:, None]
        x[..., pairs[0]], x[..., pairs[1]] = z.real, z.imag
        return x

    slots = st.slots.cpu().numpy()
    row = np.nonzero(slots >= 0)[0]
    out = dict(q=torch.from_numpy(turned(st.q)))
    for name, pages, rows in (("k_pages", st.k_pages, turned(st.k)), ("v_pages", st.v_pages, st.v.double().cpu().numpy())):
        held = pages.double().cpu().numpy().copy()
        held[slots[row] // c["page"], :, slots[row] % c["page"]] = rows[row]
        out[name] = torch.from_numpy(held)
    return out


def _exact_attend(st):
    c, cu, lengths = st.case, st.cu_rows.tolist(), st.kv_len.tolist()
    parent = None if st.parent is None else st.parent.tolist()
    out = torch.empty(st.q.shape, dtype=torch.float64, device="cuda")
    for b, length in enumerate(lengths):
        n = cu[b + 1] - cu[b]
        table = st.block_table[b, :-(-(length + n) // c["page"])].long()
        k, v = (p[table].double().permute(1, 0, 2, 3).reshape(c["hkv"], -1, c["hd"])[:, :length + n] for p in (st.k_pages, st.v_pages))
        allowed = torch.zeros((n, length + n), dtype=torch.bool)
        allowed[:, :length] = True
        for i in range(n):
            if parent is None:
                allowed[i, length:length + i + 1] = True
            else:
                if i:
                    allowed[i] = allowed[parent[cu[b] + i]]
                allowed[i, length + i] = True
        q = st.q[cu[b]:cu[b + 1]].double().reshape(n, c["hkv"], -1, c["hd"])
        s = torch.einsum("nhgd,htd->hgnt", q, k) * st.scale
        w = torch.softmax(s.masked_fill(~allowed.cuda(), -math.inf), -1)
        out[cu[b]:cu[b + 1]] = torch.einsum("hgnt,htd->nhgd", w, v).reshape(n, c["hq"], c["hd"])
    return out


def _exact_verify(st):
    cu, tokens, u = st.cu_rows.tolist(), st.tokens.tolist(), st.uniforms.double().tolist()
    parent, slots = None if st.parent is None else st.parent.tolist(), st.slots.tolist()
    n = len(tokens)
    accepted, out, rows, moved = [], [-1] * n, [-1] * n, [-1] * n
    for b in range(len(cu) - 1):
        first, count = cu[b], cu[b + 1] - cu[b]
        at, path = 0, [0]
        rest = st.target[first].double().cpu().numpy()
        left = 1.0
        for i in range(1, count):
            if (i - 1 if parent is None else parent[first + i]) != at:
                continue
            x = tokens[first + i]
            if st.draft is not None:
                q = st.draft[first + i].double().cpu().numpy()
                taken = u[first + i] * q[x] < rest[x]
            else:
                taken = u[first + i] * left < rest[x]
            if taken:
                at, left = i, 1.0
                path.append(i)
                rest = st.target[first + i].double().cpu().numpy()
            elif st.draft is not None:
                rest = np.maximum(rest - q, 0.0)
                break
            else:
                left -= rest[x]
                rest[x] = 0.0
        if not rest.sum() > 0:
            rest = st.target[first + at].double().cpu().numpy()
        total = np.cumsum(rest)
        draw = min(int(np.searchsorted(total, u[first] * total[-1], side="right")), int(np.nonzero(rest > 0)[0][-1]))
        accepted.append(len(path) - 1)
        for k, i in enumerate(path):
            rows[first + k] = i
            if k:
                out[first + k - 1] = tokens[first + i]
            if k != i:
                moved[first + i] = slots[first + k]
        out[first + len(path) - 1] = draw
    whole = lambda v: torch.tensor(np.asarray(v, dtype=np.int32))  # noqa: E731
    return dict(accepted=whole(accepted), tokens=whole(out), rows=whole(rows), slots=whole(moved))


# ------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    if case["kind"] == "rope":
        heads = case["hq"] + 2 * case["hkv"]
        return dict(bytes=case["rows"] * (4.0 * heads * case["hd"] + 8.0), flops=case["rows"] * 3.0 * (case["hq"] + case["hkv"]) * case["rot"])
    if case["kind"] == "verify":
        n = case["batch"] * case["rows"]
        vectors = 2 if case["drafts"] else 1   # the distribution behind the accepted drafts, and the rejected draft's
        return dict(bytes=case["batch"] * (4.0 * case["vocab"] * vectors) + n * 32.0, flops=case["batch"] * 2.0 * case["vocab"] * vectors)
    rows, lengths = _lengths(case)
    if case["kind"] == "slots":
        pages = sum(-(-(a + b) // case["page"]) for a, b in zip(rows, lengths))
        return dict(bytes=8.0 * pages + 12.0 * sum(rows) + 16.0 * case["batch"], flops=4.0 * sum(rows) + 2.0 * pages)
    keys = sum(a + b for a, b in zip(rows, lengths))
    return dict(bytes=4.0 * keys * case["hkv"] * case["hd"] + 4.0 * sum(rows) * case["hq"] * case["hd"],
                flops=sum(4.0 * a * (a + b) for a, b in zip(rows, lengths)) * case["hq"] * case["hd"])
