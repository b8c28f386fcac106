"""The operators on a cache kept in pages, from their definitions in 64 bits (numpy), for the tests."""
from __future__ import annotations

import numpy as np


def spans(cu_rows):
    return [(int(a), int(b)) for a, b in zip(cu_rows[:-1], cu_rows[1:])]


def up(parent, first, i):
    """The row that row i of a sequence continues."""
    if parent is None:
        return i - 1
    p = int(parent[first + i])
    return p if 0 <= p < i else 0


def path(parent, first, i):
    rows = [i]
    while rows[-1] > 0:
        rows.append(up(parent, first, rows[-1]))
    return rows[::-1]


def slots(kv_len, cu_rows, table, held, free, head, page, n_rows, parent=None):
    table, held = table.copy(), held.copy()
    out, pos = np.full(n_rows, -1, np.int64), np.zeros(n_rows, np.int64)
    taken, last, refused = head, head, 0
    for b, (r0, r1) in enumerate(spans(cu_rows)):
        want = -(-(int(kv_len[b]) + r1 - r0) // page) if r1 > r0 else 0
        wide = want <= table.shape[1]
        need = max(0, want - int(held[b])) if wide else 0
        ok = wide and (need == 0 or taken + need <= len(free))
        if ok and need:
            table[b, held[b]:held[b] + need] = free[taken:taken + need]
            held[b] += need
            last = taken + need
        taken += need
        refused += not ok
        for i in range(r1 - r0):
            pos[r0 + i] = kv_len[b] + len(path(parent, r0, i)) - 1
            t = int(kv_len[b]) + i
            if ok and table[b, t // page] >= 0:
                out[r0 + i] = int(table[b, t // page]) * page + t % page
    return out, pos, table, held, (last, refused)


def rope(x, positions, frequencies, factor, interleaved):
    """x [rows][heads][dim] in 64 bits; the rotated one and the sum of magnitudes that entered each element."""
    half = len(frequencies)
    angle = positions.astype(np.float64)[:, None] * frequencies[None]
    c, s = np.cos(angle)[:, None] * factor, np.sin(angle)[:, None] * factor
    out, size = x.copy(), np.zeros_like(x)
    lo, hi = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    a, b = x[..., lo], x[..., hi]
    out[..., lo], out[..., hi] = a * c - b * s, a * s + b * c
    size[..., lo] = size[..., hi] = (np.abs(a) + np.abs(b)) * factor
    return out, size


def attention(q, k, v, allowed, scale):
    """One sequence: q [rows][heads][dim], k, v [KV heads][tokens][dim], allowed [rows][tokens].  (out, sum of weights times
    |values|, largest sum of |q k| scale among the tokens a row sees); keys and values that a row does not see do not enter."""
    n, hq, dim = q.shape
    hkv = k.shape[0]
    out, mass, size = np.zeros((n, hq, dim)), np.zeros((n, hq, dim)), np.zeros((n, hq))
    for i in range(n):
        see = np.nonzero(allowed[i])[0]
        for h in range(hq):
            kk, vv = k[h // (hq // hkv), see], v[h // (hq // hkv), see]
            s = kk @ q[i, h] * scale
            w = np.exp(s - s.max())
            w /= w.sum()
            out[i, h] = w @ vv
            mass[i, h] = w @ np.abs(vv)
            size[i, h] = (np.abs(kk) @ np.abs(q[i, h])).max() * scale
    return out, mass, size


def verify(target, tokens, cu_rows, u, draft=None, parent=None, slot=None, most=64):
    n, vocab = target.shape
    accepted, words, rows, moved = [], np.full(n, -1), np.full(n, -1), np.full(n, -1)
    share = lambda r: np.where(target[r] > 0, target[r], 0.0).astype(np.float64)  # noqa: E731  (NaN has none)
    for r0, r1 in spans(cu_rows):
        if r1 == r0:
            accepted.append(-1)
            continue
        way, rest, left = [0], share(r0), 1.0
        for i in range(1, min(r1 - r0, most)):
            if up(parent, r0, i) != way[-1]:
                continue
            x = int(tokens[r0 + i])
            inside = 0 <= x < vocab
            p = rest[x] if inside else 0.0
            if draft is not None:
                ok = float(u[r0 + i]) * (float(draft[r0 + i, x]) if inside else 1.0) < p
            else:
                ok = float(u[r0 + i]) * left < p
            if ok:
                way.append(i)
                rest, left = share(r0 + i), 1.0
            elif draft is not None:
                d = rest - draft[r0 + i].astype(np.float64)
                rest = np.where((rest > 0) & (d > 0), d, 0.0)
                break
            else:
                left -= p
                if inside:
                    rest[x] = 0.0
        if not rest.sum() > 0:
            rest = share(r0 + way[-1])
        if rest.sum() > 0:
            c = np.cumsum(rest)
            drawn = min(int(np.searchsorted(c, float(u[r0]) * c[-1], side="right")), int(np.nonzero(rest > 0)[0][-1]))
        else:
            drawn = -1
        a = len(way) - 1
        accepted.append(a)
        for k, i in enumerate(way):
            rows[r0 + k] = i
            if k:
                words[r0 + k - 1] = tokens[r0 + i]
            if slot is not None and k != i:
                moved[r0 + i] = slot[r0 + k]
        words[r0 + a] = drawn
    return np.array(accepted), words, rows, moved
