"""Plain 64-bit forms of what a serving loop does between two verify steps: a token from a row of logits, and the paged cache's pages.

Written from the definitions, row by row and entry by entry, on numpy and lists; shares no code with the GPU path.
"""
import math

import numpy as np


# ------------------------------------------------------------------------------------------ sampling
def guided_logits(cond, uncond, scale):
    """fp32: subtract, then a multiply-add rounded once (the product of two fp32 numbers is exact in fp64, the sum rounds at 2^-53
    first, which next to never matters); -inf in either gives -inf."""
    c, u = np.asarray(cond, np.float32), np.asarray(uncond, np.float32)
    with np.errstate(invalid="ignore", over="ignore"):
        l = (u.astype(np.float64) + np.float64(np.float32(scale)) * (c - u).astype(np.float64)).astype(np.float32)
    bad = np.isnan(c) | np.isnan(u) | np.isinf(c) | np.isinf(u)
    return np.where(bad, -np.inf, l)


def sample_row(l, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """l float64 [n] (NaN and +inf count as -inf) -> (id, p [n], margin): margin is how near, as a share of the mass, a decision was to
    going the other way: the draw to a border of the running sum, top-p's target to the mass that reached it or just did not."""
    l = np.array(l, dtype=np.float64)
    l[np.isnan(l) | (l == np.inf)] = -np.inf
    n = len(l)
    if not np.isfinite(l).any():
        return -1, np.zeros(n), 1.0
    top = l.max()
    if temperature == 0:
        p = np.zeros(n)
        p[int(np.flatnonzero(l == top)[0])] = 1.0
        return int(np.flatnonzero(l == top)[0]), p, 1.0
    kept = np.isfinite(l)
    margin = 1.0
    if top_k > 0 and top_k < kept.sum():
        kept &= l >= np.sort(l[kept])[::-1][top_k - 1]
    with np.errstate(invalid="ignore", over="ignore"):
        z = (l - top) / np.float64(temperature)
    w = np.where(kept, np.exp(z), 0.0)
    if top_p < 1:
        values = np.unique(l[kept])[::-1]
        mass = np.array([math.fsum(w[l == v]) for v in values]) if len(values) < 64 else _mass_by_value(l, w, values)
        run = np.cumsum(mass)
        target = top_p * run[-1]
        at = int(np.flatnonzero(run >= target)[0]) if target > 0 else 0
        margin = min(margin, np.abs(run - target).min() / run[-1]) if target > 0 and len(values) > 1 else margin
        kept &= l >= values[at]
    if min_p > 0:
        kept &= (z >= math.log(min_p)) | (l == top)
    w = np.where(kept, w, 0.0)
    run = np.cumsum(w)
    u = min(max(float(u), 0.0), 1.0 - 2.0 ** -24) if not math.isnan(u) else 0.0
    t = u * run[-1]
    at = min(int(np.searchsorted(run, t, side="right")), n - 1)
    margin = min(margin, np.abs(run[kept] - t).min() / run[-1])
    return at, w / run[-1], margin


def _mass_by_value(l, w, values):
    order = np.argsort(-l, kind="stable")
    first = np.searchsorted(-l[order], -values, side="left")
    run = np.concatenate([[0.0], np.cumsum(w[order])])
    end = np.searchsorted(-l[order], -values, side="right")
    return run[end] - run[first]


def weight_error(n, largest):
    """How far the kernels' running sums over n ids may be off, as a share of a mass of which the id with the largest weight has the share
    `largest`: the remainder of the exponential's polynomial, and half a multiple of 2^-44 of the largest weight for each id.  (fp64
    roundings here and there add 2^-52 an id.)"""
    return (math.log(2) / 256) ** 4 / 24 + n * 2.0 ** -45 * largest + n * 2.0 ** -52


# ------------------------------------------------------------------------------------------ pages
def pages(keys, page):
    return -(-keys // page)


def resize(table, kv, new, refs, page):
    """-> (table, lengths, refs, copies, some stayed): lists; `table` holds None where an entry is not written."""
    S, W = len(table), len(table[0]) if len(table) else 0
    out = [[None] * W for _ in range(S)]
    refs, lens, copies = list(refs), list(kv), [(-1, -1, 0)] * S
    new = [b if 0 <= b <= W * page else a for a, b in zip(kv, new)]  # (out of range: the stream stays as it is)
    ok = [0 <= a <= W * page for a in kv]
    for s in range(S):
        if ok[s] and new[s] < kv[s]:
            for j in range(pages(new[s], page), pages(kv[s], page)):
                refs[table[s][j]] -= 1
    after = list(refs)
    free = [i for i, c in enumerate(refs) if c == 0]
    taken, stopped = 0, False
    for s in range(S):
        if not ok[s]:
            continue
        have, want = pages(kv[s], page), pages(new[s], page)
        shared = new[s] > kv[s] and kv[s] % page != 0 and after[table[s][have - 1]] > 1
        need = want - have + shared if new[s] > kv[s] else 0
        if need and (stopped or taken + need > len(free)):
            stopped = True
            out[s][:have] = table[s][:have]
            continue
        lens[s] = new[s]
        out[s][:min(have, want)] = table[s][:min(have, want)]
        mine = free[taken:taken + need]
        taken += need
        for p in mine:
            refs[p] = 1
        if shared:
            copies[s] = (table[s][have - 1], mine[0], kv[s] % page)
            refs[table[s][have - 1]] -= 1
            out[s][have - 1] = mine.pop(0)
        for j, p in enumerate(mine):
            out[s][have + j] = p
    return out, lens, refs, copies, stopped


def fork(table, kv, parent, refs, page, length=None):
    W = len(table[0]) if len(table) else 0
    refs, out, lens = list(refs), [], []
    for s, n in enumerate(kv):
        for j in range(pages(n, page)):
            refs[table[s][j]] -= 1
    for t, p in enumerate(parent):
        keys = 0 if p < 0 else kv[p] if length is None else max(0, min(kv[p], length[t]))
        entries = [table[p][j] for j in range(pages(keys, page))]
        for e in entries:
            refs[e] += 1
        out.append(entries + [None] * (W - len(entries)))
        lens.append(keys)
    return out, lens, refs


def compact(table, kv, refs, page, max_moves, first=0):
    """-> (table, refs, copies, top)"""
    n = len(refs)
    free = [i for i in range(first, n) if refs[i] == 0]
    used = [i for i in range(n - 1, first - 1, -1) if refs[i] != 0]
    moves = [(a, b) for a, b in list(zip(used, free))[:max_moves] if b < a]
    new = dict(moves)
    refs = list(refs)
    for a, b in moves:
        refs[b], refs[a] = refs[a], 0
    W = len(table[0]) if len(table) else 0
    out = [[new.get(table[s][j], table[s][j]) if j < pages(k, page) else None for j in range(W)] for s, k in enumerate(kv)]
    copies = [(a, b, page) for a, b in moves] + [(-1, -1, 0)] * (max_moves - len(moves))
    top = max([i + 1 for i in range(first, n) if refs[i] != 0] + [first])
    return out, refs, copies, top


def keep(row_begin, kv, path, accept_len, first):
    """-> (lengths, [(stream, cache row from, cache row to)] in the order they may be done)"""
    lens, moves = [], []
    for s, n_keys in enumerate(kv):
        n = row_begin[s + 1] - row_begin[s]
        b = s % len(accept_len)
        if n == 0:
            lens.append(n_keys)
            continue
        base = n_keys - n
        lens.append(base + min(n, first + accept_len[b]))
        if path is not None:
            moves += [(s, base + path[b][i], base + first + i) for i in range(accept_len[b])]
    return lens, moves
