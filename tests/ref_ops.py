"""Plain 64-bit implementations of the operators around a long decode step, for the tests: loops over
requests and heads in numpy, written from the definitions in include/chiron_kv.h."""
from __future__ import annotations

import math

import numpy as np

PAGE = 16


def new_tokens(lens, n_tokens, new_start=None):
    """(token, request, position) of every new token that belongs to a request."""
    B = len(lens)
    starts = [r * (n_tokens // B) for r in range(B + 1)] if new_start is None else [int(x) for x in new_start]
    return [(i, r, int(lens[r]) - (starts[r + 1] - starts[r]) + i - starts[r])
            for r in range(B) for i in range(starts[r], starts[r + 1])]


def rotate(x, pos, inv_freq, interleaved, scale=1.0):
    """x [heads][d] float64 at one position: (rotated, |x| + |y| of each element's pair)."""
    half = len(inv_freq)
    out, size = x.copy(), np.abs(x)
    for j in range(half):
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
        turn = float(pos) * float(inv_freq[j])
        c, s = scale * math.cos(turn), scale * math.sin(turn)
        out[:, a] = x[:, a] * c - x[:, b] * s
        out[:, b] = x[:, b] * c + x[:, a] * s
        size[:, a] = size[:, b] = np.abs(x[:, a]) + np.abs(x[:, b])
    return out, size


def key_bounds(keys):
    """(lo, hi, step) of keys [tokens][d]."""
    if not np.all(np.isfinite(keys)):
        return np.full(keys.shape[1], -127), np.full(keys.shape[1], 127), 2.0 ** 121
    m = max(float(np.abs(keys).max()), 2.0 ** -100)
    step = 2.0 ** (math.frexp(m)[1] - 1 - 6)
    if math.ceil(float(np.abs(keys).max()) / step) > 127:
        step *= 2
    return np.floor(keys.min(0) / step).astype(int), np.ceil(keys.max(0) / step).astype(int), step


def index_of(pool, tables, lens, last_tokens=0):
    """{(page, head): (lo, hi, step)} of the pages that an update covers; pool [pages][Hkv][2][16][d] float64."""
    found = {}
    for r, L in enumerate(int(x) for x in lens):
        n = -(-L // PAGE)
        first = max(0, L - last_tokens) // PAGE if last_tokens else 0
        for i in range(first, n):
            for h in range(pool.shape[1]):
                page = int(tables[r][i])
                found[page, h] = key_bounds(pool[page, h, 0, :min(PAGE, L - i * PAGE)])
    return found


def query_steps(q):
    """(q in whole steps, step) of one query [d]; what is not finite counts as 0."""
    q = np.where(np.isfinite(q), q, 0.0)
    step = 2.0 ** (math.frexp(max(float(np.abs(q).max()), 2.0 ** -100))[1] - 1 - 6)
    return np.clip(np.rint(q / step), -127, 127).astype(int), step


def select(index, tables, L, q, h, budget, sink, recent):
    """Page ids that a (request, kv head) attends to; q [group][d]."""
    n = -(-int(L) // PAGE)
    row = [int(x) for x in tables[:n]]
    if n <= budget:
        return row
    quants = [query_steps(x) for x in q]

    def score(page):
        lo, hi, step = index[page, h]
        return max(float(np.maximum(q8 * lo, q8 * hi).sum()) * qs for q8, qs in quants) * step

    middle = sorted(range(sink, n - recent), key=lambda i: (-score(row[i]), i))[:budget - sink - recent]
    return [row[i] for i in sorted(list(range(sink)) + middle + list(range(n - recent, n)))]


def attend(pool, pages, tokens, q, h):
    """softmax(q k / sqrt(d)) v over the first `tokens` tokens of the listed pages; q [group][d]."""
    k = pool[pages, h, 0].reshape(-1, pool.shape[-1])[:tokens]
    v = pool[pages, h, 1].reshape(-1, pool.shape[-1])[:tokens]
    s = q @ k.T / math.sqrt(q.shape[1])
    w = np.exp(s - s.max(1, keepdims=True))
    return (w @ v) / w.sum(1, keepdims=True)


def verify(drafts, p, q, u_accept, u_sample):
    """(accepted count, tokens) of one request: p [n + 1][V], q [n][V] or None, in float64."""
    tokens = []
    V = p.shape[1]
    for j, x in enumerate(int(t) for t in drafts):
        inside = 0 <= x < V
        px, qx = (p[j, x], 1.0 if q is None else q[j, x]) if inside else (0.0, 0.0)
        if inside and float(u_accept[j]) * qx < px:
            tokens.append(x)
            continue
        w = p[j].copy()
        if q is not None:
            w = p[j] - q[j]
        elif inside:
            w[x] = 0.0
        w = np.where(w > 0, w, 0.0)
        if w.sum() == 0:
            w = np.where(p[j] > 0, p[j], 0.0)
        break
    else:
        j = len(drafts)
        w = np.where(p[j] > 0, p[j], 0.0)
    upto = np.cumsum(w)
    if not upto[-1] > 0:
        return len(tokens), tokens + [-1]
    above = np.nonzero(upto > float(u_sample) * upto[-1])[0]
    return len(tokens), tokens + [int(above[0]) if above.size else int(np.nonzero(w)[0][-1])]
