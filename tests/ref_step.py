"""Plain 64-bit implementations of the operators of a decode step whose state stays on the GPU, for the tests:
loops over requests and heads in numpy, written from the definitions in include/chiron_kv.h."""
from __future__ import annotations

import math

import numpy as np

PAGE = 16


def pages(n):
    return -(-n // PAGE)


# ---- the 8-bit cache

def need_step(rows):
    """Step that rows (any shape) need; NaN if one is not finite."""
    if not np.all(np.isfinite(rows)):
        return math.nan
    m = max(float(np.abs(rows).max()), 2.0 ** -100)
    return 2.0 ** (math.frexp(m)[1] - 1 - 6)


def append8(records, steps, page, a, rows):
    """Quantise rows [n][Hkv][2][d] (float64) into slots a .. a+n-1 of a page of records [pages][Hkv][2][16][d]."""
    for h in range(rows.shape[1]):
        for kv in range(2):
            x = rows[:, h, kv]
            need, old = need_step(x), float(steps[page, h, kv])
            step = need if a == 0 else math.nan if math.isnan(need) or math.isnan(old) else max(old, need)
            if a > 0 and step > old:
                records[page, h, kv, :a] = np.rint(records[page, h, kv, :a] * (old / step))
            records[page, h, kv, a:a + len(x)] = 0 if math.isnan(step) else np.clip(np.rint(x / step), -127, 127)
            steps[page, h, kv] = step


def append8_tokens(records, steps, table, length, rows):
    """Append rows [n][Hkv][2][d] of one request whose length afterwards is `length`, as one call does."""
    pos, at = length - len(rows), 0
    while at < len(rows):
        a = pos % PAGE
        n = min(PAGE - a, len(rows) - at)
        append8(records, steps, int(table[pos // PAGE]), a, rows[at:at + n])
        pos, at = pos + n, at + n


# ---- attention with a window and sinks

def attend(q, k, v, length, window, sink, steps=None):
    """q [N][G][d], k, v [tokens][d] float64: (out [N][G][d], weighted mean of |v| [N][G][d], largest scaled sum of |q k| [N][G]);
    with the steps [tokens] of an 8-bit cache's v also what weights below fp16's normal numbers may be off by [N][G]."""
    N, G, d = q.shape
    out, size, mass, floor = np.zeros(q.shape), np.zeros(q.shape), np.zeros((N, G)), np.zeros((N, G))
    for i in range(N):
        p = length - N + i
        t = np.arange(p + 1)
        t = t[(t > p - window) | (t < sink)] if window else t
        s = q[i] @ k[t].T / math.sqrt(d)
        with np.errstate(invalid="ignore"):
            w = np.exp(s - s.max(1, keepdims=True))
            w /= w.sum(1, keepdims=True)
        out[i], size[i] = w @ v[t], w @ np.abs(v[t])
        mass[i] = (np.abs(q[i]) @ np.abs(k[t]).T / math.sqrt(d)).max(1)
        if steps is not None:
            # queries are rounded to 2^-21 of their largest element: a quarter of 2^-19 on top of what scores are summed with
            mass[i] += (np.abs(q[i]).max(1, keepdims=True) * np.abs(k[t]).sum(1)).max(1) / math.sqrt(d) / 4
            # a weight is held as a fraction of a reference no larger than the largest weight * step, in fp16: fractions below
            # 2^-14 are off by 2^-25 at most, times a record of at most 127
            floor[i] = 2.0 ** -25 * 127 * len(t) * (w * steps[t]).max(1)
    return (out, size, mass) if steps is None else (out, size, mass, floor)


def attend_tolerance(out, size, mass, weight_bits, floor=None):
    """The output's rounding to bf16; the weights' to fp16 or bf16 (half a step of `weight_bits` bits below 1) with 2^-9 of
    that again for sums and exponentials; scores summed in fp32 over at most 128 products (2^-19 of the sum of
    magnitudes: 24 bits, 8 additions and as many roundings again), which moves every weight by twice that at most."""
    error = 2.0 ** -weight_bits * (1 + 2.0 ** -9) + 2 * mass[..., None] * 2.0 ** -19 + 2.0 ** -18
    error = error * size + (0 if floor is None else floor[..., None])
    return 2.0 ** -8 * (np.abs(out) + error) + error + 1e-37             # at last the flush of numbers below 2^-126


# ---- pages

def release(tables, lens, keep, free, count, num_pages):
    """(lens out, count out, flagged); writes free."""
    out, going, bad = list(lens), [], False
    for r, (L, x) in enumerate(zip(lens, keep)):
        if not (0 <= x <= L <= len(tables[r]) * PAGE):
            bad = True
            continue
        out[r] = x
        going += [int(p) for p in tables[r][pages(x):pages(L)]]
    for k, p in enumerate(going):
        place = count + len(going) - 1 - k
        good = 0 <= p < num_pages
        bad |= not good
        if place < num_pages:
            free[place] = p if good else -1
        else:
            bad = True
    return out, min(count + len(going), num_pages), bad


def assign(tables, lens, new, free, count, num_pages):
    """(lens out, count out, step lens, new_start, slots, flagged); writes tables."""
    out, step, start, slots, bad = list(lens), [], [0], [], False
    upto = taken = 0
    for r, (L, n) in enumerate(zip(lens, new)):
        fits = L >= 0 and n >= 0 and L + n <= len(tables[r]) * PAGE
        need = pages(L + n) - pages(L) if fits else 0
        upto += need
        served = fits and (need == 0 or upto <= count)
        bad |= not fits
        if served:
            for i in range(need):
                p = int(free[count - 1 - taken])
                taken += 1
                bad |= not 0 <= p < num_pages
                tables[r][pages(L) + i] = p if 0 <= p < num_pages else -1
            out[r] = L + n
        step.append(out[r] if served else 0)
        for pos in range(L, L + n) if n > 0 else ():
            p = int(tables[r][pos // PAGE]) if served else -1
            bad |= served and not 0 <= p < num_pages
            slots.append(p * PAGE + pos % PAGE if served and 0 <= p < num_pages else -1)
        start.append(start[-1] + max(n, 0))
    return out, count - taken, step, start, slots, bad


# ---- logits

def logits(x, params=None, prompt=(), said=(), bias=(), mask=None):
    """(processed, probabilities) of one row x [V] float64; bias: (id, value) pairs; mask: truth values."""
    V = len(x)
    rep, pres, freq, temperature = (1.0, 0.0, 0.0, 1.0) if params is None else (float(p) for p in params)
    x = x.copy()
    count, seen = np.zeros(V), np.zeros(V, bool)
    for t in said:
        if 0 <= t < V:
            count[t] += 1
            seen[t] = True
    for t in prompt:
        if 0 <= t < V:
            seen[t] = True
    x[seen] = np.where(x[seen] > 0, x[seen] / rep, x[seen] * rep)
    x[seen] -= freq * count[seen]
    x[count > 0] -= pres
    last = {int(t): float(b) for t, b in bias if 0 <= t < V}
    for t, b in last.items():
        x[t] += b
    if mask is not None:
        x[~mask] = -np.inf
    allowed = x if mask is None else x[mask]
    p = np.zeros(V)
    if np.isnan(allowed).any() or (allowed == np.inf).any():
        return x, np.full(V, np.nan)
    top = x.max()
    if top > -np.inf:
        if temperature > 0:
            p = np.exp((x - top) / temperature)
            p /= p.sum()
        else:
            p[int(np.argmax(x))] = 1.0
    return x, p
