"""draft_verify's draw right beside the borders between tokens of a full vocabulary, against exact sums.

A row's running sums are formed in whole numbers (every fp32 is a multiple of 2^-149).  For each border the two fp32
numbers next to (running sum / sum) are draws that fall just before and just behind it, 2^-25 of the sum away or less;
the closest ones are taken.

How close: with one CTA a row, a thread adds up V / 256 weights, two at a time, in two chains.  The rounding error of
each pair (at most 2^-24 of it) and the lower part of each difference (2^-24 of it) are exact and summed in fp32: at
most V / 512 additions a chain, each rounded by 2^-24 of a sum that is at most 2^-23 of the weights.  That is V / 512 *
2^-47 < 2^-39 of the sum for V = 128256, and fp64 adds V / 1024 * 2^-52, the threads' and the draw's own few roundings of
2^-53.  Draws closer than 2^-38 of the sum are left out."""
from itertools import accumulate

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

V, CLOSEST = 128256, 38


def whole(t):
    """fp32 or bf16 numbers as whole multiples of 2^-149."""
    mantissa, exponent = np.frexp(t.double().numpy())
    return [int(m) << int(e) if e >= 0 else int(m) >> -int(e) for m, e in zip(mantissa * 2.0 ** 53, exponent + 149 - 53)]


def first_above(upto, goal):
    """The first place whose running sum exceeds the goal (fractions with one denominator)."""
    lo, hi = 0, len(upto) - 1
    while lo < hi:
        mid = (lo + hi) // 2
        lo, hi = (lo, mid) if upto[mid] > goal else (mid + 1, hi)
    return lo


def draws(weights, n):
    """(n draws beside borders, their tokens) for whole weights."""
    upto = list(accumulate(weights))
    total = upto[-1]
    scale = 1 << 60                                                  # every fp32 in [2^-30, 1) is a multiple of 2^-60
    near = np.array([c / total for c in upto[:-1]], dtype=np.float64).astype(np.float32)
    found = []
    for u32 in (near, np.nextafter(near, np.float32(0)), np.nextafter(near, np.float32(1))):
        for c, u in zip(upto, u32.tolist()):
            if 2.0 ** -30 < u < 1.0:
                away = abs(int(u * scale) * total - c * scale)
                if away << CLOSEST >= total * scale:
                    found.append((away, u))
    found = sorted(set(found))[:n]
    assert len(found) == n and found[-1][0] << 30 < total * scale    # within 2^-30 of the sum, far less than a token
    us = [u for _, u in found]
    return us, [first_above([c * scale for c in upto], int(u * scale) * total) for u in us]


def rows(dtype, difference):
    g = torch.Generator().manual_seed(7)
    logits = 1.5 * torch.randn(V, generator=g)
    logits[V // 3] += 9.0                                            # a heavy token among them
    p = torch.softmax(logits, -1).to(dtype)
    q = torch.softmax(logits + 0.5 * torch.randn(V, generator=g), -1).to(dtype) if difference else None
    return p, q


@pytest.mark.parametrize("B", [600, 40, 4])                          # one CTA a row, clusters of 8 and of 16
@pytest.mark.parametrize("difference", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_draws_beside_the_borders(dtype, difference, B):
    from paper_2501_08090_b200 import binding as b
    p, q = rows(dtype, difference)
    weights = whole(p)
    if difference:
        weights = [max(x - y, 0) for x, y in zip(weights, whole(q))]
    us, want = draws(weights, B)

    if B == 600:
        # sums in 32 bits draw other tokens for these numbers; so do fp64 sums of fp32 pairs without their rounding errors
        w32, goal = np.array([w / (1 << 149) for w in weights]).astype(np.float32), np.array(us)
        sums = np.cumsum(w32)
        assert (np.searchsorted(sums, goal.astype(np.float32) * sums[-1], side="right") != want).mean() > 0.4
        if dtype == torch.float32:
            pairs = np.cumsum((w32[0::2] + w32[1::2]).astype(np.float64))
            assert (np.searchsorted(pairs, goal * pairs[-1], side="right") != np.array(want) // 2).mean() > 0.05

    target = p.cuda().expand(B, 1, V).contiguous()
    us_d, accepted = torch.tensor(us, dtype=torch.float32, device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda")
    if not difference:
        tokens = torch.empty(B, 1, dtype=torch.int32, device="cuda")
        b.draft_verify(torch.empty(B, 0, dtype=torch.int32, device="cuda"), target, None, torch.empty(B, 0, device="cuda"), us_d, tokens, accepted)
    else:
        x = int((q.float() - p.float()).argmax())                    # refused: u q >= p
        tokens = torch.empty(B, 2, dtype=torch.int32, device="cuda")
        b.draft_verify(torch.full((B, 1), x, dtype=torch.int32, device="cuda"), torch.cat([target, target], 1), q.cuda().expand(B, 1, V).contiguous(),
                       torch.full((B, 1), 1.0 - 2.0 ** -24, device="cuda"), us_d, tokens, accepted)
    assert not accepted.any()
    assert tokens[:, 0].tolist() == want
