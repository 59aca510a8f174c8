"""Attention over an 8-bit cache whose pages' V steps lie far apart: every token keeps its share of the softmax's sum,
however small its block's step is beside the others'.  In one tile, in tiles of different warps, CTAs and launches."""
import numpy as np
import pytest
import torch

import ref_step as ref
from test_gpu_cache8 import Cache, check_attention, queries, tables_for, to_dev

pytestmark = pytest.mark.gpu

# (context, pages of a table, launches): the kernel of a cluster per pair (1, 2 and 16 CTAs), then even spans and their fold
SHAPES = [(64, 4, 1), (400, 25, 1), (4000, 250, 1), (2000, 1700, 2), (26000, 1700, 2)]


def place(c, exps, lens, head=0):
    """V's steps of the live pages in turn, those of a pattern that has no period in tiles or warps."""
    for r, L in enumerate(lens):
        for i in range(ref.pages(L)):
            c.steps[c.layer, c.bt[r, i], head, 1] = 2.0 ** exps[(i + i // 7) % len(exps)]


def upload(c):
    c.kp.pool_view()[1].copy_(torch.from_numpy(c.steps).float())


def attend(c, lens, q, launches, **options):
    before = c.kp.launch_count()
    outs = []
    for _ in range(2):
        out = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
        c.kp.kv8_attention(c.layer, c.btd, c.lens(lens), to_dev(q), out, **options)
        outs.append(out)
    assert c.kp.launch_count() - before == 2 * launches and torch.equal(outs[0], outs[1])
    c.check()
    return outs[0]


@pytest.mark.parametrize("length,width,launches", SHAPES)
@pytest.mark.parametrize("exps", [(-106, 20), (20, -106), (-106, -6, 100), (121, -106, 0, -60), (-106, -106, -106, -106, -106, -106, 40)])
def test_steps_side_by_side(length, width, launches, exps):
    """Tiles of the smallest step and of a large one, next to one another and mixed in a tile; queries of ordinary size."""
    bt, n = tables_for([length], width, 1)
    c = Cache((4, 1, 64), bt, n, seed=2)
    c.steps[0, :, :, 0] = 2.0 ** -7
    if max(exps) > 119:                                      # values must stay below 2^128: records of 64 at most
        c.rec[0] = np.trunc(c.rec[0] / 2)
        c.kp.pool_view()[0].copy_(torch.from_numpy(c.rec).to(torch.int8))
    place(c, exps, [length])
    upload(c)
    live = {float(np.log2(c.steps[0, p, 0, 1])) for p in bt[0, :ref.pages(length)]}
    assert live == {float(e) for e in exps[:ref.pages(length)]}
    q = queries(1, 1, 4, 64, 3)
    check_attention(c, [length], q, attend(c, [length], q, launches))
    c.kp.close()


@pytest.mark.parametrize("length,width,launches", SHAPES)
@pytest.mark.parametrize("top", [2.0 ** 20, 2.0 ** 27, 2.0 ** 100])
def test_pages_of_zeros_beside_pages_of_large_values(length, width, launches, top):
    """Equal scores (queries of zeros): the mean of the values, half of whose pages are zeros, written by kv8_append."""
    bt, n = tables_for([length], width, 4)
    c = Cache((8, 2, 64), bt, n, seed=5)
    rows = np.zeros((length, 2, 2, 64))
    t = np.arange(length)
    rows[:, 0, 1] = np.where((t // 16 % 2 == 0)[:, None], top, 0)            # every tile has a page of either
    rows[:, 1, 1] = np.where((t // 32 % 2 == 1)[:, None], -top, 0)           # every other tile
    c.kp.kv8_append(0, c.btd, c.lens([length]), to_dev(rows[:, :, 0]), to_dev(rows[:, :, 1]))
    c.append_ref(0, length, rows)
    assert {-106.0, np.log2(top) - 6} == {float(x) for x in np.log2(c.steps[0, bt[0, :ref.pages(length)], 0, 1])}
    q = np.zeros((1, 1, 8, 64))
    out = attend(c, [length], q, launches)
    check_attention(c, [length], q, out)
    mean = rows[:, :, 1].mean(0)
    assert np.all(np.abs(out[0, 0].double().cpu().numpy().reshape(2, 4, 64) - mean[:, None]) <= 2.0 ** -8 * np.abs(mean[:, None]) + 2.0 ** -16 * top)
    c.kp.close()


@pytest.mark.parametrize("length,width,launches", SHAPES)
def test_scores_that_rise_and_fall_against_the_steps(length, width, launches):
    """The largest score beside the smallest step, and the other way round: the references of sum and product part."""
    for sign in (1, -1):
        bt, n = tables_for([length], width, 6)
        c = Cache((4, 1, 64), bt, n, seed=7)
        c.steps[0, :, :, 0] = 2.0 ** -7
        exps = [-60, -20, 0, 25]
        place(c, exps, [length])
        for i in range(ref.pages(length)):                   # keys along one direction, larger from page to page of a group
            p = bt[0, i]
            c.rec[0, p, 0, 0, :, 0] = np.clip(sign * -1.4 * (np.log2(c.steps[0, p, 0, 1]) - 5), -127, 127).round()
        c.kp.pool_view()[0].copy_(torch.from_numpy(c.rec).to(torch.int8))
        upload(c)
        q = queries(1, 1, 4, 64, 8)
        q[..., 0] = 512.0                                    # scores of up to 45 either way
        out = attend(c, [length], q, launches)
        check_attention(c, [length], q, out)
        c.kp.close()


def test_windows_and_several_tokens_over_such_pages():
    lens = [300, 77, 1024, 40]
    for width, passes, launches in ((64, 5, 1), (3000, 5, 10)):
        bt, n = tables_for(lens, width, 9)
        c = Cache((16, 2, 128), bt, n, seed=10)
        for h in range(2):
            place(c, (-106, 20, -3, 60, -40), lens, h)
        upload(c)
        q = queries(4, passes, 16, 128, 11)
        check_attention(c, lens, q, attend(c, lens, q, launches))
        check_attention(c, lens, q, attend(c, lens, q, 1, window=50, sink=20), 50, 20)
        c.kp.close()
