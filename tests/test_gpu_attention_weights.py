"""Softmax weights reach the product with V unrounded, to fp32's order: what their rounding to the matrix instruction's type
leaves is multiplied too.  Keys that are alike and values that cancel show it: outputs are far smaller than what is summed."""
import numpy as np
import pytest
import torch

import ref_step as ref
import test_gpu_window
from test_gpu_cache8 import Cache, bf16, queries, tables_for, to_dev

pytestmark = pytest.mark.gpu

# cut to bf16 a weight loses 2^-7 at most, and what that leaves is rounded by half a step, 2^-8 of it: 2^-15; half a step of
# fp16 is 2^-11, and of what that leaves as much again: 2^-22
BF16_BITS, FP16_BITS = 15, 22
LENS = [2, 31, 100, 700, 33, 1500]
# layout, new tokens, pages of a table, window, sink, launches
CASES = [((4, 1, 64), 1, 94, 300, 0, 1), ((32, 8, 128), 2, 94, 1000, 20, 1), ((8, 1, 128), 2, 94, 40, 5, 1), ((8, 2, 64), 1, 6000, 10 ** 6, 0, 2),
         ((8, 2, 128), 2, 6000, 10 ** 6, 0, 2)]


def alike(rows, seed):
    """Rows [pages][Hkv][2][16][d] whose keys nearly agree and whose values, a token's and the next's, nearly cancel."""
    rng = np.random.default_rng(seed)
    rows[:, :, 0] = rng.standard_normal(rows.shape[:2] + (1, rows.shape[-1])) * 2.0 ** -4 + rng.standard_normal(rows[:, :, 0].shape) * 2.0 ** -7
    rows[:, :, 1, 1::2] = -rows[:, :, 1, ::2]
    return rows


@pytest.mark.parametrize("layout,q_len,width,window,sink,launches", CASES)
def test_window(layout, q_len, width, window, sink, launches):
    bt, n = tables_for(LENS, width, 1)
    c = test_gpu_window.Cache(layout, bt, n, seed=2)
    c.pool = bf16(alike(c.pool, 3))
    c.upload()
    q = queries(len(LENS), q_len, c.H, c.D, 4)
    before = c.kp.launch_count()
    out = c.run(LENS, q, window, sink)
    assert c.kp.launch_count() - before == launches
    check(c, lambda r, L, h: (c.pool[bt[r][np.arange(L) // 16], h, 0, np.arange(L) % 16], c.pool[bt[r][np.arange(L) // 16], h, 1, np.arange(L) % 16]), q, out,
          window, sink, BF16_BITS)
    c.kp.close()


def check(c, kv, q, out, window, sink, bits, steps=None):
    G = c.H // c.K
    got = out.double().cpu().numpy().reshape(q.shape)
    small = 0
    for r, L in enumerate(LENS):
        for h in range(c.K):
            k, v = kv(r, L, h)
            args = (q[r][:, h * G:(h + 1) * G], k, v, L, window, sink)
            want, size, mass, floor = ref.attend(*args) + (None,) if steps is None else ref.attend(*args, steps(r, L, h))
            off, most = np.abs(got[r][:, h * G:(h + 1) * G] - want), ref.attend_tolerance(want, size, mass, bits, floor)
            assert np.all(off <= most), (r, h, (off / most).max())
            small += np.sum(np.abs(want) < size / 64)
    assert small > 1000                                      # there is something to see


@pytest.mark.parametrize("layout,q_len,width,window,sink,launches", CASES)
def test_cache_in_8_bits(layout, q_len, width, window, sink, launches):
    bt, n = tables_for(LENS, width, 5)
    c = Cache(layout, bt, n, seed=6)
    rows = alike(np.random.default_rng(7).standard_normal((n, c.K, 2, 16, c.D)), 8)
    for page in range(n):
        ref.append8(c.rec[0], c.steps[0], page, 0, bf16(rows[page].transpose(2, 0, 1, 3)))
    rec, steps = c.kp.pool_view()
    rec.copy_(torch.from_numpy(c.rec).to(torch.int8))
    steps.copy_(torch.from_numpy(c.steps).float())
    q = queries(len(LENS), q_len, c.H, c.D, 9)
    out = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
    before = c.kp.launch_count()
    c.kp.kv8_attention(0, c.btd, c.lens(LENS), to_dev(q), out, window=window, sink=sink)
    assert c.kp.launch_count() - before == launches
    c.check()
    check(c, lambda r, L, h: (c.values(r, L)[:, h, 0], c.values(r, L)[:, h, 1]), q, out, window, sink, FP16_BITS, lambda r, L, h: c.v_steps(r, L, h))
    c.kp.close()


@pytest.mark.parametrize("layout,q_len,width,window,sink,launches", CASES)
def test_infinite_values_that_are_seen_stay_infinite(layout, q_len, width, window, sink, launches):
    """In the bf16 cache; a value of either sign makes its element that infinity, both make it NaN, others are as they were."""
    bt, n = tables_for(LENS, width, 10)
    c = test_gpu_window.Cache(layout, bt, n, seed=11)
    q = queries(len(LENS), q_len, c.H, c.D, 12)
    want = c.run(LENS, q, window, sink).float()
    for r, L in enumerate(LENS):
        for t, element, value in ((L - 2, 3, np.inf), (max(L - 30, 0), 8, -np.inf), (max(L - 25, 0), 17, np.inf), (L - q_len, 17, -np.inf), (max(L - 25, 0), 40, np.inf)):
            c.pool[bt[r, t // 16], 0, 1, t % 16, element] = value
            want[r, :, :c.H // c.K, element] = value if element != 17 or max(L - 25, 0) == L - q_len else np.nan
    c.upload()
    got = c.run(LENS, q, window, sink).float()
    for r, L in enumerate(LENS):
        for i in range(q_len):                               # what a new token does not see yet leaves it alone
            if L - 2 > L - q_len + i:
                want[r, i, :, 3] = got[r, i, :, 3]
                assert torch.isfinite(got[r, i, :, 3]).all()
    assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(7.0, 1e38, -1e38), want.nan_to_num(7.0, 1e38, -1e38))
    assert c.kp.check_status() == 0
    c.kp.close()
