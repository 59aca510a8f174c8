"""What rows that are appended to an 8-bit page leave to the others: each growth of the step rounds older records again, and
rows that are cut off again, as rejected drafts are, leave the step as it is -- until the page is begun again."""
import numpy as np
import pytest

import ref_step as ref


def test_an_older_rows_error_stays_below_a_step():
    """Half of the step that wrote it, and half of each coarser one: below 1/2 + 1/4 + .. of the last, and beyond half of it."""
    from test_gpu_cache8 import bf16
    rng = np.random.default_rng(0)
    worst = 0.0
    for _ in range(200):
        rec, steps, rows = np.zeros((1, 1, 2, 16, 64)), np.zeros((1, 1, 2)), []
        for slot in range(16):
            rows.append(bf16(rng.standard_normal((1, 1, 2, 64)) * 2.0 ** (slot if slot < 4 else 3)))      # 8 bits: at most 127.5 steps
            ref.append8(rec, steps, 0, slot, rows[-1])
            x = np.concatenate(rows)
            off = np.abs(rec[0, :, :, :slot + 1].transpose(2, 0, 1, 3) * steps[0, None, :, :, None] - x) / steps[0, None, :, :, None]
            # a row of this call: half a step; a step lies in (m / 128, m / 64] of the largest m so far
            assert off[-1].max() <= 0.5 and off.max() < 1.0
            m = np.abs(x).max((0, 3))
            assert np.all(m / 128 < steps[0]) and np.all(steps[0] <= m / 64)
            worst = max(worst, off.max())
    assert worst > 0.55
    assert ref.need_step(np.zeros(4)) == 2.0 ** -106 > 2.0 ** -101 / 64 and ref.need_step(np.array([2.0 ** -101])) == 2.0 ** -106


@pytest.mark.gpu
@pytest.mark.parametrize("layout", [(32, 8, 128), (4, 1, 64)])
@pytest.mark.parametrize("factor", [1.0, 64.0, 2.0 ** -20, np.inf])
def test_rejected_drafts_of_another_size(layout, factor):
    """Steps of four drafts, of which some stay; the rejected ones are `factor` times as large."""
    from test_gpu_cache8 import Cache, bf16, tables_for, to_dev
    start, total = [0, 3, 14], 70
    bt, n = tables_for([s + total + 8 for s in start], 8, 1)
    c = Cache(layout, bt, n, seed=2)
    rng = np.random.default_rng(3)
    lens, kept = list(start), [np.zeros((0, c.K, 2, c.D)) for _ in start]
    clean = c.rec.copy(), c.steps.copy()                     # the same appends without the rejected rows
    while min(L - s for L, s in zip(lens, start)) < total - 4:
        stay = rng.integers(0, 4, 3) + 1
        rows = bf16(rng.standard_normal((3, 4, c.K, 2, c.D)))
        for r in range(3):
            rows[r, stay[r]:] = bf16(rows[r, stay[r]:] * factor)
        new = rows.reshape(12, c.K, 2, c.D)
        c.kp.kv8_append(0, c.btd, c.lens([L + 4 for L in lens]), to_dev(new[:, :, 0]), to_dev(new[:, :, 1]))
        for r in range(3):
            c.append_ref(r, lens[r] + 4, rows[r])
            ref.append8_tokens(clean[0][0], clean[1][0], bt[r], lens[r] + stay[r], rows[r, :stay[r]])
            kept[r] = np.concatenate([kept[r], rows[r, :stay[r]]])
            lens[r] = int(min(lens[r] + stay[r], start[r] + total))
            kept[r] = kept[r][:lens[r] - start[r]]
    c.check()
    for r in range(3):
        t = np.arange(-(-start[r] // 16) * 16, lens[r])      # pages that were begun here
        step = c.steps[0][bt[r][t // 16]][..., None]
        fine = clean[1][0][bt[r][t // 16]][..., None]
        value, x = c.values(r, lens[r])[t], kept[r][t - start[r]]
        if np.isinf(factor):                                 # no step says how large the rows that stay are
            assert np.isnan(step).any() and np.all(np.isnan(step) | (step >= fine))
            good = np.broadcast_to(np.isfinite(step), value.shape)
            assert np.all(np.abs(value - x)[good] < np.broadcast_to(step, value.shape)[good])
        else:
            assert np.all(step >= fine) and np.all(np.abs(value - x) < step)
            assert (np.median(step / fine) >= 16) == (factor == 64.0)
    # a page that is begun again forgets
    rows = bf16(rng.standard_normal((3 * 16, c.K, 2, c.D)))
    c.kp.kv8_append(0, c.btd, c.lens([16] * 3), to_dev(rows[:, :, 0]), to_dev(rows[:, :, 1]))
    for r in range(3):
        c.append_ref(r, 16, rows[16 * r:16 * r + 16])
    c.check()
    assert np.isfinite(c.steps[0][bt[:, 0]]).all() and c.steps[0][bt[:, 0]].max() <= 2.0 ** -3
    c.kp.close()
