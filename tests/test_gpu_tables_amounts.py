"""Pages handed out and taken back with the lengths written over the amounts, which are read no more then."""
import numpy as np
import pytest
import torch

import ref_step as ref
from test_gpu_tables import State, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("count_in_place", [False, True])
@pytest.mark.parametrize("batch", [1, 33, 300, 1030, 8192])
def test_lengths_over_the_amounts(batch, count_in_place):
    rng = np.random.default_rng(batch)
    lens = [int(x) for x in rng.integers(0, 60, batch)]
    s = State(lens, 9, 9 * batch + 7, 2 * batch + 1, batch)
    d = s.dev
    for step in range(3):
        new = [int(min(x, 144 - n)) for x, n in zip(rng.integers(0, 30, batch), s.lens)]
        if step == 1:
            new[batch // 2] = -1                             # unusable: its length stays
        amounts, total = ints(new), sum(max(0, x) for x in new)
        start, step_lens, slots = ints([-9] * (batch + 1)), ints([-9] * batch), ints([-9] * (total + 1), torch.int64)
        count = d["count"] if count_in_place else ints([-9])
        s.kp.pages_assign(d["tables"], d["lens"], amounts, d["free"], d["count"], lens_out=amounts, count_out=count, step_lens=step_lens, new_start=start,
                          slots=slots[:total] if total else None)
        out, left, step_, start_, slots_, bad = ref.assign(s.tables, s.lens, new, s.free, s.count, s.num_pages)
        assert amounts.tolist() == out and count.tolist() == [left] and d["lens"].tolist() == s.lens
        assert step_lens.tolist() == step_ and start.tolist() == start_ and slots.tolist() == slots_ + [-9]
        np.testing.assert_array_equal(d["tables"].cpu().numpy(), s.tables)
        assert (s.kp.check_status(raise_on_error=False) != 0) == bad
        s.lens, s.count, d["lens"], d["count"] = out, left, amounts, count

        keep = [n if rng.random() < 0.6 else int(rng.integers(0, n + 1)) for n in s.lens]
        if step == 2:
            keep[0] = s.lens[0] + 1
        amounts, count = ints(keep), d["count"] if count_in_place else ints([-9])
        s.kp.pages_release(d["tables"], d["lens"], amounts, d["free"], d["count"], lens_out=amounts, count_out=count)
        out, left, bad = ref.release(s.tables, s.lens, keep, s.free, s.count, s.num_pages)
        assert amounts.tolist() == out and count.tolist() == [left] and d["lens"].tolist() == s.lens
        np.testing.assert_array_equal(d["free"].cpu().numpy(), s.free)
        assert (s.kp.check_status(raise_on_error=False) != 0) == bad
        s.lens, s.count, d["lens"], d["count"] = out, left, amounts, count
    s.kp.close()
