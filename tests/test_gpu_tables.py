"""Pages handed out and taken back on the GPU, against loops over requests: exactly."""
import numpy as np
import pytest
import torch

import ref_step as ref

pytestmark = pytest.mark.gpu


def ints(x, dtype=torch.int32):
    return torch.tensor(np.asarray(x), dtype=dtype, device="cuda")


class State:
    def __init__(self, lens, width, num_pages, free, seed, max_batch=None):
        from paper_2501_08090_b200 import binding as b
        self.b, rng = b, np.random.default_rng(seed)
        order = rng.permutation(num_pages).astype(np.int32)
        self.tables = np.full((len(lens), width), -1, dtype=np.int32)
        at = 0
        for r, n in enumerate(lens):
            k = min(max(0, ref.pages(n)), width)
            self.tables[r, :k] = order[at:at + k]
            at += k
        assert at + free <= num_pages
        self.free = np.full(num_pages, -7, dtype=np.int32)
        self.free[:free] = order[at:at + free]
        self.lens, self.count, self.num_pages = list(lens), free, num_pages
        self.kp = b.KvPool(b.make_config(1, 4, 1, 64, num_pages, width, max_batch or len(lens)))
        self.dev = dict(tables=ints(self.tables), lens=ints(lens), free=ints(self.free), count=ints([free]))

    def assign(self, new, n_slots=None, in_place=False, want=True):
        d, B = self.dev, len(self.lens)
        total = sum(max(0, x) for x in new)
        n_slots = total if n_slots is None else n_slots
        out = dict(lens=d["lens"] if in_place else ints([-9] * B), count=d["count"] if in_place else ints([-9]), step=ints([-9] * B),
                   start=ints([-9] * (B + 1)), slots=ints([-9] * (n_slots + 2), torch.int64))
        self.kp.pages_assign(d["tables"], d["lens"], ints(new), d["free"], d["count"], lens_out=out["lens"], count_out=out["count"],
                             step_lens=out["step"] if want else None, new_start=out["start"] if want else None,
                             slots=out["slots"][:n_slots] if want and n_slots else None)
        lens, count, step, start, slots, bad = ref.assign(self.tables, self.lens, new, self.free, self.count, self.num_pages)
        assert out["lens"].tolist() == lens and out["count"].tolist() == [count]
        if want:
            assert out["step"].tolist() == step and out["start"].tolist() == start
            assert out["slots"].tolist() == slots[:n_slots] + [-9] * (n_slots + 2 - min(n_slots, total))
        np.testing.assert_array_equal(d["tables"].cpu().numpy(), self.tables)
        np.testing.assert_array_equal(d["free"].cpu().numpy(), self.free)
        bits = self.kp.check_status(raise_on_error=False)
        assert (bits != 0) == bad
        self.lens, self.count = lens, count
        d["lens"], d["count"] = out["lens"], out["count"]
        return bits

    def release(self, keep, in_place=False):
        d, B = self.dev, len(self.lens)
        out = dict(lens=d["lens"] if in_place else ints([-9] * B), count=d["count"] if in_place else ints([-9]))
        self.kp.pages_release(d["tables"], d["lens"], ints(keep), d["free"], d["count"], lens_out=out["lens"], count_out=out["count"])
        lens, count, bad = ref.release(self.tables, self.lens, keep, self.free, self.count, self.num_pages)
        assert out["lens"].tolist() == lens and out["count"].tolist() == [count]
        np.testing.assert_array_equal(d["tables"].cpu().numpy(), self.tables)
        np.testing.assert_array_equal(d["free"].cpu().numpy(), self.free)
        bits = self.kp.check_status(raise_on_error=False)
        assert (bits != 0) == bad
        self.lens, self.count = lens, count
        d["lens"], d["count"] = out["lens"], out["count"]
        return bits


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("batch", [1, 2, 31, 256, 257, 1025, 3000])
def test_steps_of_growing_and_shrinking_requests(batch, in_place):
    rng = np.random.default_rng(batch)
    lens = [int(x) for x in rng.integers(0, 100, batch)]
    s = State(lens, 12, batch * 12 + 5, 4 * batch, batch)
    for step in range(5):
        s.assign([int(min(x, 192 - n)) for x, n in zip(rng.integers(0, 20, batch), s.lens)], in_place=in_place)
        s.release([int(rng.integers(0, n + 1)) if rng.random() < 0.3 else n for n in s.lens], in_place=in_place)
    held = [p for r, n in enumerate(s.lens) for p in s.tables[r][:ref.pages(n)]] + list(s.free[:s.count])
    assert len(set(held)) == len(held) and len(held) == sum(ref.pages(n) for n in lens) + 4 * batch
    s.kp.close()


def test_one_token_each():
    s = State([16 * (i % 3) + i % 17 for i in range(300)], 5, 1500, 200, 1)
    for _ in range(20):
        s.assign([1] * 300)
    s.kp.close()


def test_prompts_fill_many_slots():
    """A cluster of thread blocks writes them; one request's prompt is longer than all others' together."""
    new = [1, 0, 40000, 17, 16, 0, 2047, 1]
    s = State([0, 5, 33, 16, 0, 7, 100, 31], 2600, 3000, 2900, 2)
    s.assign(new)
    s.release([0] * 8)
    s.assign(new[::-1], in_place=True, n_slots=9000)
    s.release([n // 2 for n in s.lens], in_place=True)
    s.kp.close()


def test_the_largest_batch():
    rng = np.random.default_rng(3)
    s = State([int(x) for x in rng.integers(0, 40, 8192)], 5, 8192 * 5, 9000, 3)
    s.assign([int(x) for x in rng.integers(0, 30, 8192)])
    s.release([n if i % 5 else 0 for i, n in enumerate(s.lens)])
    s.kp.close()


def test_an_assignment_that_is_released_leaves_the_list_as_it_was():
    s = State([3, 100, 0, 64], 20, 60, 40, 4)
    before, lens = s.free.copy(), list(s.lens)
    s.assign([50, 1, 200, 16])
    assert s.count < 40
    s.release(lens)
    np.testing.assert_array_equal(s.free, before)
    assert s.count == 40 and s.lens == lens


def test_too_few_pages():
    """Who does not fit takes nothing, nor does anybody behind it that needs a page; who needs none is served."""
    s = State([16, 10, 16, 5, 0], 8, 20, 3, 5)
    assert s.assign([32, 3, 40, 2, 16]) == 0
    assert s.lens == [48, 13, 16, 7, 0] and s.count == 1
    assert s.assign([0, 0, 0, 0, 1]) == 0 and s.lens[4] == 1 and s.count == 0
    assert s.assign([1, 3, 1, 9, 15]) == 0 and s.lens == [48, 16, 16, 16, 16] and s.count == 0
    s.kp.close()


def test_bad_lengths_counts_and_pages():
    s = State([10, 20, 30, 40], 4, 30, 9, 6)
    s.lens[1] = -2
    s.dev["lens"][1] = -2
    assert s.assign([5, 3, -1, 100]) == s.b.STATUS_BAD_LENGTH
    assert s.lens == [15, -2, 30, 40]
    s.lens[1] = 20
    s.dev["lens"][1] = 20
    assert s.release([16, 5, -1, 41]) == s.b.STATUS_BAD_LENGTH and s.lens == [15, 5, 30, 40]
    s.free[s.count - 1] = 30                                # a page outside the pool lies on top
    s.dev["free"][s.count - 1] = 30
    assert s.assign([0, 0, 5, 0]) == s.b.STATUS_BAD_PAGE and s.tables[2, 2] == -1
    assert s.release([15, 5, 30, 0]) == s.b.STATUS_BAD_PAGE
    s.kp.close()
    for count, cut in ((-5, 0), (31, 30)):
        s = State([10], 4, 30, 0, 7)
        s.free[:] = np.arange(30)
        s.dev["free"].copy_(ints(s.free))
        s.dev["count"].fill_(count)
        s.count = cut
        lens_out, count_out = ints([0]), ints([0])
        s.kp.pages_assign(s.dev["tables"], s.dev["lens"], ints([16]), s.dev["free"], s.dev["count"], lens_out=lens_out, count_out=count_out)
        assert s.kp.check_status(raise_on_error=False) == s.b.STATUS_BAD_PAGE
        assert (lens_out.tolist(), count_out.tolist()) == (([10], [0]) if cut == 0 else ([26], [29]))
        s.kp.close()


def test_pages_beyond_the_list_are_dropped():
    """Pages given back twice: the list is never written past its end."""
    s = State([160], 10, 12, 2, 8)
    s.free[2:] = 1
    s.dev["free"].copy_(ints(s.free))
    s.dev["count"].fill_(7)
    s.count = 7
    assert s.release([0]) == s.b.STATUS_BAD_PAGE and s.count == 12
    s.kp.close()


def test_amounts_whose_sums_pass_32_bits():
    """Refused requests' tokens count in the sums, which stop at 2^31 - 1."""
    s = State([5, 5, 5], 4, 20, 10, 9)
    d, start, slots = s.dev, ints([0] * 4), ints([-9] * 8, torch.int64)
    step, lens, count = ints([0] * 3), ints([0] * 3), ints([0])
    s.kp.pages_assign(d["tables"], d["lens"], ints([3, 2 ** 31 - 1, 2 ** 31 - 1]), d["free"], d["count"], lens_out=lens, count_out=count, step_lens=step,
                      new_start=start, slots=slots)
    assert s.kp.check_status(raise_on_error=False) == s.b.STATUS_BAD_LENGTH
    assert start.tolist() == [0, 3, 2 ** 31 - 1, 2 ** 31 - 1] and step.tolist() == [8, 0, 0] and lens.tolist() == [8, 5, 5]
    page = int(s.tables[0, 0])
    assert slots.tolist() == [page * 16 + 5, page * 16 + 6, page * 16 + 7, -1, -1, -1, -1, -1]
    s.kp.close()


def test_outputs_that_are_not_wanted_and_eight_bit_handles():
    s = State([5, 30], 4, 20, 10, 10)
    s.assign([20, 3], want=False)
    eight = s.b.Kv8Pool(s.b.make_config(1, 4, 1, 64, 20, 4, 2))
    d, lens, count = s.dev, ints([0, 0]), ints([0])
    eight.pages_release(d["tables"], d["lens"], ints([0, 0]), d["free"], d["count"], lens_out=lens, count_out=count)
    assert lens.tolist() == [0, 0] and count.tolist() == [s.count + sum(ref.pages(n) for n in s.lens)] and eight.check_status() == 0
    eight.close(); s.kp.close()


def test_a_decode_step_right_behind_reads_the_new_tables():
    """pages_assign, then decode_step, which otherwise reads its tables ahead of its predecessor's end."""
    from paper_2501_08090_b200 import binding as b
    B, steps = 64, 50
    kp = b.KvPool(b.make_config(1, 8, 2, 128, B * 8, 8, B))
    kp.pool.zero_()
    tables, lens, free, count = ints(np.full((B, 8), -1)), ints([0] * B), ints(np.random.default_rng(11).permutation(B * 8)), ints([B * 8])
    new, one = ints([1] * B), torch.ones(B, 2, 128, dtype=torch.bfloat16, device="cuda")
    q, outs = torch.zeros(B, 8, 128, dtype=torch.bfloat16, device="cuda"), []
    graph = torch.cuda.CUDAGraph()
    out = torch.empty_like(q)

    def step():
        kp.pages_assign(tables, lens, new, free, count, lens_out=lens, count_out=count)
        kp.decode_step(0, tables, lens, q, one, one, out)

    step()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    for i in range(steps):
        if i % 2:
            step()
        else:
            graph.replay()
        outs.append(out.clone())
    torch.cuda.synchronize()
    assert lens.tolist() == [steps + 1] * B and count.tolist() == [B * 8 - B * ref.pages(steps + 1)] and kp.check_status() == 0
    for o in outs:                                          # every value row that a length covers is ones
        assert torch.all(o == 1)
    kp.close()


def test_refusals():
    from paper_2501_08090_b200 import binding as b
    kp = b.KvPool(b.make_config(1, 4, 1, 64, 20, 4, 2))
    t, lens, new, free, count = ints(np.zeros((2, 4))), ints([1, 1]), ints([1, 1]), ints(range(20)), ints([20])
    out, cnt = ints([0, 0]), ints([0])
    n = kp.launch_count()
    for bad in (dict(lens_out=t.view(-1)[:2]), dict(count_out=lens[:1]), dict(step_lens=out), dict(step_lens=lens), dict(new_start=free[:3]),
                dict(new_start=t.view(-1)[5:8]), dict(count_out=out[1:]), dict(step_lens=new), dict(slots=free.view(torch.int64)[:2])):
        with pytest.raises(b.CkvError) as e:
            kp.pages_assign(t, lens, new, free, count, **{**dict(lens_out=out, count_out=cnt), **bad})
        assert e.value.code == b.CKV_EINVAL and "overlap" in str(e.value)
    for bad in (dict(lens_out=t.view(-1)[:2]), dict(count_out=free[:1]), dict(lens_out=free[3:5])):
        with pytest.raises(b.CkvError):
            kp.pages_release(t, lens, new, free, count, **{**dict(lens_out=out, count_out=cnt), **bad})
    for args in ((t[:, :3], lens, new, free, count), (t, lens, new[:1], free, count), (t, lens, new, free[:19], count), (t, lens, new, free, ints([1, 2])),
                 (t, lens.long(), new, free, count)):
        with pytest.raises(ValueError):
            kp.pages_assign(*args, lens_out=out, count_out=cnt)
        with pytest.raises(ValueError):
            kp.pages_release(*args, lens_out=out, count_out=cnt)
    with pytest.raises(ValueError):
        kp.pages_assign(t, lens, new, free, count, lens_out=out, count_out=cnt, slots=ints([0, 0]))
    with pytest.raises(b.CkvError):
        kp.pages_assign(ints(np.zeros((3, 4))), ints([1] * 3), ints([1] * 3), free, count, lens_out=ints([0] * 3), count_out=cnt)
    assert kp.launch_count() == n
    kp.close()
