"""The 8-bit cache against its definition: appended records and steps bit by bit, gathered values exactly, attention
within its roundings."""
import math

import numpy as np
import pytest
import torch

import ref_step as ref
from helpers import bits_to_dev, dev_to_bits, widen

pytestmark = pytest.mark.gpu

LAYOUTS = [(32, 8, 128), (64, 8, 128), (4, 1, 64), (6, 6, 128), (35, 5, 128), (12, 4, 64), (8, 1, 128)]


def bf16(x):
    """Nearest bf16 of an array, as float64."""
    return torch.from_numpy(np.asarray(x, dtype=np.float64)).to(torch.bfloat16).double().numpy()


def to_dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).cuda()


def tables_for(lens, width, seed, spare=3):
    """(tables [B][width] with -1 behind each request's pages, pages of the pool)."""
    rng = np.random.default_rng(seed)
    counts = [max(0, ref.pages(n)) for n in lens]
    order = rng.permutation(sum(counts) + spare).astype(np.int32)
    bt = np.full((len(lens), width), -1, dtype=np.int32)
    at = 0
    for r, n in enumerate(counts):
        bt[r, :n] = order[at:at + n]
        at += n
    return bt, len(order)


class Cache:
    """A Kv8Pool beside its records and steps in numpy."""

    def __init__(self, layout, bt, num_pages, layers=1, layer=0, fill=True, seed=0):
        from paper_2501_08090_b200 import binding as b
        self.b, self.layer, self.bt = b, layer, bt
        self.H, self.K, self.D = layout
        cfg = b.make_config(layers, self.H, self.K, self.D, num_pages, bt.shape[1], bt.shape[0])
        self.kp = b.Kv8Pool(cfg)
        rec, steps = self.kp.pool_view()
        rng = np.random.default_rng(seed)
        if fill:                                             # what older calls left: any bytes, steps of any size
            rec.copy_(torch.from_numpy(rng.integers(-127, 128, rec.shape, dtype=np.int8)))
            steps.copy_(torch.from_numpy(2.0 ** rng.integers(-9, -4, steps.shape)).float())
        self.rec, self.steps = rec.cpu().numpy().astype(np.float64), steps.double().cpu().numpy()
        self.btd = torch.from_numpy(bt).cuda()

    def lens(self, lens):
        return torch.tensor(lens, dtype=torch.int32, device="cuda")

    def check(self, status=0):
        bits = self.kp.check_status(raise_on_error=False)
        assert bits == status
        rec, steps = self.kp.pool_view()
        np.testing.assert_array_equal(rec.cpu().numpy(), self.rec)
        np.testing.assert_array_equal(steps.double().cpu().numpy(), self.steps)

    def append_ref(self, r, length, rows):
        ref.append8_tokens(self.rec[self.layer], self.steps[self.layer], self.bt[r], length, rows)

    def values(self, r, length):
        """float64 [tokens][Hkv][2][d]."""
        t = np.arange(length)
        page, slot = self.bt[r][t // 16], t % 16
        return self.rec[self.layer][page, :, :, slot] * self.steps[self.layer][page][..., None]

    def v_steps(self, r, length, h):
        """float64 [tokens]."""
        return self.steps[self.layer][self.bt[r][np.arange(length) // 16], h, 1]


def rows_of(n, K, D, seed, spread=2.0):
    """Keys and values [n][K][2][D] of very different size from token to token, bf16."""
    rng = np.random.default_rng(seed)
    return bf16(rng.standard_normal((n, K, 2, D)) * 2.0 ** rng.uniform(-spread, spread, (n, 1, 1, 1)))


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("chunks", [[1] * 40, [3, 5, 8, 1, 30], [16, 16, 1, 15, 2], [37]])
def test_appends_token_by_token_and_in_chunks(layout, chunks):
    """Every prefix of the chunks for three requests that start at different slots; older rows requantised as steps grow."""
    starts, total = [0, 5, 31], sum(chunks)
    bt, n = tables_for([s + total for s in starts], 8, 1)
    c = Cache(layout, bt, n, layers=2, layer=1)
    data = [rows_of(total, c.K, c.D, 10 + r) for r in range(3)]
    at = 0
    for m in chunks:
        lens = [s + at + m for s in starts]
        new = np.concatenate([d[at:at + m] for d in data])
        c.kp.kv8_append(1, c.btd, c.lens(lens), to_dev(new[:, :, 0]), to_dev(new[:, :, 1]))
        for r in range(3):
            c.append_ref(r, lens[r], data[r][at:at + m])
        at += m
    c.check()
    # a value is within half a step of the last row that was written exactly (its own requantisations apart)
    last = c.values(0, starts[0] + total)[-1]
    step = c.steps[1][bt[0][(starts[0] + total - 1) // 16]]
    assert np.all(np.abs(last - data[0][-1]) <= step[..., None] / 2)
    c.kp.close()


def test_borders_of_the_steps():
    """Largest magnitudes beside powers of two, halves that round to even, 127.5 steps, tiny and huge rows, zeros."""
    tops = [1.0, 0.99609375, 127.5 / 64, -127.5 / 64, 2.0 ** -100, 2.0 ** -101, 2.0 ** -133, 0.0, 3.3895e38, -3.3895e38, 2.0 ** 120, 1.5]
    bt, n = tables_for([1] * len(tops), 1, 2)
    c = Cache((4, 1, 64), bt, n)
    rows = np.zeros((len(tops), 1, 2, 64))
    for r, top in enumerate(tops):
        rows[r, 0, :, 0] = top
        rows[r, 0, 0, 1:] = top * (np.arange(63) + 0.5) / 64
        rows[r, 0, 1, 1:] = -top * np.arange(63) / 127
    rows = bf16(rows)
    c.kp.kv8_append(0, c.btd, c.lens([1] * len(tops)), to_dev(rows[:, :, 0]), to_dev(rows[:, :, 1]))
    for r in range(len(tops)):
        c.append_ref(r, 1, rows[r:r + 1])
    c.check()
    c.kp.close()


def test_rows_that_are_not_finite_poison_their_block_until_the_page_begins_again():
    bt, n = tables_for([20, 20], 2, 3)
    c = Cache((8, 2, 128), bt, n)
    rows = rows_of(40, 2, 128, 4).reshape(2, 20, 2, 2, 128)
    rows[0, 3, 1, 0, 77] = np.inf
    rows[1, 17, 0, 1, 0] = np.nan

    def append(a, b):
        new = np.concatenate([rows[0, a:b], rows[1, a:b]])
        c.kp.kv8_append(0, c.btd, c.lens([b, b]), to_dev(new[:, :, 0]), to_dev(new[:, :, 1]))
        for r in range(2):
            c.append_ref(r, b, rows[r, a:b])

    for a, b in ((0, 2), (2, 4), (4, 9), (9, 16), (16, 20)):
        append(a, b)
    c.check()
    assert np.isnan(c.steps[0, bt[0, 0], 1, 0]) and np.isnan(c.steps[0, bt[1, 1], 0, 1]) and np.isnan(c.steps).sum() == 2
    rows[0, 3] = 1.0
    append(0, 16)
    c.check()
    assert np.isnan(c.steps).sum() == 1
    c.kp.close()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("layout,rotary", [((32, 8, 128), 128), ((35, 5, 128), 16), ((4, 1, 64), 64), ((12, 4, 64), 32)])
def test_rotated_append_quantises_what_the_bf16_cache_would_hold(layout, rotary, interleaved):
    """Queries and keys as kv_append_rope turns them: ragged prompts, rows of one projection's output, padding rows around."""
    H, K, D = layout
    new, ctx = [37, 0, 1, 16, 90, 5], [0, 9, 30, 16, 7, 43]
    lens = [a + b for a, b in zip(new, ctx)]
    bt, n = tables_for(lens, 8, 5)
    c = Cache(layout, bt, n)
    from paper_2501_08090_b200 import binding as b
    kp = b.KvPool(b.make_config(1, H, K, D, n, 8, len(lens)))
    pad, T = 3, sum(new) + 7
    qkv = to_dev(np.random.default_rng(6).standard_normal((T, H + 2 * K, D)) * 3)
    q, k, v = qkv[:, :H], qkv[:, H:H + K], qkv[:, H + K:]
    start = torch.tensor(np.cumsum([pad] + new), dtype=torch.int32, device="cuda")
    freq = (10000.0 ** (-torch.arange(rotary // 2, device="cuda") / (rotary // 2))).float()
    outs = [torch.full((T, H, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    kp.kv_append_rope(0, c.btd, c.lens(lens), q, k, v, outs[0], freq, new_start=start, interleaved=interleaved, scale=1.25)
    c.kp.kv8_append(0, c.btd, c.lens(lens), k, v, q=q, q_out=outs[1], inv_freq=freq, new_start=start, interleaved=interleaved, scale=1.25)
    assert torch.equal(outs[0].view(torch.int16), outs[1].view(torch.int16))
    pool = kp.pool_view()[0].double().cpu().numpy()
    for r, L in enumerate(lens):
        t = np.arange(ctx[r], L)
        c.append_ref(r, L, pool[bt[r][t // 16], :, :, t % 16].reshape(-1, K, 2, D))
    c.check()
    # in place of the queries, and a list that goes on behind the rows
    c.kp.kv8_append(0, c.btd, c.lens(lens), k, v, q=q, q_out=q, inv_freq=freq, new_start=start, interleaved=interleaved, scale=1.25)
    assert torch.equal(q[pad:pad + sum(new)], outs[0][pad:pad + sum(new)])
    c.check()
    c.kp.close(); kp.close()


def test_a_list_that_goes_on_behind_the_rows():
    """Rows from n_tokens on are nobody's; the positions of those before it stay what the list says."""
    lens = [20, 40]
    bt, n = tables_for(lens, 3, 7)
    c = Cache((4, 1, 64), bt, n)
    rows = rows_of(50, 1, 64, 8)
    start = torch.tensor([0, 20, 60], dtype=torch.int32, device="cuda")
    c.kp.kv8_append(0, c.btd, c.lens(lens), to_dev(rows[:, :, 0]), to_dev(rows[:, :, 1]), new_start=start)
    c.append_ref(0, 20, rows[:20])
    c.append_ref(1, 30, rows[20:])                          # 30 of request 1's 40 tokens have rows
    c.check()
    c.kp.close()


def test_unusable_lengths_and_pages_are_flagged_and_skipped():
    lens = [5, 0, 33, 2, 17]                                # 33: beyond the table of two pages; 2: fewer than its three new tokens
    bt, n = tables_for([5, 0, 0, 0, 17], 2, 9)
    bt[4, 1] = n                                            # outside the pool
    c = Cache((8, 2, 64), bt, n)
    rows = rows_of(15, 2, 64, 10)
    q = to_dev(np.ones((15, 8, 64)))
    q_out = torch.full_like(q, 9.0)
    freq = torch.zeros(32, device="cuda")                   # turns by nothing
    c.kp.kv8_append(0, c.btd, c.lens(lens), to_dev(rows[:, :, 0]), to_dev(rows[:, :, 1]), q=q, q_out=q_out, inv_freq=freq)
    c.append_ref(0, 5, rows[:3])
    ref.append8(c.rec[0], c.steps[0], bt[4, 0], 14, rows[12:14])          # its third token's page does not exist
    c.check(c.b.STATUS_BAD_LENGTH | c.b.STATUS_BAD_PAGE)
    want = torch.ones_like(q)
    want[3:12] = 0
    assert torch.equal(q_out, want)
    k, v = (torch.full((15, 2, 64), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    c.kp.kv8_gather(0, c.btd, c.lens(lens), k, v)
    assert c.kp.check_status(raise_on_error=False) == c.b.STATUS_BAD_LENGTH | c.b.STATUS_BAD_PAGE
    assert torch.equal(k[:3].double().cpu(), torch.from_numpy(c.values(0, 5)[2:, :, 0])) and not k[3:12].any() and not v[3:12].any()
    assert torch.equal(v[12:14].double().cpu(), torch.from_numpy(c.values(4, 16)[14:, :, 1])) and not k[14].any()
    c.kp.close()


@pytest.mark.parametrize("layout", LAYOUTS[1:4])
def test_gather_is_exact_and_writes_its_rows_alone(layout):
    lens, back = [1, 300, 16, 47, 33], [1, 300, 0, 20, 17]
    bt, n = tables_for(lens, 20, 11)
    c = Cache(layout, bt, n, layers=3, layer=2)
    c.steps[2, bt[3, 2], 0, 1] = np.nan
    c.kp.pool_view()[1].copy_(torch.from_numpy(c.steps).float())
    start, T = np.cumsum([2] + back), sum(back) + 6
    both = torch.full((T, 2 * c.K + 1, c.D), 5.0, dtype=torch.bfloat16, device="cuda")        # values beside keys, tokens apart
    k, v = both[:, :c.K], both[:, c.K:2 * c.K]
    c.kp.kv8_gather(2, c.btd, c.lens(lens), k, v, start=torch.tensor(start, dtype=torch.int32, device="cuda"))
    got = both.double().cpu().numpy()
    want = np.full(got.shape, 5.0)
    for r, L in enumerate(lens):
        x = c.values(r, L)[L - back[r]:]
        want[start[r]:start[r + 1], :c.K], want[start[r]:start[r + 1], c.K:2 * c.K] = x[:, :, 0], x[:, :, 1]
    np.testing.assert_array_equal(got, want)
    k1, v1 = (torch.empty(5 * 1, c.K, c.D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    c.kp.kv8_gather(2, c.btd, c.lens(lens), k1, v1)          # the last token of each
    np.testing.assert_array_equal(v1.double().cpu().numpy(), np.stack([c.values(r, L)[-1][:, 1] for r, L in enumerate(lens)]))
    c.check()
    c.kp.close()


# ---- attention

def queries(B, N, H, D, seed):
    return bf16(np.random.default_rng(seed).standard_normal((B, N, H, D)) * 1.5)


def check_attention(c, lens, q, out, window=0, sink=0, skip=()):
    G = c.H // c.K
    got = out.double().cpu().numpy().reshape(q.shape)
    for r, L in enumerate(lens):
        if r in skip:
            continue
        kv = c.values(r, L)
        for h in range(c.K):
            want, size, mass, floor = ref.attend(q[r][:, h * G:(h + 1) * G], kv[:, h, 0], kv[:, h, 1], L, window, sink, c.v_steps(r, L, h))
            off = np.abs(got[r][:, h * G:(h + 1) * G] - want)
            assert np.all(off <= ref.attend_tolerance(want, size, mass, 11, floor)), (r, h, off.max())


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("q_len", [1, 2, 5, 8])
def test_attention_over_ragged_contexts(layout, q_len):
    lens = [q_len, 8, 15, 16, 17, 31, 32, 33, 64, 100, 511, 1000]
    lens = [max(n, q_len) for n in lens]
    bt, n = tables_for(lens, 64, 12)
    c = Cache(layout, bt, n, layers=2, layer=1, seed=13)
    q = queries(len(lens), q_len, c.H, c.D, 14)
    for window, sink in ((0, 0), (17, 3), (100, 0)):
        out = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
        c.kp.kv8_attention(1, c.btd, c.lens(lens), to_dev(q), out, window=window, sink=sink)
        c.check()
        check_attention(c, lens, q, out, window, sink)
    c.kp.close()


@pytest.mark.parametrize("lens", [[1], [20000], [3] * 300 + [9000], [100] * 40, [4096, 1, 4096, 1, 700]])
def test_attention_however_the_work_is_cut(lens):
    bt, n = tables_for(lens, ref.pages(max(lens)), 15)
    c = Cache((8, 2, 128), bt, n, seed=16)
    q = queries(len(lens), 1, 8, 128, 17)
    outs = []
    for _ in range(2):
        out = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
        c.kp.kv8_attention(0, c.btd, c.lens(lens), to_dev(q), out)
        outs.append(out)
    assert torch.equal(outs[0], outs[1])
    check_attention(c, lens, q, outs[0])
    c.kp.close()


@pytest.mark.parametrize("batch", [1, 2, 3, 5, 9, 18, 36])
@pytest.mark.parametrize("layout,window,q_len", [((16, 8, 128), 0, 1), ((16, 8, 128), 900, 3), ((32, 8, 64), 0, 1)])
def test_attention_of_few_requests_and_many(batch, layout, window, q_len):
    """Short tables and windows, from as many CTAs a pair as fit to one."""
    lens = [40 + (577 * r) % 1100 for r in range(batch)]
    bt, n = tables_for(lens, ref.pages(1200), 41)
    c = Cache(layout, bt, n, seed=42)
    q = queries(batch, q_len, c.H, c.D, 43)
    out = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
    c.kp.kv8_attention(0, c.btd, c.lens(lens), to_dev(q), out, window=window, sink=5 if window else 0)
    c.check()
    check_attention(c, lens, q, out, window, 5 if window else 0)
    c.kp.close()


def test_attention_three_dimensional_queries_and_unusable_lengths():
    lens = [40, 0, 500, -3, 16, 10 ** 9]
    bt, n = tables_for([40, 0, 500, 0, 16, 0], 32, 18)
    c = Cache((12, 4, 64), bt, n, seed=19)
    q = queries(6, 1, 12, 64, 20)
    out = torch.full((6, 12, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    c.kp.kv8_attention(0, c.btd, c.lens(lens), to_dev(q[:, 0]), out, window=100)
    c.check(c.b.STATUS_BAD_LENGTH)
    assert not out[1].any() and not out[3].any() and not out[5].any()
    check_attention(c, lens, q, out, 100, 0, skip=(1, 3, 5))
    c.kp.close()


def test_attention_with_blocks_of_very_different_steps():
    """Steps from 2^-106 to 2^20 side by side: weights are taken against the largest contribution."""
    lens = [400]
    bt, n = tables_for(lens, 25, 21)
    c = Cache((4, 1, 64), bt, n, seed=22)
    rng = np.random.default_rng(23)
    c.steps[0, :, :, 1] = 2.0 ** rng.choice([-106, -60, -20, -6, 0, 9, 20], c.steps[0, :, :, 1].shape)
    c.steps[0, :, :, 0] = 2.0 ** -7
    c.kp.pool_view()[1].copy_(torch.from_numpy(c.steps).float())
    q = queries(1, 1, 4, 64, 24)
    out = torch.empty(1, 4, 64, dtype=torch.bfloat16, device="cuda")
    c.kp.kv8_attention(0, c.btd, c.lens(lens), to_dev(q[:, 0]), out)
    check_attention(c, lens, q, out)
    # every block tiny, or every block huge: sums stay normal numbers
    for exp in (-106, 100):
        c.steps[0, :, :, 1] = 2.0 ** exp
        c.kp.pool_view()[1].copy_(torch.from_numpy(c.steps).float())
        c.kp.kv8_attention(0, c.btd, c.lens(lens), to_dev(q[:, 0]), out)
        check_attention(c, lens, q, out)
    c.kp.close()


def test_attention_poisoned_blocks_reach_those_who_see_them():
    """A block that holds NaN makes rows that see one of its tokens NaN, keys or values; others are as if it were not there."""
    lens = [64, 64, 64, 64]
    bt, n = tables_for(lens, 4, 25)
    c = Cache((8, 2, 64), bt, n, seed=26)
    c.steps[0, bt[0, 1], 0, 0] = np.nan                    # keys of head 0, tokens 16 .. 31
    c.steps[0, bt[1, 1], 1, 1] = np.nan                    # values of head 1
    c.steps[0, bt[2, 3], 0, 1] = np.nan                    # tokens 48 .. 63
    c.kp.pool_view()[1].copy_(torch.from_numpy(c.steps).float())
    q = queries(4, 2, 8, 64, 27)
    for window, sink, seen in ((0, 0, (0, 1, 2)), (34, 0, (0, 1, 2)), (32, 16, (0, 1, 2)), (31, 4, (2,)), (20, 17, (0, 1, 2))):
        out = torch.empty(4, 2, 8, 64, dtype=torch.bfloat16, device="cuda")
        c.kp.kv8_attention(0, c.btd, c.lens(lens), to_dev(q), out, window=window, sink=sink)
        got = out.double().cpu().numpy()
        G = 4
        for r in range(4):
            kv = c.values(r, 64)
            for h in range(2):
                for i in range(2):
                    p = 62 + i
                    vis = [t for t in range(p + 1) if not window or t > p - window or t < sink]
                    x = got[r, i, h * G:(h + 1) * G]
                    if np.isnan(kv[vis, h]).any():
                        assert r in seen and np.isnan(x).all()
                    else:
                        kv0 = np.nan_to_num(kv[:, h])
                        want, size, mass, floor = ref.attend(q[r][:, h * G:(h + 1) * G], kv0[:, 0], kv0[:, 1], 64, window, sink,
                                                             np.nan_to_num(c.v_steps(r, 64, h)))
                        assert np.all(np.abs(x - want[i]) <= ref.attend_tolerance(want, size, mass, 11, floor)[i])
    c.kp.close()


def test_attention_queries_of_any_size():
    """Powers of two on the queries are taken off and put back; zeros give the mean; what is not finite gives NaN."""
    lens = [200] * 6
    bt, n = tables_for(lens, 13, 28)
    c = Cache((4, 1, 128), bt, n, seed=29)
    q = queries(6, 1, 4, 128, 30)
    q[1] *= 2.0 ** -60
    q[2] = 0.0
    q[3] *= 2.0 ** 6
    q[3, 0, :, 5] = 2.0 ** -30                              # far below the largest
    q[4, 0, 2, 9] = np.nan
    q[5, 0, 1, 3] = np.inf
    out = torch.empty(6, 1, 4, 128, dtype=torch.bfloat16, device="cuda")
    c.kp.kv8_attention(0, c.btd, c.lens(lens), to_dev(q), out)
    check_attention(c, lens, q, out, skip=(4, 5))
    got = out.double().cpu().numpy()
    assert np.isnan(got[4, 0, 2]).all() and np.isfinite(got[4, 0, [0, 1, 3]]).all()
    # an infinite query element: scores of plus or minus infinity, or NaN where the key is 0 there
    assert np.isnan(got[5, 0, 1]).all() and np.isfinite(got[5, 0, [0, 2, 3]]).all()
    c.kp.close()


def test_offsets_beyond_32_bits_and_bad_pages():
    """The last pages of a cache of 5 GB; then a page id outside it, which is flagged and not followed."""
    K, D, num = 8, 128, 150000
    bt = np.full((2, 4), -1, dtype=np.int32)
    bt[0], bt[1, :2] = [num - 1, num - 2, 3, num - 7], [num - 3, num - 4]
    from paper_2501_08090_b200 import binding as b
    kp = b.Kv8Pool(b.make_config(1, 32, K, D, num, 4, 2))
    rows = rows_of(64 + 20, K, D, 31, 1.0)
    lens = torch.tensor([64, 20], dtype=torch.int32, device="cuda")
    start = torch.tensor([0, 64, 84], dtype=torch.int32, device="cuda")
    btd = torch.from_numpy(bt).cuda()
    kp.kv8_append(0, btd, lens, to_dev(rows[:, :, 0]), to_dev(rows[:, :, 1]), new_start=start)
    k, v = (torch.empty(84, K, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    kp.kv8_gather(0, btd, lens, k, v, start=start)
    values = np.stack([k.double().cpu().numpy(), v.double().cpu().numpy()], 2)
    small_rec, small_steps = np.zeros((6, K, 2, 16, D)), np.ones((6, K, 2))
    ref.append8_tokens(small_rec, small_steps, [0, 1, 2, 3], 64, rows[:64])
    ref.append8_tokens(small_rec, small_steps, [4, 5], 20, rows[64:])
    t = np.arange(84)
    page, slot = np.where(t < 64, t // 16, 4 + (t - 64) // 16), np.where(t < 64, t % 16, (t - 64) % 16)
    np.testing.assert_array_equal(values, small_rec[page, :, :, slot] * small_steps[page][..., None])
    q = queries(2, 1, 32, D, 32)
    out = torch.empty(2, 32, D, dtype=torch.bfloat16, device="cuda")
    kp.kv8_attention(0, btd, lens, to_dev(q[:, 0]), out)
    assert kp.check_status() == 0
    got = out.double().cpu().numpy()
    for r, (a, L) in enumerate(((0, 64), (64, 20))):
        for h in range(K):
            want, size, mass, floor = ref.attend(q[r][:, h * 4:h * 4 + 4], values[a:a + L, h, 0], values[a:a + L, h, 1], L, 0, 0,
                                                 small_steps[page[a:a + L], h, 1])
            assert np.all(np.abs(got[r, h * 4:h * 4 + 4] - want[0]) <= ref.attend_tolerance(want, size, mass, 11, floor)[0])
    before = out[0].clone()
    btd[1, 0] = num
    kp.kv8_attention(0, btd, lens, to_dev(q[:, 0]), out)
    assert kp.check_status(raise_on_error=False) == b.STATUS_BAD_PAGE and torch.equal(out[0], before)
    kp.close()


def test_calls_for_the_other_cache_are_refused():
    from paper_2501_08090_b200 import binding as b
    cfg = b.make_config(1, 8, 2, 64, 10, 4, 2)
    eight, sixteen = b.Kv8Pool(cfg), b.KvPool(cfg)
    bt = torch.zeros(2, 4, dtype=torch.int32, device="cuda")
    sl = torch.ones(2, dtype=torch.int32, device="cuda")
    q = torch.zeros(2, 8, 64, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(2, 2, 64, dtype=torch.bfloat16, device="cuda")
    freq = torch.zeros(32, device="cuda")
    image = torch.zeros(10 * eight.swap_image_bytes(1), dtype=torch.uint8).pin_memory()
    for call in (lambda: eight.kv_append(0, bt, sl, k, k), lambda: eight.decode_attention(0, bt, sl, q, q.clone()),
                 lambda: eight.decode_step(0, bt, sl, q, k, k, q.clone()), lambda: eight.kv_append_rope(0, bt, sl, None, k, k, None, freq),
                 lambda: eight.decode_attention_window(0, bt, sl, q, q.clone(), window=4), lambda: eight.read_probe(0, bt, sl),
                 lambda: eight.kv_index_update(0, bt, sl, torch.zeros(eight._index_bytes, dtype=torch.uint8, device="cuda")),
                 lambda: eight.swap_out(sl, image), lambda: eight.swap_in(sl, image), lambda: eight.read_span_trace(),
                 lambda: b.Kv8Pool.kv8_append(sixteen, 0, bt, sl, k, k), lambda: b.Kv8Pool.kv8_gather(sixteen, 0, bt, sl, k, k),
                 lambda: b.Kv8Pool.kv8_attention(sixteen, 0, bt, sl, q, q.clone())):
        with pytest.raises(b.CkvError) as e:
            call()
        assert e.value.code == b.CKV_EINVAL and "bits" in str(e.value)
    assert eight.launch_count() == 0 and sixteen.launch_count() == 0
    for bad in (dict(window=-1), dict(window=3, sink=-1)):
        with pytest.raises(b.CkvError):
            eight.kv8_attention(0, bt, sl, q, q.clone(), **bad)
    with pytest.raises(b.CkvError):
        eight.kv8_attention(0, bt, sl, torch.zeros(2, 9, 8, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 9, 8, 64, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(b.CkvError):
        eight.kv8_append(0, bt, sl, k, k, q=q, q_out=q.clone())                               # queries without frequencies
    with pytest.raises(ValueError):
        eight.kv8_append(0, bt, sl, k, k, q=q, inv_freq=freq)
    with pytest.raises(ValueError):
        eight.kv8_attention(0, bt[:, :3], sl, q, q.clone())
    with pytest.raises(ValueError):
        eight.kv8_attention(0, bt, sl, q, q[:1])
    with pytest.raises(ValueError):
        eight.kv8_gather(0, bt, sl, k, k[:, :1])
    eight.close(); sixteen.close()
