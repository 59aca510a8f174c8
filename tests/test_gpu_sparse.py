"""Key bounds, page selection and page-sparse attention against their definitions in 64 bits: bounds and
chosen pages exactly, attention within the tolerance of the whole-context kernel."""
import numpy as np
import pytest
import torch

from paper_2501_08090_b200 import workloads as wl

import ref_ops
from helpers import assert_close, bits_to_dev, dev_to_bits, widen

pytestmark = pytest.mark.gpu


class Case:
    """A pool whose pages differ (some keys large, some tiny, unused slots NaN), its index and a batch."""

    def __init__(self, lens, Hq, Hkv, d, seed, width=None, distinct=None, spare=3, layers=1):
        from paper_2501_08090_b200 import binding as b
        self.b, self.Hq, self.Hkv, self.d = b, Hq, Hkv, d
        self.lens = np.asarray(lens, dtype=np.int32)
        pages = int(wl.pages_of(np.maximum(self.lens, 0)).sum()) + spare
        self.bt = wl.block_tables(np.maximum(self.lens, 1), pages + len(lens), seed, max_pages_per_req=width)
        pages += len(lens)
        rng = np.random.default_rng([seed, 77])
        pool = rng.standard_normal((pages, Hkv, 2, 16, d))
        pool[:, :, 0] += rng.standard_normal((pages, Hkv, 1, d)) * rng.choice([0.1, 1.0], size=(pages, Hkv, 1, 1))
        pool[:, :, 0] *= 2.0 ** rng.integers(-3, 4, size=(pages, Hkv, 1, 1))
        if distinct is not None:                                     # few different pages: scores tie
            pool = pool[rng.integers(0, distinct, size=pages)]
        self.pool = torch.from_numpy(pool).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)
        for r, L in enumerate(self.lens):
            if L > 0 and L % 16:
                self.pool[self.bt[r][L // 16], :, :, L % 16:] = 0x7fc0        # slots behind the context
        cfg = b.make_config(layers, Hq, Hkv, d, pages, self.bt.shape[1], len(lens))
        stack = np.concatenate([np.zeros_like(self.pool)] * (layers - 1) + [self.pool])
        self.layer = layers - 1
        self.kp = b.KvPool(cfg, pool=bits_to_dev(stack.reshape(-1)))
        self.btd, self.sld = torch.from_numpy(self.bt).cuda(), torch.from_numpy(self.lens).cuda()
        self.index = self.kp.make_index()
        q = rng.standard_normal((len(lens), Hq, d)) * rng.choice([0.05, 1.0, 3.0], size=(len(lens), Hq, 1))
        self.q = torch.from_numpy(q).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)
        self.qd = bits_to_dev(self.q)

    def update(self, last_tokens=0):
        self.kp.kv_index_update(self.layer, self.btd, self.sld, self.index, last_tokens=last_tokens)

    def host_index(self, index=None):
        """(records int8 [pages][Hkv][2][d], steps [pages][Hkv]) of the case's layer."""
        raw = (self.index if index is None else index).cpu().numpy()
        c = self.kp.cfg
        n = c.num_layers * c.num_pages * c.num_kv_heads
        rec = raw[:n * 2 * self.d].view(np.int8).reshape(c.num_layers, c.num_pages, c.num_kv_heads, 2, self.d)
        step = raw[n * 2 * self.d:].view(np.float32).reshape(c.num_layers, c.num_pages, c.num_kv_heads)
        return rec[self.layer], step[self.layer]

    def out(self, budget):
        B = len(self.lens)
        return (torch.full((B, self.Hkv, budget), -7, dtype=torch.int32, device="cuda"),
                torch.full((B,), -7, dtype=torch.int32, device="cuda"),
                torch.full((B, self.Hq, self.d), float("nan"), dtype=torch.bfloat16, device="cuda"))

    def check(self, budget, sink, recent, requests=None):
        """Selection exactly, lengths, and attention of every usable request."""
        pages, lens, out = self.out(budget)
        self.kp.decode_attention_sparse(self.layer, self.btd, self.sld, self.qd, self.index, pages, lens, out, sink=sink, recent=recent)
        # the two halves of the call give the same lists and the same bits
        pages2, lens2, out2 = self.out(budget)
        self.kp.decode_select_pages(self.layer, self.btd, self.sld, self.qd, self.index, pages2, lens2, sink=sink, recent=recent)
        self.kp.decode_attention_pages(self.layer, pages2, lens2, self.qd, out2)
        assert self.kp.check_status() == 0
        assert torch.equal(pages, pages2) and torch.equal(lens, lens2) and torch.equal(out, out2)
        pages, lens = pages.cpu().numpy(), lens.cpu().numpy()
        rec, step = self.host_index()
        pool, q = widen(self.pool), widen(self.q)
        G = self.Hq // self.Hkv
        for r in (range(len(self.lens)) if requests is None else requests):
            L = int(self.lens[r])
            n = -(-L // 16)
            index = {(int(p), h): (rec[p, h, 0].astype(int), rec[p, h, 1].astype(int), float(step[p, h]))
                     for p in self.bt[r][:n] for h in range(self.Hkv)}
            for h in range(self.Hkv):
                want = ref_ops.select(index, self.bt[r], L, q[r, h * G:(h + 1) * G], h, budget, sink, recent)
                assert pages[r, h].tolist() == want + [-1] * (budget - len(want)), (r, h)
                assert lens[r] == L - (n - len(want)) * 16
                ref = ref_ops.attend(pool, want, int(lens[r]), q[r, h * G:(h + 1) * G], h)
                assert_close(dev_to_bits(out[r, h * G:(h + 1) * G]), ref, "request %d kv head %d" % (r, h))

    def close(self):
        self.kp.close()


LAYOUTS = [(32, 8, 128), (8, 1, 128), (4, 1, 64), (12, 4, 64), (6, 6, 128), (35, 5, 128), (1, 1, 64), (16, 2, 64)]


@pytest.mark.parametrize("Hq,Hkv,d", LAYOUTS)
def test_bounds_of_every_page(Hq, Hkv, d):
    c = Case([1, 15, 16, 17, 100, 333, 48], Hq, Hkv, d, seed=Hq + d, layers=2)
    c.update()
    assert c.kp.check_status() == 0
    rec, step = c.host_index()
    want = ref_ops.index_of(widen(c.pool), c.bt, c.lens)
    for (page, h), (lo, hi, st) in want.items():
        assert np.array_equal(rec[page, h, 0], lo) and np.array_equal(rec[page, h, 1], hi) and step[page, h] == st, (page, h)
    touched = np.array(sorted({p for p, _ in want}))
    rest = np.setdiff1d(np.arange(rec.shape[0]), touched)
    assert not rec[rest].any() and not step[rest].any()              # pages of no request stay as they were
    values = torch.empty(c.kp.cfg.num_pages, Hkv, 2, d, dtype=torch.bfloat16, device="cuda")
    c.kp.kv_index_values(c.layer, c.index, values)
    assert np.array_equal(values.double().cpu().numpy(), rec * step[:, :, None, None].astype(np.float64))
    c.kp.kv_index_values(0, c.index, values)
    assert not values.any()
    c.close()


@pytest.mark.parametrize("last", [1, 2, 16, 17, 40, 10 ** 6])
def test_update_of_the_last_tokens_touches_their_pages_alone(last):
    c = Case([1, 16, 17, 32, 33, 200], 8, 2, 64, seed=last % 1000)
    c.index.fill_(0x55)
    c.update(last_tokens=last)
    rec, step = c.host_index()
    want = ref_ops.index_of(widen(c.pool), c.bt, c.lens, last)
    blank = np.frombuffer(b"\x55\x55\x55\x55", dtype=np.float32)[0]
    for page in range(rec.shape[0]):
        for h in range(2):
            if (page, h) in want:
                lo, hi, st = want[page, h]
                assert np.array_equal(rec[page, h], [lo, hi]) and step[page, h] == st
            else:
                assert np.all(rec[page, h] == 0x55) and step[page, h] == blank
    c.close()


def test_bounds_at_the_ends_of_the_range():
    """Zero pages, tiny and huge keys, a magnitude that needs the doubled step, infinities and NaN."""
    c = Case([16 * 9], 2, 1, 64, seed=4)
    keys = np.zeros((9, 16, 64))
    keys[1, 3, 5] = -2.0 ** -133                                     # the smallest bf16
    keys[2] = 1.5 * 2.0 ** 127
    keys[3, 0, 0] = 127.5                                            # 127.5 steps of 1: the step doubles
    keys[4, 0, 0], keys[4, 1, 0] = -127.5, 127.0
    keys[5, 7, 63] = 2.0 ** -100
    keys[6, 7, 1] = 3.3895313892515355e38                            # the largest bf16
    bits = torch.from_numpy(keys).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16).copy()
    bits[7, 5, 9], bits[8, 2, 3] = 0xff80, 0x7fc3
    for i, page in enumerate(c.bt[0]):
        c.pool[page, 0, 0] = bits[i]
    c.kp.pool.copy_(bits_to_dev(c.pool.reshape(-1)))
    c.update()
    rec, step = c.host_index()
    for (page, h), (lo, hi, st) in ref_ops.index_of(widen(c.pool), c.bt, c.lens).items():
        assert np.array_equal(rec[page, h], [lo, hi]) and step[page, h] == st, list(c.bt[0]).index(page)
    assert rec[c.bt[0][8], 0].tolist() == [[-127] * 64, [127] * 64] and step[c.bt[0][7], 0] == 2.0 ** 121
    c.close()


def test_bounds_balance_over_very_uneven_requests():
    lens = [1] * 40 + [7001] + [1] * 40 + [33]
    c = Case(lens, 2, 2, 64, seed=5)
    c.update()
    rec, step = c.host_index()
    for (page, h), (lo, hi, st) in ref_ops.index_of(widen(c.pool), c.bt, c.lens).items():
        assert np.array_equal(rec[page, h], [lo, hi]) and step[page, h] == st
    c.close()


@pytest.mark.parametrize("Hq,Hkv,d", LAYOUTS)
@pytest.mark.parametrize("budget,sink,recent", [(6, 1, 2), (9, 0, 1), (4, 2, 2), (40, 3, 5), (1, 0, 1)])
@pytest.mark.parametrize("width", [None, 300, 5000])                       # one kernel scores and selects, or two
def test_selection_and_attention(Hq, Hkv, d, budget, sink, recent, width):
    c = Case([1, 16 * budget, 16 * budget + 1, 17, 1000, 333, 16 * 70], Hq, Hkv, d, seed=Hq * 7 + d + budget, width=width)
    c.update()
    c.check(budget, sink, recent)
    c.close()


@pytest.mark.parametrize("distinct", [1, 2, 5])
@pytest.mark.parametrize("width", [None, 260, 4200, 9000])
def test_equal_scores_go_to_the_earlier_page(distinct, width):
    c = Case([1600, 3217, 48], 8, 2, 128, seed=distinct, distinct=distinct, width=width)
    c.update()
    c.check(17, 1, 2)
    c.close()


def test_one_long_context():
    """8192 and 11004 pages of one request; also with nearly all and with hardly any taken."""
    for length in (131072 - 5, 16 * 11003 + 9):
        c = Case([length], 8, 2, 64, seed=6)
        c.update()
        for budget, sink, recent in ((128, 1, 2), (-(-length // 16) - 1, 4, 4), (3, 1, 1)):
            c.check(budget, sink, recent)
        c.close()


@pytest.mark.parametrize("Hq,Hkv,d", [(4, 4, 64), (8, 4, 128), (28, 4, 128), (16, 2, 64)])
def test_many_requests(Hq, Hkv, d):
    """More (request, kv head) pairs than CTAs fit the GPU at a time."""
    rng = np.random.default_rng(8)
    c = Case(rng.integers(1, 900, size=150), Hq, Hkv, d, seed=7)
    c.update()
    c.check(12, 1, 3, requests=range(0, 150, 11))
    c.close()


@pytest.mark.parametrize("seed", [0, 1])
def test_more_requests_than_a_block_has_threads(seed):
    """The work is cut over the sums of all requests, in several turns of a block's threads."""
    rng = np.random.default_rng(seed)
    lens = np.where(rng.random(700) < 0.4, 1, rng.integers(1, 700, size=700))
    lens[[0, 191, 192, 255, 256, 383, 384, 699]] = 640
    c = Case(lens, 2, 1, 64, seed=20 + seed, width=80)
    c.update()
    rec, step = c.host_index()
    for (page, h), (lo, hi, st) in ref_ops.index_of(widen(c.pool), c.bt, c.lens).items():
        assert np.array_equal(rec[page, h], [lo, hi]) and step[page, h] == st
    c.check(9, 1, 2, requests=[0, 191, 192, 255, 256, 383, 384, 699] + list(range(5, 700, 41)))
    c.close()


@pytest.mark.parametrize("Hq,Hkv,d", [(4, 1, 64), (32, 8, 128), (14, 2, 128)])
@pytest.mark.parametrize("budget", [1, 2, 11, 12, 13, 25, 33, 64, 127, 200, 229])
def test_few_pairs_of_every_list_length(Hq, Hkv, d, budget):
    """One request alone: from one CTA to a cluster of 16 a pair, one tile a warp and more."""
    c = Case([16 * 230 + 3], Hq, Hkv, d, seed=budget)
    c.update()
    c.check(budget, 0, 1)
    for tokens in {1, 16 * budget, 16 * budget - 15, max(1, 8 * budget)}:
        lists = torch.from_numpy(np.stack([c.bt[:, 1:1 + budget]] * Hkv, 1)).cuda()
        out = c.out(budget)[2]
        c.kp.decode_attention_pages(0, lists, torch.tensor([tokens], dtype=torch.int32, device="cuda"), c.qd, out)
        assert c.kp.check_status() == 0
        pool, q = widen(c.pool), widen(c.q)
        for h in range(Hkv):
            G = Hq // Hkv
            ref = ref_ops.attend(pool, [int(x) for x in c.bt[0][1:1 + budget]], tokens, q[0, h * G:h * G + G], h)
            assert_close(dev_to_bits(out[0, h * G:h * G + G]), ref, "tokens %d kv head %d" % (tokens, h))
    c.close()


def test_queries_out_of_range():
    """Zero queries, infinities, NaN, the extremes of bf16: the selection is the definition's; a NaN or an
    infinity only reaches its own head's output."""
    c = Case([900, 900], 8, 2, 64, seed=9)
    c.q[0, 0] = 0
    c.q[0, 1, 3], c.q[0, 2, 5], c.q[0, 3, :] = 0x7f80, 0x7fc0, 0x7f7f
    c.q[1, 4, :] = 0x0001
    c.qd = bits_to_dev(c.q)
    c.update()
    pages, lens, out = c.out(10)
    c.kp.decode_attention_sparse(0, c.btd, c.sld, c.qd, c.index, pages, lens, out, sink=1, recent=2)
    rec, step = c.host_index()
    q, got = widen(c.q), out.float().cpu().numpy()
    for r in range(2):
        index = {(int(p), h): (rec[p, h, 0].astype(int), rec[p, h, 1].astype(int), float(step[p, h])) for p in c.bt[r] for h in range(2)}
        for h in range(2):
            assert pages[r, h].tolist() == ref_ops.select(index, c.bt[r], 900, q[r, h * 4:h * 4 + 4], h, 10, 1, 2)
    assert np.isfinite(got[1]).all() and np.isfinite(got[0, [0, 4, 5, 6, 7]]).all()
    c.close()


def test_unusable_lengths_and_bad_pages():
    c = Case([500, 500, 500, 500], 4, 2, 64, seed=10)
    c.update()
    lens = torch.tensor([500, 0, -3, 10 ** 6], dtype=torch.int32)
    c.sld.copy_(lens)
    pages, got_lens, out = c.out(8)
    c.kp.decode_attention_sparse(0, c.btd, c.sld, c.qd, c.index, pages, got_lens, out)
    assert c.kp.check_status(raise_on_error=False) == c.b.STATUS_BAD_LENGTH
    assert got_lens.tolist()[1:] == [0, 0, 0] and not out[1:].any() and (pages[1:] == -1).all() and out[0].all()
    before = c.index.clone()
    c.kp.kv_index_update(0, c.btd, c.sld, c.index)
    assert c.kp.check_status(raise_on_error=False) == c.b.STATUS_BAD_LENGTH
    assert torch.equal(before, c.index)
    c.sld.fill_(500)
    c.btd[2, 7] = 10 ** 7
    c.btd[3, 0] = -1
    c.kp.decode_select_pages(0, c.btd, c.sld, c.qd, c.index, pages, got_lens, sink=0, recent=1)
    assert c.kp.check_status(raise_on_error=False) == c.b.STATUS_BAD_PAGE
    assert torch.equal(pages[0].sort()[0] >= 0, torch.ones(2, 8, dtype=torch.bool, device="cuda"))
    c.kp.kv_index_update(0, c.btd, c.sld, c.index)
    assert c.kp.check_status(raise_on_error=False) == c.b.STATUS_BAD_PAGE
    c.close()


def test_attention_over_lists_of_the_callers_own():
    """Any list of pages works, head by head; a list may follow the kernel that writes it."""
    c = Case([700, 90, 300], 8, 2, 128, seed=11)
    rng = np.random.default_rng(1)
    budget = 13
    lists = np.full((3, 2, budget), -1, dtype=np.int32)
    tokens = np.array([16 * 12 + 5, 90, 16 * 4], dtype=np.int32)
    for r, n in enumerate((13, 6, 4)):
        for h in range(2):
            full = c.bt[r][:int(c.lens[r]) // 16]
            lists[r, h, :n] = rng.choice(full, n, replace=False) if r != 1 else c.bt[r][:6]
    lists_d = torch.full((3, 2, budget), -1, dtype=torch.int32, device="cuda")
    lens_d = torch.zeros(3, dtype=torch.int32, device="cuda")
    out = c.out(budget)[2]
    src, src_lens = torch.from_numpy(lists).cuda(), torch.from_numpy(tokens).cuda()
    for _ in range(3):
        lists_d.fill_(-1); lens_d.zero_(); out.fill_(float("nan"))
        lists_d.copy_(src)
        lens_d.add_(src_lens)                                            # written by the kernel just before
        c.kp.decode_attention_pages(0, lists_d, lens_d, c.qd, out)
        assert c.kp.check_status() == 0
        pool, q = widen(c.pool), widen(c.q)
        for r in range(3):
            for h in range(2):
                live = [int(x) for x in lists[r, h] if x >= 0]
                ref = ref_ops.attend(pool, live, int(tokens[r]), q[r, 4 * h:4 * h + 4], h)
                assert_close(dev_to_bits(out[r, 4 * h:4 * h + 4]), ref, "request %d head %d" % (r, h))
    c.close()


def test_requests_that_share_full_pages():
    """A common prefix: the shared pages' bounds are written twice, with the same bits."""
    c = Case([700, 700, 900], 8, 2, 64, seed=19)
    c.bt[1][:30] = c.bt[0][:30]
    c.bt[2][:43] = c.bt[0][:43]
    c.btd.copy_(torch.from_numpy(c.bt))
    c.update()
    rec, step = c.host_index()
    for (page, h), (lo, hi, st) in ref_ops.index_of(widen(c.pool), c.bt, c.lens).items():
        assert np.array_equal(rec[page, h], [lo, hi]) and step[page, h] == st
    c.check(9, 1, 2)
    c.close()


def test_two_handles_on_two_streams():
    """Calls on two handles at once, of different kinds and sizes, do not touch each other's work."""
    cases = [Case([3000, 517, 90, 2048] * 10, 8, 2, 128, seed=23, width=400), Case([1500, 33], 4, 1, 64, seed=24)]
    streams, want, bufs = [torch.cuda.Stream(), torch.cuda.Stream()], [], []
    for c in cases:
        c.update()
        bufs.append(c.out(20))
        c.kp.decode_attention_sparse(0, c.btd, c.sld, c.qd, c.index, *bufs[-1])
        want.append([t.clone() for t in bufs[-1]])
    torch.cuda.synchronize()
    for _ in range(60):
        for c, s, b in zip(cases, streams, bufs):
            c.kp.kv_index_update(0, c.btd, c.sld, c.index, stream=s)
            c.kp.decode_attention_sparse(0, c.btd, c.sld, c.qd, c.index, *b, stream=s)
    torch.cuda.synchronize()
    for c, w, b in zip(cases, want, bufs):
        assert all(torch.equal(x, y) for x, y in zip(w, b))
        assert c.kp.check_status() == 0
        c.close()


def test_the_widest_table():
    c = Case([3000, 17], 4, 1, 64, seed=25, width=49152)
    c.update()
    c.check(9, 1, 2)
    c.close()


def test_lists_longer_than_their_rows_are_flagged():
    c = Case([700, 90], 8, 2, 128, seed=15)
    pages, lens, out = c.out(4)
    pages.copy_(torch.from_numpy(np.stack([c.bt[:, :4]] * 2, 1)).cuda())
    lens.copy_(torch.tensor([65, 64], dtype=torch.int32))                  # 4 pages hold 64 tokens
    c.kp.decode_attention_pages(0, pages, lens, c.qd, out)
    assert c.kp.check_status(raise_on_error=False) == c.b.STATUS_BAD_LENGTH
    assert not out[0].any() and out[1].all()
    c.close()


def test_layers_have_their_own_pages_and_bounds():
    c = Case([1000, 333], 8, 2, 128, seed=16, layers=3)
    c.update()
    c.check(9, 1, 2)
    c.close()


@pytest.mark.parametrize("width", [None, 600])
def test_plain_stream_order(width):
    """With kernel overlap off, and with inputs that the kernel just before writes, results are the same."""
    c = Case([3000, 517, 90, 2048], 32, 8, 128, seed=17, width=width)
    c.update()
    pages, lens, out = c.out(20)
    c.kp.decode_attention_sparse(0, c.btd, c.sld, c.qd, c.index, pages, lens, out)
    want = [t.clone() for t in (pages, lens, out)]
    q, sl, bt = torch.empty_like(c.qd), torch.empty_like(c.sld), torch.empty_like(c.btd)
    for overlap in (False, True):
        c.kp.set_overlap(overlap)
        for order in range(3):
            for _ in range(30):
                q.zero_(); sl.fill_(1); bt.fill_(0)
                moves = [lambda: q.copy_(c.qd), lambda: sl.copy_(c.sld), lambda: bt.copy_(c.btd)]
                for k in range(3):
                    moves[(order + k) % 3]()
                c.kp.decode_attention_sparse(0, bt, sl, q, c.index, pages, lens, out)
            assert all(torch.equal(a, b) for a, b in zip(want, (pages, lens, out)))
    assert c.kp.check_status() == 0
    c.close()


def test_contexts_wider_than_the_registers_hold():
    """Tables of more than 16384 pages select from shared memory: ties, few and nearly all pages."""
    c = Case([300007, 262144 + 16 * 700], 2, 1, 64, seed=18, distinct=300)
    c.update()
    for budget, sink, recent in ((64, 1, 2), (17000, 5, 7)):
        c.check(budget, sink, recent, requests=[0, 1])
    c.close()


@pytest.mark.parametrize("batch", [1, 40])
def test_a_budget_beyond_the_context_is_whole_attention(batch):
    c = Case([700, 33, 1] * batch, 8, 2, 128, seed=12)
    c.update()
    pages, lens, out = c.out(64)
    c.kp.decode_attention_sparse(0, c.btd, c.sld, c.qd, c.index, pages, lens, out)
    assert lens.tolist() == [700, 33, 1] * batch
    pool, q = widen(c.pool), widen(c.q)
    for r in range(0, 3 * batch, 1 + 2 * (batch > 1)):
        L = int(c.lens[r])
        for h in range(2):
            ref = ref_ops.attend(pool, [int(x) for x in c.bt[r][:-(-L // 16)]], L, q[r, 4 * h:4 * h + 4], h)
            assert_close(dev_to_bits(out[r, 4 * h:4 * h + 4]), ref, "request %d head %d" % (r, h))
    c.close()


@pytest.mark.parametrize("width", [None, 600])
def test_streams_graphs_and_repetition(width):
    """The same bits eagerly, on another stream, captured and replayed after the inputs changed and back."""
    c = Case([3000, 517, 90, 2048], 32, 8, 128, seed=13, width=width)
    c.update()
    pages, lens, out = c.out(20)
    args = (0, c.btd, c.sld, c.qd, c.index, pages, lens, out)
    c.kp.decode_attention_sparse(*args)
    want = [t.clone() for t in (pages, lens, out)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out.zero_()
    torch.cuda.synchronize()
    c.kp.decode_attention_sparse(*args, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (pages, lens, out)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.kp.kv_index_update(0, c.btd, c.sld, c.index, last_tokens=4)
        c.kp.decode_attention_sparse(*args)
    keep = c.qd.clone()
    c.qd.neg_()
    graph.replay()
    assert not torch.equal(want[2], out)
    c.qd.copy_(keep)
    for _ in range(50):
        graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(want, (pages, lens, out)))
    assert c.kp.check_status() == 0
    del graph
    c.close()


def test_refusals():
    c = Case([100, 100], 8, 2, 64, seed=14)
    b, kp = c.b, c.kp
    pages, lens, out = c.out(8)
    n0 = kp.launch_count()
    for sink, recent in ((-1, 1), (0, 0), (7, 2), (8, 1)):
        for call in (lambda: kp.decode_select_pages(0, c.btd, c.sld, c.qd, c.index, pages, lens, sink=sink, recent=recent),
                     lambda: kp.decode_attention_sparse(0, c.btd, c.sld, c.qd, c.index, pages, lens, out, sink=sink, recent=recent)):
            with pytest.raises(b.CkvError) as e:
                call()
            assert e.value.code == b.CKV_EINVAL and "budget" in str(e.value)
    with pytest.raises(ValueError):
        kp.decode_attention_sparse(0, c.btd, c.sld, c.qd, c.index[:-4], pages, lens, out)
    with pytest.raises(ValueError):
        kp.decode_attention_sparse(0, c.btd, c.sld, c.qd.float(), c.index, pages, lens, out)
    with pytest.raises(ValueError):
        kp.decode_attention_sparse(0, c.btd, c.sld, c.qd, c.index, pages[:, :1], lens, out)
    with pytest.raises(ValueError):
        kp.decode_attention_pages(0, pages, lens, c.qd[:1], out)
    with pytest.raises(b.CkvError):
        kp.kv_index_update(3, c.btd, c.sld, c.index)
    with pytest.raises(b.CkvError):
        kp.kv_index_update(0, c.btd, c.sld, c.index, last_tokens=-1)
    rc = b.lib.kv_index_update(kp._h, 0, 2, c.btd.data_ptr(), c.sld.data_ptr(), 0, c.index.data_ptr(), c.index.numel() - 1, None)
    assert rc == b.CKV_ENOMEM
    rc = b.lib.kv_index_update(kp._h, 0, 2, c.btd.data_ptr(), c.sld.data_ptr(), 0, c.index.data_ptr() + 4, c.index.numel(), None)
    assert rc == b.CKV_EINVAL and "aligned" in b.last_error()
    assert kp.launch_count() == n0
    c.close()
    cfg = b.make_config(1, 4, 1, 64, 8, 49153, 1)
    kp = b.KvPool(cfg)
    bt = torch.zeros(1, 49153, dtype=torch.int32, device="cuda")
    with pytest.raises(b.CkvError) as e:
        kp.decode_select_pages(0, bt, torch.ones(1, dtype=torch.int32, device="cuda"), torch.zeros(1, 4, 64, dtype=torch.bfloat16, device="cuda"),
                               kp.make_index(), pages[:1, :1].contiguous(), lens[:1].contiguous())
    assert "49152" in str(e.value)
    kp.close()
