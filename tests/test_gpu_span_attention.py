"""Attention whose work is cut into even spans of all contexts' tiles, over both caches: shapes that the rule sends there,
which the number of launches shows -- a kernel for the spans and one for the cut contexts, for every block of new tokens."""
import numpy as np
import pytest
import torch

import ref_step as ref
import test_gpu_cache8
import test_gpu_window
from test_gpu_attention_weights import BF16_BITS, FP16_BITS
from test_gpu_cache8 import queries, tables_for, to_dev

pytestmark = pytest.mark.gpu

KINDS = [test_gpu_cache8.Cache, test_gpu_window.Cache]
ALL = 10 ** 6


class Spans:
    """A cache with its queries; run() attends and checks the launches, check() compares with 64 bits."""

    def __init__(self, kind, layout, lens, width, q_len, seed, layers=1):
        self.lens, self.q_len = lens, q_len
        bt, n = tables_for([max(x, 0) for x in lens], width, seed)
        self.c = kind(layout, bt, n, layers=layers, layer=layers - 1, seed=seed + 1)
        self.eight = kind is test_gpu_cache8.Cache
        self.q = queries(len(lens), q_len, self.c.H, self.c.D, seed + 2)
        self.passes = -(-q_len // (8 // (self.c.H // self.c.K)))

    def run(self, window=ALL, sink=0, lens=None, stream=None):
        c = self.c
        call = c.kp.kv8_attention if self.eight else c.kp.decode_attention_window
        out = torch.full(self.q.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
        sl = torch.tensor(self.lens if lens is None else lens, dtype=torch.int32, device="cuda")
        before = c.kp.launch_count()
        call(c.layer, c.btd, sl, to_dev(self.q), out, window=window, sink=sink, stream=stream)
        assert c.kp.launch_count() - before == 2 * self.passes
        return out

    def kv(self, r, L):
        t = np.arange(L)
        if self.eight:
            return self.c.values(r, L)
        return self.c.pool[self.c.bt[r][t // 16], :, :, t % 16]

    def check(self, out, window=ALL, sink=0, only=None):
        c, G = self.c, self.c.H // self.c.K
        got = out.double().cpu().numpy()
        for r, L in enumerate(self.lens):
            if only is not None and r not in only:
                continue
            kv = self.kv(r, L)
            for h in range(c.K):
                args = (self.q[r][:, h * G:(h + 1) * G], kv[:, h, 0], kv[:, h, 1], L, window, sink)
                want, size, mass, floor = ref.attend(*args, c.v_steps(r, L, h)) if self.eight else ref.attend(*args) + (None,)
                off = np.abs(got[r][:, h * G:(h + 1) * G] - want)
                assert np.all(off <= ref.attend_tolerance(want, size, mass, FP16_BITS if self.eight else BF16_BITS, floor)), (r, h, off.max())

    def close(self):
        assert self.c.kp.check_status() == 0
        self.c.kp.close()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("layout", [(4, 1, 64), (16, 2, 128), (6, 2, 64), (5, 5, 128), (8, 1, 64)])
@pytest.mark.parametrize("q_len", [1, 3, 8])
def test_contexts_that_differ_a_thousandfold(kind, layout, q_len):
    """Under a table far wider than they are; causal masks among the new tokens, tiles of one page and of two."""
    lens = [max(n, q_len) for n in (1, 15, 16, 17, 31, 32, 33, 47, 64, 700, 5001, 1, 49)]
    s = Spans(kind, layout, lens, 6000, q_len, 1, layers=2)
    out = s.run()
    s.check(out)
    assert torch.equal(out, s.run())
    s.close()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("layout,q_len", [((4, 1, 64), 1), ((8, 1, 128), 2), ((2, 1, 64), 4), ((3, 1, 128), 5)])
@pytest.mark.parametrize("window,sink", [(27000, 0), (25003, 21), (30001, 16)])
def test_windows_and_sinks(kind, layout, q_len, window, sink):
    """Windows too long for a cluster, of contexts longer and shorter: gaps, and masks at the windows' starts and the sinks' ends."""
    s = Spans(kind, layout, [31000, 25019, 40007 if layout[0] < 8 else 300], 2600, q_len, 4)
    s.check(s.run(window, sink), window, sink)
    s.close()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("lens", [[90000], [1] * 700, [9] * 64 + [20000] + [9] * 64, [700] * 150, [1, 60000, 2, 3, 15000]])
def test_spans_of_every_kind(kind, lens):
    """One context in all spans, hundreds in one, contexts cut at every place."""
    s = Spans(kind, (2, 2, 64), lens, 6000, 1, 7)
    s.check(s.run())
    s.close()


@pytest.mark.parametrize("q_len", [1, 4])
def test_what_a_token_does_not_see_does_not_reach_it(q_len):
    """The bf16 cache: NaN in everything outside the window and the sinks, later new tokens among it."""
    window, sink = 25003, 21
    for i in range(q_len):
        s = Spans(test_gpu_window.Cache, (8, 1, 64), [31007, 26000], 2000, q_len, 10)
        c, clean = s.c, s.c.pool.copy()
        c.pool[:] = np.nan
        for r, L in enumerate(s.lens):
            p = L - q_len + i
            t = np.concatenate([np.arange(sink), np.arange(p - window + 1, p + 1)])
            c.pool[c.bt[r][t // 16], :, :, t % 16] = clean[c.bt[r][t // 16], :, :, t % 16]
        c.upload()
        out = s.run(window, sink)
        c.pool = clean
        for r, L in enumerate(s.lens):
            kv = s.kv(r, L)
            want, size, mass = ref.attend(s.q[r], kv[:, 0, 0], kv[:, 0, 1], L, window, sink)
            off = np.abs(out[r, i].double().cpu().numpy() - want[i])
            assert np.all(off <= ref.attend_tolerance(want, size, mass, BF16_BITS)[i]), (r, i)
        s.close()


def test_poisoned_blocks_reach_those_who_see_them():
    """The 8-bit cache: a block that is not finite, in the middle, at a cut and beside the window's start."""
    window, sink = 25003, 21
    s = Spans(test_gpu_cache8.Cache, (8, 1, 64), [31007, 31007, 31007, 31007], 2000, 1, 13)
    for r, page, kv in ((0, 1000, 0), (1, 100, 1), (2, (31007 - 25003) // 16, 0)):
        s.c.steps[0, s.c.bt[r, page], 0, kv] = np.nan
    s.c.kp.pool_view()[1].copy_(torch.from_numpy(s.c.steps).float())
    out = s.run(window, sink)
    assert out[0].isnan().all() and out[2].isnan().all()                 # page 100 lies between sinks and window
    s.check(out, window, sink, only=(3,))
    s.c.steps = np.nan_to_num(s.c.steps)
    s.check(out, window, sink, only=(1, 3))
    s.close()


@pytest.mark.parametrize("kind", KINDS)
def test_a_bad_page_is_flagged_and_not_followed(kind):
    s = Spans(kind, (8, 2, 128), [3000, 17, 9000], 6000, 2, 16)
    want = s.run()
    s.check(want)
    for r, page, value in ((0, 100, s.c.bt.max() + 1000), (2, 562, -1)):
        kept = s.c.btd[r, page].item()
        s.c.btd[r, page] = int(value)
        got = s.run()
        assert s.c.kp.check_status(raise_on_error=False) == s.c.b.STATUS_BAD_PAGE
        others = [i for i in range(3) if i != r]
        assert torch.equal(got[others], want[others])
        s.c.btd[r, page] = kept
    s.close()


@pytest.mark.parametrize("kind", KINDS)
def test_streams_and_replays(kind):
    """Two handles on two streams at once, captured, replayed with lengths that grow and some that are unusable."""
    cs = [Spans(kind, (8, 2, 64), [3000, 1, 500, 8000], 6000, 5, 19 + i) for i in range(2)]
    sl = torch.tensor(cs[0].lens, dtype=torch.int32, device="cuda")
    qs, outs, graphs, streams = [to_dev(s.q) for s in cs], [torch.empty(4, 5, 8, 64, dtype=torch.bfloat16, device="cuda") for _ in cs], [], []
    torch.cuda.synchronize()
    for s, q, out in zip(cs, qs, outs):
        call = s.c.kp.kv8_attention if s.eight else s.c.kp.decode_attention_window
        streams.append(torch.cuda.Stream())
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=streams[-1]):
            for _ in range(2):
                call(0, s.c.btd, sl, q, out, window=ALL)
    for lens in ([3000, 5, 500, 8000], [2990, 16, 490, 7984], [3000, 4, 0, 33]):
        sl.copy_(torch.tensor(lens, dtype=torch.int32))
        torch.cuda.synchronize()
        for g, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                g.replay()
        torch.cuda.synchronize()
        for s, out in zip(cs, outs):
            s.lens = lens
            good = [r for r, n in enumerate(lens) if n >= 5]
            # two requests share no page, but a table of one page holds positions 0 .. 15 alone
            s.check(out, only=[r for r in good if ref.pages(lens[r]) <= (s.c.bt[r] >= 0).sum()])
            assert not out[[r for r in range(4) if lens[r] < 5]].any()
            assert s.c.kp.check_status(raise_on_error=False) == (0 if len(good) == 4 else s.c.b.STATUS_BAD_LENGTH)
    del graphs
    for s in cs:
        s.close()
