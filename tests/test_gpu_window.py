"""Sliding windows with sinks over the bf16 cache against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import ref_step as ref
from test_gpu_cache8 import LAYOUTS, bf16, queries, tables_for, to_dev

pytestmark = pytest.mark.gpu


class Cache:
    def __init__(self, layout, bt, num_pages, layers=1, layer=0, seed=0):
        from paper_2501_08090_b200 import binding as b
        self.b, self.layer, self.bt = b, layer, bt
        self.H, self.K, self.D = layout
        self.kp = b.KvPool(b.make_config(layers, self.H, self.K, self.D, num_pages, bt.shape[1], bt.shape[0]))
        self.pool = bf16(np.random.default_rng(seed).standard_normal((num_pages, self.K, 2, 16, self.D)))
        self.btd = torch.from_numpy(bt).cuda()
        self.upload()

    def upload(self):
        self.kp.pool.fill_(float("nan"))
        self.kp.pool_view()[self.layer].copy_(torch.from_numpy(self.pool))

    def run(self, lens, q, window, sink, stream=None):
        out = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
        self.kp.decode_attention_window(self.layer, self.btd, torch.tensor(lens, dtype=torch.int32, device="cuda"), to_dev(q), out, window=window,
                                        sink=sink, stream=stream)
        return out

    def check(self, lens, q, out, window, sink):
        G = self.H // self.K
        got = out.double().cpu().numpy()
        for r, L in enumerate(lens):
            t = np.arange(L)
            kv = self.pool[self.bt[r][t // 16], :, :, t % 16]
            for h in range(self.K):
                want, size, mass = ref.attend(q[r][:, h * G:(h + 1) * G], kv[:, h, 0], kv[:, h, 1], L, window, sink)
                off = np.abs(got[r][:, h * G:(h + 1) * G] - want)
                assert np.all(off <= ref.attend_tolerance(want, size, mass, 8)), (r, h, window, sink, np.nanmax(off))


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("q_len", [1, 3, 8])
def test_windows_and_sinks(layout, q_len):
    lens = [max(n, q_len) for n in (1, 15, 16, 17, 31, 32, 33, 100, 257, 700)]
    bt, n = tables_for(lens, 44, 1)
    c = Cache(layout, bt, n, layers=2, layer=1, seed=2)
    q = queries(len(lens), q_len, c.H, c.D, 3)
    for window, sink in ((1, 0), (1, 1), (2, 40), (16, 0), (17, 16), (33, 17), (250, 4), (10 ** 6, 3), (2 ** 31 - 1, 2 ** 31 - 1), (5, 2 ** 31 - 1)):
        c.check(lens, q, c.run(lens, q, window, sink), window, sink)
    assert c.kp.check_status() == 0
    c.kp.close()


@pytest.mark.parametrize("lens,window,sink", [([30000], 4000, 4), ([5] * 200 + [8000] * 3, 2000, 0), ([4096] * 20, 128, 16), ([1], 1, 0)])
def test_however_the_work_is_cut(lens, window, sink):
    bt, n = tables_for(lens, ref.pages(max(lens)), 4)
    c = Cache((8, 2, 128), bt, n, seed=5)
    q = queries(len(lens), 1, 8, 128, 6)
    a, b = c.run(lens, q, window, sink), c.run(lens, q, window, sink)
    assert torch.equal(a, b)
    c.check(lens, q, a, window, sink)
    c.kp.close()


@pytest.mark.parametrize("batch", [1, 2, 3, 5, 9, 18, 36])
@pytest.mark.parametrize("layout,window,q_len", [((32, 8, 128), 1500, 1), ((16, 8, 64), 700, 6)])
def test_few_requests_and_many(batch, layout, window, q_len):
    """Pairs of one length from as many CTAs as fit to one each; an unusable length among them."""
    lens = [window // 2 + (577 * r) % (2 * window) for r in range(batch)]
    bt, n = tables_for(lens, ref.pages(3 * window), 13)
    c = Cache(layout, bt, n, seed=14)
    q = queries(batch, q_len, c.H, c.D, 15)
    out = c.run(lens, q, window, 20)
    c.check(lens, q, out, window, 20)
    assert c.kp.check_status() == 0
    if batch > 2:
        again = c.run(lens[:1] + [q_len - 1] + lens[2:], q, window, 20)
        assert not again[1].any() and torch.equal(again[0], out[0]) and torch.equal(again[2:], out[2:])
        assert c.kp.check_status(raise_on_error=False) == 1
    c.kp.close()


@pytest.mark.parametrize("q_len", [1, 4])
@pytest.mark.parametrize("what", [np.nan, np.inf, -np.inf])
def test_what_a_token_does_not_see_does_not_reach_it(q_len, what):
    """Everything outside the windows and the sinks, later new tokens among it, holds NaN or infinities."""
    lens = [q_len, 20, 77, 130]
    bt, n = tables_for(lens, 9, 7)
    for window, sink in ((1, 0), (7, 3), (16, 16), (40, 18)):
        for i in range(q_len):                              # checked for new token i: only what it sees is finite
            c = Cache((8, 2, 64), bt, n, seed=8)
            clean, q = c.pool.copy(), queries(len(lens), q_len, 8, 64, 9)
            c.pool[:] = what
            for r, L in enumerate(lens):
                p = L - q_len + i
                t = np.array([x for x in range(p + 1) if x > p - window or x < sink])
                c.pool[bt[r][t // 16], :, :, t % 16] = clean[bt[r][t // 16], :, :, t % 16]
            c.upload()
            got = c.run(lens, q, window, sink).double().cpu().numpy()
            for r, L in enumerate(lens):
                t = np.arange(L)
                kv = clean[bt[r][t // 16], :, :, t % 16]
                for h in range(2):
                    want, size, mass = ref.attend(q[r][:, h * 4:h * 4 + 4], kv[:, h, 0], kv[:, h, 1], L, window, sink)
                    off = np.abs(got[r, i, h * 4:h * 4 + 4] - want[i])
                    assert np.all(off <= ref.attend_tolerance(want, size, mass, 8)[i]), (r, h, i, window, sink)
            c.kp.close()


def test_infinite_keys_weigh_nothing_and_a_window_of_them_is_nan():
    """As decode_attention: a score of minus infinity weighs 0; a row of nothing else is NaN."""
    lens = [100, 100]
    bt, n = tables_for(lens, 7, 10)
    c = Cache((4, 1, 64), bt, n, seed=11)
    q = np.abs(queries(2, 1, 4, 64, 12)) + 0.125
    for t in (99, 98, 60):
        c.pool[bt[0][t // 16], 0, 0, t % 16, 5] = -np.inf
    for t in range(90, 100):
        c.pool[bt[1][t // 16], 0, 0, t % 16, 5] = -np.inf
    c.upload()
    got = c.run(lens, q, 10, 0)
    t = np.arange(90, 98)
    kv = c.pool[bt[0][t // 16], 0, :, t % 16]
    want, size, mass = ref.attend(q[0], kv[:, 0], kv[:, 1], 8, 0, 0)
    assert np.all(np.abs(got[0].double().cpu().numpy() - want) <= ref.attend_tolerance(want, size, mass, 8))
    assert torch.isnan(got[1].float()).all()
    c.kp.close()


def test_pages_that_nobody_sees_are_not_read():
    """Their table entries may be anything; a bad entry among those read is flagged."""
    lens = [500, 321]
    bt, n = tables_for(lens, 40, 13)
    c = Cache((8, 2, 128), bt, n, seed=14)
    q = queries(2, 1, 8, 128, 15)
    want = c.run(lens, q, 50, 20)
    seen = {0, 1} | set(range((499 - 49) // 16, 32)), {0, 1} | set(range((320 - 49) // 16, 21))
    for r in range(2):
        for i in range(40):
            if i not in seen[r]:
                c.btd[r, i] = 10 ** 9
    assert torch.equal(c.run(lens, q, 50, 20), want) and c.kp.check_status() == 0
    c.btd[1, 1] = -1
    got = c.run(lens, q, 50, 20)
    assert torch.equal(got[0], want[0]) and c.kp.check_status(raise_on_error=False) == c.b.STATUS_BAD_PAGE
    c.kp.close()


def test_unusable_lengths_give_zeros():
    lens = [50, 2, 0, 641, 30]
    bt, n = tables_for([50, 2, 0, 0, 30], 40, 16)
    c = Cache((8, 2, 64), bt, n, seed=17)
    q = queries(5, 3, 8, 64, 18)
    out = c.run(lens, q, 9, 1)                               # 2: fewer than its three new tokens
    assert c.kp.check_status(raise_on_error=False) == c.b.STATUS_BAD_LENGTH
    assert not out[1:4].any()
    for r in (0, 4):
        c.bt, keep = bt[r:r + 1], c.bt
        c.check([lens[r]], q[r:r + 1], out[r:r + 1], 9, 1)
        c.bt = keep
    c.kp.close()


def test_streams_graphs_and_two_handles_at_once():
    """Two handles on two streams, captured and replayed with lengths that grow between replays."""
    lens = [300, 40]
    bt, n = tables_for([400, 140], 25, 19)
    cs = [Cache((8, 2, 128), bt, n, seed=20 + i) for i in range(2)]
    q = queries(2, 1, 8, 128, 22)
    streams = [torch.cuda.Stream() for _ in cs]
    sl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    qd, outs, graphs = to_dev(q), [torch.empty(2, 1, 8, 128, dtype=torch.bfloat16, device="cuda") for _ in cs], []
    torch.cuda.synchronize()
    for c, s, out in zip(cs, streams, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            for _ in range(3):
                c.kp.decode_attention_window(0, c.btd, sl, qd, out, window=64, sink=2)
        graphs.append(g)
    for step in range(0, 100, 33):
        sl.copy_(torch.tensor([x + step for x in lens], dtype=torch.int32))
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for c, out in zip(cs, outs):
            c.check([x + step for x in lens], q, out, 64, 2)
    for c in cs:
        assert c.kp.check_status() == 0
        c.kp.close()


def test_beside_the_other_attention_calls_on_one_handle():
    """A window as long as the context is decode_attention; the calls share a workspace in stream order."""
    lens = [777, 30, 129]
    bt, n = tables_for(lens, 49, 23)
    c = Cache((32, 8, 128), bt, n, seed=24)
    q = queries(3, 1, 32, 128, 25)
    sl, qd = torch.tensor(lens, dtype=torch.int32, device="cuda"), to_dev(q[:, 0])
    out = torch.empty(3, 32, 128, dtype=torch.bfloat16, device="cuda")
    for _ in range(20):
        c.kp.decode_attention(0, c.btd, sl, qd, out)
        got = c.run(lens, q, 777, 0)
        far = c.run(lens, q, 100, 5)
    c.check(lens, q, got, 777, 0)
    c.check(lens, q, far, 100, 5)
    c.check(lens, q, out.view(3, 1, 32, 128), 777, 0)
    c.kp.close()


def test_offsets_beyond_32_bits():
    """A cache of 5 GB, its last pages."""
    num = 75000
    bt = np.full((1, 5), -1, dtype=np.int32)
    bt[0] = [num - 1, 5, num - 2, num - 9, 0]
    from paper_2501_08090_b200 import binding as b
    kp = b.KvPool(b.make_config(1, 32, 8, 128, num, 5, 1))
    small = bf16(np.random.default_rng(26).standard_normal((5, 8, 2, 16, 128)))
    kp.pool_view()[0, torch.from_numpy(bt[0].astype(np.int64)).cuda()] = to_dev(small)
    q = queries(1, 1, 32, 128, 27)
    out = torch.empty(1, 32, 128, dtype=torch.bfloat16, device="cuda")
    kp.decode_attention_window(0, torch.from_numpy(bt).cuda(), torch.tensor([75], dtype=torch.int32, device="cuda"), to_dev(q[:, 0]), out, window=30, sink=2)
    assert kp.check_status() == 0
    t = np.arange(75)
    kv = small[t // 16, :, :, t % 16]
    for h in range(8):
        want, size, mass = ref.attend(q[0][:, h * 4:h * 4 + 4], kv[:, h, 0], kv[:, h, 1], 75, 30, 2)
        assert np.all(np.abs(out[0, h * 4:h * 4 + 4].double().cpu().numpy() - want[0]) <= ref.attend_tolerance(want, size, mass, 8)[0])
    kp.close()


def test_refusals():
    from paper_2501_08090_b200 import binding as b
    kp = b.KvPool(b.make_config(1, 8, 2, 64, 10, 4, 2))
    bt = torch.zeros(2, 4, dtype=torch.int32, device="cuda")
    sl = torch.ones(2, dtype=torch.int32, device="cuda")
    q = torch.zeros(2, 8, 64, dtype=torch.bfloat16, device="cuda")
    for bad in (dict(window=0), dict(window=-4), dict(window=4, sink=-1)):
        with pytest.raises(b.CkvError) as e:
            kp.decode_attention_window(0, bt, sl, q, q.clone(), **bad)
        assert e.value.code == b.CKV_EINVAL
    for layer in (-1, 1):
        with pytest.raises(b.CkvError):
            kp.decode_attention_window(layer, bt, sl, q, q.clone(), window=4)
    for args in ((bt[:1], sl, q, q.clone()), (bt, sl, q.float(), q.clone()), (bt, sl, q, q[:, :4]), (bt, sl.long(), q, q.clone()), (bt, sl, q[0], q[0].clone())):
        with pytest.raises(ValueError):
            kp.decode_attention_window(0, *args, window=4)
    assert kp.launch_count() == 0
    kp.close()
