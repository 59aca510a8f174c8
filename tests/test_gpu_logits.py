"""Penalties, biases, masks and probabilities against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import ref_step as ref

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def dev(x, dtype=torch.int32):
    return torch.tensor(np.asarray(x), dtype=dtype, device="cuda")


def pack_mask(mask):
    """Truth values [B][R][V] as words."""
    B, R, V = mask.shape
    bits = np.zeros((B, R, (V + 31) // 32 * 32), dtype=np.uint8)
    bits[..., :V] = mask
    words = np.packbits(bits.reshape(B, R, -1, 32), axis=-1, bitorder="little").view(np.uint32)[..., 0]
    return torch.from_numpy(words.astype(np.int64).astype(np.uint32).view(np.int32)).cuda()


class Case:
    """Inputs of a call in numpy; every part is optional."""

    def __init__(self, B, R, V, seed, dtype=F32, sharp=3.0):
        self.rng = np.random.default_rng(seed)
        self.B, self.R, self.V = B, R, V
        self.x = torch.from_numpy(self.rng.standard_normal((B, R, V)) * sharp).to(dtype)
        self.params = self.history = self.prompt = self.told = self.drafts = self.ids = self.bias = self.mask = None

    def text(self, *shape):
        return (self.rng.random(shape) ** 3 * self.V).astype(np.int32)

    def penalise(self, length, params=None):
        B, R = self.B, self.R
        self.params = np.float32(params) if params is not None else np.float32(
            np.stack([self.rng.uniform(0.7, 1.6, B), self.rng.uniform(-0.5, 1, B), self.rng.uniform(-0.2, 0.6, B), self.rng.uniform(0.3, 1.5, B)], 1))
        self.history = self.text(B, length)
        self.told = self.rng.integers(0, length + 1, B).astype(np.int32)
        self.prompt = (self.told * self.rng.random(B)).astype(np.int32)
        if R > 1:
            self.drafts = self.text(B, R - 1)
        return self

    def with_bias(self, n):
        self.ids = self.text(self.B, n)
        self.ids[self.rng.random(self.ids.shape) < 0.2] = -1
        self.bias = np.float32(self.rng.standard_normal((self.B, n)) * 3)
        return self

    def with_mask(self, share=0.5):
        self.mask = self.rng.random((self.B, self.R, self.V)) < share
        return self

    def options(self):
        o = {}
        if self.params is not None:
            o["params"] = dev(self.params, F32)
        if self.history is not None:
            o.update(history=dev(self.history), prompt_lens=dev(self.prompt), history_lens=dev(self.told))
        if self.drafts is not None:
            o["drafts"] = dev(self.drafts)
        if self.ids is not None:
            o.update(bias_ids=dev(self.ids), bias=dev(self.bias, F32))
        if self.mask is not None:
            o["mask"] = pack_mask(self.mask)
        return o

    def reference(self, b, j):
        prompt, said = (), ()
        if self.history is not None:
            n = int(np.clip(self.told[b], 0, self.history.shape[1]))
            m = int(np.clip(self.prompt[b], 0, n))
            prompt, said = self.history[b, :m], list(self.history[b, m:n])
        if self.drafts is not None:
            said = list(said) + list(self.drafts[b, :j])
        bias = zip(self.ids[b], self.bias[b]) if self.ids is not None else ()
        return ref.logits(self.x[b, j].double().numpy(), None if self.params is None else self.params[b].astype(np.float64), prompt, said, bias,
                          None if self.mask is None else self.mask[b, j])

    def run(self, out_dtype=F32, probs=True, x=None, out=None):
        from paper_2501_08090_b200 import binding as b
        x = self.x.cuda() if x is None else x
        out = torch.full(x.shape, float("nan"), dtype=out_dtype, device="cuda") if out is None else out
        b.logits_process(x, out, probs=probs, **self.options())
        return out

    def check(self, out, probs=True):
        """x: at most six fp32 roundings of numbers no larger than `size`.  p: x - max and its product with log2(e) / T add three
        roundings of the exponent, the exponential, the sum (of at most 262128 terms by 512 threads, 16 warps and 16 CTAs in turn: 40
        additions deep at most), the quotient and the factor between CTAs 2^-22 each at most, 64 in all; then the output's own."""
        got = out.double().cpu().numpy()
        half = torch.finfo(out.dtype).eps / 2
        for b in range(self.B):
            for j in range(self.R):
                x, p = self.reference(b, j)
                given = self.x[b, j].double().numpy()
                size = np.abs(np.where(np.isfinite(given), given, 0.0)) * (2.0 if self.params is None else max(2.0, 2 * self.params[b, 0], 2 / self.params[b, 0])) + 40
                ex = 6 * 2.0 ** -24 * size
                if not probs:
                    fine = np.isfinite(x)
                    np.testing.assert_array_equal(np.isnan(got[b, j]), np.isnan(x))
                    np.testing.assert_array_equal(got[b, j][~fine & ~np.isnan(x)], x[~fine & ~np.isnan(x)])
                    assert np.all(np.abs(got[b, j][fine] - x[fine]) <= (ex + half * (np.abs(np.where(fine, x, 0)) + ex))[fine])
                    continue
                if np.isnan(p).any():
                    assert np.isnan(got[b, j]).all(), (b, j)
                    continue
                t = 1.0 if self.params is None else float(self.params[b, 3])
                if not t > 0 or not p.any():
                    np.testing.assert_array_equal(got[b, j], p)
                    continue
                top = x.max()
                e = (ex + ex[np.argmax(x)] + 3 * 2.0 ** -24 * np.where(np.isfinite(x), np.abs(x - top), 0)) / t
                e = np.where(p > 0, e, 0.0)                  # a weight that vanishes in 64 bits vanishes in 32
                bound = p * (np.expm1(2 * e) + np.expm1(2 * float((p * e).sum())) + 64 * 2.0 ** -22)
                assert np.all(np.abs(got[b, j] - p) <= bound + half * (p + bound) + 2.0 ** -126), (b, j)


@pytest.mark.parametrize("out_dtype", [F32, BF16])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [1, 2, 31, 33, 1000, 4099, 16384, 16385, 32000, 50257, 128256])
def test_vocabularies(V, dtype, out_dtype):
    c = Case(3, 2, V, V, dtype).penalise(64).with_bias(9).with_mask(0.7)
    c.check(c.run(out_dtype))
    c.check(c.run(out_dtype, probs=False), probs=False)


@pytest.mark.parametrize("V", [131073, 151936, 262128])
def test_the_largest_vocabularies(V):
    c = Case(1, 1, V, V, BF16).penalise(100).with_bias(50)
    c.check(c.run())


@pytest.mark.parametrize("B,R,V,length,dtype", [(60, 1, 50257, 700, F32), (1, 5, 128256, 4096, BF16), (1, 2, 99991, 9000, F32), (140, 1, 16384, 0, BF16)])
def test_few_long_slices(B, R, V, length, dtype):
    """What wide CTAs take: probabilities, the best tokens, logits, and in place."""
    c = Case(B, R, V, V + B, dtype)
    c.with_mask(0.6)
    if length:
        c.penalise(length).with_bias(40)
    c.check(c.run())
    x = c.x.cuda()
    c.check(c.run(probs=False, x=x, out=x), probs=False)
    if length:
        c.params[:, 3] = 0.0
        c.check(c.run())


@pytest.mark.parametrize("part", ["nothing", "params", "history", "drafts", "bias", "mask"])
@pytest.mark.parametrize("B,R", [(1, 1), (1, 7), (5, 4), (150, 2)])
def test_each_part_alone(B, R, part):
    c = Case(B, R, 1003, B * 10 + R)
    if part in ("params", "history", "drafts"):
        c.penalise(40)
    if part != "drafts":
        c.drafts = None
    if part != "history":
        c.history = c.prompt = c.told = None
    if part == "bias":
        c.with_bias(30)
    if part == "mask":
        c.with_mask(0.3)
    c.check(c.run())


def test_histories_of_every_length_and_foreign_tokens():
    """Lengths beyond the rows or below 0 are cut, a prompt longer than the history is all of it, foreign tokens count for nothing."""
    c = Case(8, 1, 500, 1).penalise(300)
    c.told[:] = [0, 1, 300, 299, 400, -3, 200, 31]
    c.prompt[:] = [0, 1, 0, 299, 500, -1, 250, -7]
    c.history[2, ::3] = -1
    c.history[3, ::4] = 500
    c.history[4, ::4] = 2 ** 31 - 1
    c.check(c.run())
    long = Case(2, 3, 700, 2).penalise(9000)
    long.told[:] = [9000, 8999]
    long.check(long.run())


def test_one_token_many_times():
    """Counts beyond 2^16, and one token that is all the history."""
    c = Case(1, 2, 50, 3).penalise(70000, [[1.1, 0.5, 0.0001, 1.0]])
    c.history[:] = 7
    c.told[:], c.prompt[:] = 70000, 3
    c.check(c.run())


def test_the_same_bias_twice():
    """The last of equal ids counts, whoever processes it."""
    c = Case(2, 1, 2000, 4).with_bias(1200)
    c.ids[0] = np.repeat(np.arange(12), 100)
    c.ids[1, 5:] = 77
    c.check(c.run())
    c.check(c.run(probs=False), probs=False)


def test_best_tokens():
    """temperature 0 (or below): the first of the largest, after penalties and masks."""
    for V in (5, 3000, 40000):
        c = Case(6, 2, V, V + 1, BF16).penalise(20)
        c.params[:, 3] = [0, 0, -1, 0, 0.5, 0]
        c.x[3] = c.x[3].round()                              # many equal ones
        c.x[5] = 0.0
        c.with_mask(0.6)
        c.mask[1] = False
        c.check(c.run())


def test_masks_that_leave_nothing_or_one():
    c = Case(3, 3, 777, 5).penalise(10).with_mask(0.0)
    c.mask[1, 1, 776] = True
    c.mask[2, 0, 0] = c.mask[2, 2, 31] = c.mask[2, 2, 32] = True
    out = c.run()
    c.check(out)
    assert not out[0].any() and out[1, 1, 776] == 1 and out[2, 0, 0] == 1 and out[1, 0].sum() == 0
    c.check(c.run(probs=False), probs=False)


@pytest.mark.parametrize("level", [-5000.0, -150.0, 150.0, 5000.0])
def test_slices_without_anything_allowed_beside_logits_far_from_zero(level):
    """Whole slices of a row are masked; what is allowed lies far above or below 0."""
    c = Case(3, 1, 60000, 13).with_mask(0.0)
    c.mask[0, 0, 100:120] = c.mask[1, 0, 59990:] = c.mask[2, 0, 20000:40000] = True
    c.x += level
    c.check(c.run())
    c.x[:, :, ::7] = float("-inf")
    c.check(c.run())


def test_what_is_not_finite():
    """NaN and infinities in masked places count for nothing; allowed, they make the row NaN; minus infinity is no weight."""
    c = Case(7, 1, 5000, 6).with_mask(0.5)
    c.mask[:, :, :8] = True
    c.x[0, 0, np.nonzero(~c.mask[0, 0])[0][:50]] = float("nan")
    c.x[1, 0, np.nonzero(~c.mask[1, 0])[0][-3:]] = float("inf")
    c.x[2, 0, 3] = float("nan")
    c.x[3, 0, 4] = float("inf")
    c.x[4, 0, :8] = float("-inf")
    c.x[5] = float("-inf")
    c.x[6, 0, 1:] = torch.finfo(F32).min                     # a mask of the lowest value
    out = c.run()
    c.check(out)
    assert torch.isnan(out[2]).all() and torch.isnan(out[3]).all() and not out[5].any() and out[6, 0, 0] == 1
    low = Case(1, 1, 64, 7)
    low.x[:] = torch.finfo(F32).min                          # nothing else: all the same
    low.params = np.float32([[1, 0, 0, 0.5]])
    assert torch.equal(low.run(), torch.full((1, 1, 64), 1 / 64, device="cuda"))


def test_extreme_temperatures():
    c = Case(4, 1, 3000, 8).penalise(5)
    c.params[:, 3] = [1e-30, 1e-40, 1e4, 1e30]
    out = c.run().double().cpu().numpy()[:, 0]
    for b in (0, 1):
        assert np.argmax(c.reference(b, 0)[0]) == np.argmax(out[b]) and out[b].max() == 1 and out[b].sum() == 1
    for b in (2, 3):
        assert abs(out[b].sum() - 1) < 1e-5 and out[b].max() / out[b].min() < 1.01


def test_an_infinite_temperature():
    """What is allowed gets the same weight, what is not gets none: sums of ones are exact, so only 1 / n is rounded."""
    c = Case(3, 2, 40000, 9).with_mask(0.5).penalise(20)
    c.params[:, 3] = [float("inf"), 3e38, float("inf")]
    c.mask[2, 1] = False
    out = c.run().double().cpu().numpy()
    for b in range(3):
        for j in range(2):
            n = int(c.mask[b, j].sum())
            want = np.where(c.mask[b, j], 1 / max(n, 1), 0)
            assert np.all(np.abs(out[b, j] - want) <= want * 2.0 ** -23), (b, j)


@pytest.mark.parametrize("dtype,out_dtype", [(F32, F32), (BF16, BF16), (BF16, F32), (F32, BF16)])
@pytest.mark.parametrize("V", [7, 64, 1001])
def test_rows_of_every_alignment(V, dtype, out_dtype):
    """Rows that start at every offset within 16 bytes, results at every offset against them; nothing beside a row is written."""
    c = Case(2, 2, V, V, dtype).penalise(10).with_mask(0.8)
    n_in, n_out = 16 // dtype.itemsize, 16 // out_dtype.itemsize
    stride = (V + 40) // 8 * 8 + 1                           # rows at different offsets too
    for i in range(n_in):
        for j in range(n_out):
            base = torch.full((4 * stride + 64,), float("nan"), dtype=dtype, device="cuda")
            x = base[i:].as_strided((2, 2, V), (2 * stride, stride, 1))
            x.copy_(c.x)
            place = torch.full((4 * stride + 64,), 3.0, dtype=out_dtype, device="cuda")
            out = place[j:].as_strided((2, 2, V), (2 * stride, stride, 1))
            c.run(x=x, out=out)
            c.check(out)
            out.fill_(3.0)
            assert torch.all(place == 3.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_in_place(dtype):
    for probs in (False, True):
        c = Case(3, 2, 20001, 9, dtype).penalise(30).with_bias(4)
        x = c.x.cuda()
        c.run(probs=probs, x=x, out=x)
        c.check(x, probs)


def test_rows_far_apart():
    """Rows 2^29 elements apart: offsets beyond 32 bits."""
    c = Case(2, 2, 300, 10, BF16).penalise(20)
    far = torch.empty(3 * 2 ** 29 + 512, dtype=BF16, device="cuda")
    x = far.as_strided((2, 2, 300), (2 ** 30, 2 ** 29, 1))
    x.copy_(c.x)
    c.check(c.run(x=x))
    c.run(x=x, out=x)
    c.check(x)


def test_streams_and_graphs():
    c, d = Case(4, 2, 9000, 11).penalise(50), Case(4, 2, 9000, 12).penalise(50)
    from paper_2501_08090_b200 import binding as b
    x, o = c.x.cuda(), c.options()
    out, s, g = torch.empty_like(x), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=s):
        b.logits_process(x, out, **o)
        b.logits_process(out, out, probs=False)              # straight behind: reads what the first one writes
    g.replay()
    torch.cuda.synchronize()
    c.check(out)
    x.copy_(d.x)
    for name, t in d.options().items():
        o[name].copy_(t)
    g.replay()
    torch.cuda.synchronize()
    d.check(out)
    out.zero_()
    torch.cuda.synchronize()
    b.logits_process(x, out, stream=s, **o)
    s.synchronize()
    d.check(out)


def test_refusals():
    from paper_2501_08090_b200 import binding as b
    x = torch.zeros(2, 3, 100, device="cuda")
    h, n, d = torch.zeros(2, 5, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(2, 2, dtype=torch.int32, device="cuda")
    p, ids, bias = torch.ones(2, 4, device="cuda"), torch.zeros(2, 6, dtype=torch.int32, device="cuda"), torch.zeros(2, 6, device="cuda")
    mask = torch.zeros(2, 3, 4, dtype=torch.int32, device="cuda")
    good = dict(params=p, history=h, prompt_lens=n, history_lens=n, drafts=d, bias_ids=ids, bias=bias, mask=mask)
    b.logits_process(x, x.clone(), **good)
    for bad in (dict(params=p[:, :3]), dict(params=p.double()), dict(history=h[:1]), dict(history=h.long()), dict(prompt_lens=None), dict(history_lens=n[:1]),
                dict(drafts=d[:, :1].contiguous()), dict(bias=None), dict(bias=bias[:, :5]), dict(bias_ids=ids.long()), dict(mask=mask[:, :, :3].contiguous()),
                dict(mask=mask.cpu())):
        with pytest.raises(ValueError):
            b.logits_process(x, x.clone(), **{**good, **bad})
    for bad in (x[0], x.half(), x.cpu(), x[..., ::2]):
        with pytest.raises(ValueError):
            b.logits_process(bad, bad)
    with pytest.raises(ValueError):
        b.logits_process(x, x[:, :2])
    with pytest.raises(b.CkvError):
        b.logits_process(x, x.clone(), **{**good, "params": None})
    both = torch.zeros(1300, device="cuda")
    for off in (4, 599):
        with pytest.raises(b.CkvError) as e:
            b.logits_process(both[:600].view(2, 3, 100), both[off:off + 600].view(2, 3, 100))
        assert "overlap" in str(e.value)
    b.logits_process(both[:600].view(2, 3, 100), both[600:1200].view(2, 3, 100))
    with pytest.raises(b.CkvError):
        b.logits_process(torch.zeros(1, 1, 262129, device="cuda"), torch.zeros(1, 1, 262129, device="cuda"))
