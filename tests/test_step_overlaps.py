"""Results written over a call's own inputs are refused by the calls of a step whose state stays on the GPU; rows that lie
between one another's, or in place where that is allowed, are not."""
import ctypes
import itertools

import numpy as np
import pytest


@pytest.fixture(scope="module")
def b():
    from paper_2501_08090_b200 import build
    build.build()
    from paper_2501_08090_b200 import binding
    return binding


LOGITS = dict(batch=2, rows=3, vocab=100, in_dtype=0, out_dtype=0, probs=1, logits=1 << 20, logits_stride=100, params=64, history=128, history_stride=5,
              prompt=256, told=512, drafts=1024, ids=2048, bias=4096, n_bias=4, mask=8192, mask_stride=4, out=1 << 24, out_stride=100, stream=None)


@pytest.mark.parametrize("name,at,size,shown", [
    ("params", 1 << 21, 32, "params"), ("history", 1 << 21, 40, "history"), ("prompt", 1 << 21, 8, "prompt_lens"), ("told", 1 << 21, 8, "history_lens"),
    ("drafts", 1 << 21, 16, "drafts"), ("ids", 1 << 21, 32, "bias_ids"), ("bias", 1 << 21, 32, "bias"), ("mask", 1 << 21, 96, "mask")])
def test_logits_process_out_over_its_inputs(b, name, at, size, shown):
    """Out holds 6 rows of 400 bytes; the input's first or last bytes lie in them."""
    for out in (at, at + size - 4, at - 2396, at - 800):
        a = dict(LOGITS, out=out, **{name: at})
        assert b.lib.logits_process(*a.values()) == b.CKV_EINVAL
        assert b.last_error().endswith("out overlaps " + shown)


def touches(p, row_p, step_p, q, row_q, step_q, n):
    a = {p + i * step_p + k for i in range(n) for k in range(row_p)}
    return any(q + i * step_q + k in a for i in range(n) for k in range(row_q))


@pytest.mark.parametrize("in_dtype,out_dtype", [(0, 0), (1, 1), (0, 1), (1, 0)])
def test_rows_between_rows(b, in_dtype, out_dtype):
    """Rows of out beside, in the gaps of and over the logits' rows: refused exactly where a byte is shared.  The
    call never gets to the GPU: its parameters lie in out's first row."""
    size = (4, 2)
    base, vocab, n = 1 << 20, 5, 6
    seen = set()
    for step_in, step_out in itertools.product((5, 7, 10, 13, 40), (5, 7, 10, 11, 40)):
        for shift in range(-60, 61, 2 if in_dtype == out_dtype == 1 else 4):
            out = base + shift * (5 if shift % 8 == 0 else 1)
            a = dict(LOGITS, vocab=vocab, in_dtype=in_dtype, out_dtype=out_dtype, logits=base, logits_stride=step_in, out=out, out_stride=step_out,
                     params=out + 4, history=None, drafts=None, ids=None, bias=None, n_bias=0, mask=None)
            bad = touches(base, vocab * size[in_dtype], step_in * size[in_dtype], out, vocab * size[out_dtype], step_out * size[out_dtype], n)
            bad = bad and not (out == base and in_dtype == out_dtype and step_in == step_out)
            seen.add(bad)
            assert b.lib.logits_process(*a.values()) == b.CKV_EINVAL
            assert ("overlaps the logits" in b.last_error()) == bad, (step_in, step_out, shift, b.last_error())
            assert bad or "overlaps params" in b.last_error()
    assert seen == {False, True}


@pytest.mark.gpu
def test_logits_in_the_gaps_of_one_array(b):
    import torch
    both = torch.randn(3, 4, 300, device="cuda")
    logits, out = both[..., :137], both[..., 140:277]
    want = torch.softmax(logits.double(), -1)
    b.logits_process(logits, out)
    assert (out.double() - want).abs().max() < 1e-6
    with pytest.raises(b.CkvError):
        b.logits_process(logits, both[..., 136:273])
    place = torch.full((2000,), -1, dtype=torch.int32, device="cuda")
    with pytest.raises(b.CkvError) as e:
        b.logits_process(logits, place[:1644].view(torch.float32).view(3, 4, 137), mask=place[1600:1660].view(3, 4, 5))
    assert "out overlaps mask" in str(e.value) and (place == -1).all()
