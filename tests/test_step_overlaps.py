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


@pytest.fixture(scope="module")
def pools(b):
    cfg = b.make_config(1, 8, 2, 64, 12, 4, 3)
    eight, sixteen = b.Kv8Pool(cfg), b.KvPool(cfg)
    yield eight, sixteen
    eight.close(); sixteen.close()


def refused(b, pool, call, name):
    before = pool.launch_count()
    with pytest.raises(b.CkvError) as e:
        call()
    assert e.value.code == b.CKV_EINVAL and "overlaps " + name in str(e.value) and pool.launch_count() == before


def tensors():
    import torch
    bt = torch.arange(12, dtype=torch.int32, device="cuda").view(3, 4)
    sl = torch.tensor([5, 40, 17], dtype=torch.int32, device="cuda")
    return bt, sl


def as_rows(t, heads, n=3):
    """The memory of an int32 tensor, from its start on, as bf16 rows (it has to be long enough)."""
    import torch
    return t.view(-1).view(torch.bfloat16)[:n * heads * 64].view(n, heads, 64)


@pytest.mark.gpu
def test_append_of_queries(b, pools):
    import torch
    pool, (bt, sl) = pools[0], tensors()
    freq = torch.ones(32, device="cuda")
    qkv = torch.randn(4, 3, 12, 64, device="cuda").to(torch.bfloat16)                         # three rows of queries, keys, values, four times
    q, k, v = qkv[0, :, :8], qkv[0, :, 8:10], qkv[0, :, 10:]
    wide = torch.zeros(1 << 14, dtype=torch.int32, device="cuda")
    for q_out, name in ((qkv[0, :, 1:9], "q"), (qkv[0, :, 4:], "q"), (qkv.view(-1)[128:][:3 * 768].view(3, 12, 64)[:, :8], "q"),
                        (qkv.view(-1, 64)[8:8 + 24].view(3, 8, 64), "q")):
        refused(b, pool, lambda: pool.kv8_append(0, bt, sl, k, v, q=q, q_out=q_out, inv_freq=freq), name)
    other = torch.randn(3, 8, 64, device="cuda").to(torch.bfloat16)
    for q_out, name in ((qkv[0, :, 1:9], "k_new"), (qkv[0, :, 4:], "k_new"), (qkv.view(-1, 64)[10:10 + 36].view(3, 12, 64)[:, :8], "v_new")):
        refused(b, pool, lambda: pool.kv8_append(0, bt, sl, k, v, q=other, q_out=q_out, inv_freq=freq), name)
    tables = wide[:12].view(3, 4).copy_(bt)
    refused(b, pool, lambda: pool.kv8_append(0, tables, sl, k, v, q=other, q_out=as_rows(wide, 8), inv_freq=freq), "block_tables")
    refused(b, pool, lambda: pool.kv8_append(0, bt, wide[765:768].copy_(sl), k, v, q=other, q_out=as_rows(wide, 8), inv_freq=freq), "seq_lens")
    start = wide[64:68].copy_(torch.arange(4, device="cuda"))
    refused(b, pool, lambda: pool.kv8_append(0, bt, sl, k, v, q=other, q_out=as_rows(wide, 8), inv_freq=freq, new_start=start), "new_start")
    refused(b, pool, lambda: pool.kv8_append(0, bt, sl, k, v, q=other, q_out=as_rows(wide, 8), inv_freq=wide[700:732].view(torch.float32)), "inv_freq")
    # in place, into the gap that another projection's rows leave, and behind the lists
    want = torch.empty_like(other)
    pool.kv8_append(0, bt, sl, k, v, q=q, q_out=want, inv_freq=freq)
    gap = torch.empty(3, 20, 64, dtype=torch.bfloat16, device="cuda")
    gap[:, :12] = qkv[0]
    for q_in, out in ((gap[:, :8], gap[:, 12:]), (q, q)):
        pool.kv8_append(0, bt, sl, k, v, q=q_in, q_out=out, inv_freq=freq)
        assert torch.equal(out, want)


@pytest.mark.gpu
def test_gather(b, pools):
    import torch
    pool, (bt, sl) = pools[0], tensors()
    both = torch.zeros(40, 64, dtype=torch.bfloat16, device="cuda")
    k = both[:24].view(3, 8, 64)
    for v in (k[:, 1:3], k[:, :2], both[6:12].view(3, 2, 64), both[17:23].view(3, 2, 64)):
        refused(b, pool, lambda: pool.kv8_gather(0, bt, sl, k[:, :2], v), "v")
    wide = torch.zeros(1 << 10, dtype=torch.int32, device="cuda")
    v = torch.empty(3, 2, 64, dtype=torch.bfloat16, device="cuda")
    rows = as_rows(wide, 2)
    tables, lens, start = wide[180:192].view(3, 4), wide[189:192], wide[188:192]
    for k_, v_ in ((rows, v), (v, rows)):
        refused(b, pool, lambda: pool.kv8_gather(0, tables, sl, k_, v_), "block_tables")
        refused(b, pool, lambda: pool.kv8_gather(0, bt, lens, k_, v_), "seq_lens")
        refused(b, pool, lambda: pool.kv8_gather(0, bt, sl, k_, v_, start=start), "start")
    pool.kv8_gather(0, bt, sl, k[:, 2:4], k[:, 4:6])         # beside one another
    assert pool.check_status() == 0


@pytest.mark.gpu
def test_attention(b, pools):
    import torch
    bt, sl = tensors()
    for pool, name, options in ((pools[0], "kv8_attention", {}), (pools[1], "decode_attention_window", dict(window=9))):
        pool.pool.zero_()
        call = getattr(pool, name)
        line = torch.randn(64, 64, device="cuda").to(torch.bfloat16)
        q = line[:24].view(3, 8, 64)
        for at in (1, 8, 23):
            refused(b, pool, lambda: call(0, bt, sl, q, line[at:at + 24].view(3, 8, 64), **options), "q")
            refused(b, pool, lambda: call(0, bt, sl, line[at:at + 24].view(3, 8, 64), q, **options), "q")
        wide = torch.zeros(1 << 10, dtype=torch.int32, device="cuda")
        refused(b, pool, lambda: call(0, wide[760:772].view(3, 4), sl, q, as_rows(wide, 8), **options), "block_tables")
        refused(b, pool, lambda: call(0, bt, wide[:3], q, as_rows(wide, 8), **options), "seq_lens")
        call(0, bt, sl, q, line[24:48].view(3, 8, 64), **options)
        assert pool.check_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("width,window,q_len", [(64, 0, 1), (64, 300, 5), (4000, 0, 1), (4000, 0, 5)])
def test_attention_in_place_of_the_queries(width, window, q_len):
    """By clusters and by even spans, blocks of new tokens one after another."""
    import torch
    import test_gpu_cache8
    import test_gpu_window
    lens = [1000, 5, 333, 17, 1024]
    bt, n = test_gpu_cache8.tables_for(lens, width, 1)
    q = test_gpu_cache8.to_dev(test_gpu_cache8.queries(5, q_len, 16, 64, 2))
    for kind in (test_gpu_cache8.Cache, test_gpu_window.Cache):
        c = kind((16, 4, 64), bt, n, seed=3)
        sl = torch.tensor(lens, dtype=torch.int32, device="cuda")
        call = c.kp.kv8_attention if kind is test_gpu_cache8.Cache else c.kp.decode_attention_window
        out, place = torch.empty_like(q), q.clone()
        call(0, c.btd, sl, q, out, window=window or 10 ** 6, sink=3)
        call(0, c.btd, sl, place, place, window=window or 10 ** 6, sink=3)
        assert torch.equal(out, place) and c.kp.check_status() == 0
        c.kp.close()


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
