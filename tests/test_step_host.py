"""Host-only checks of the operators of a decode step whose state stays on the GPU: arguments that are refused
before any CUDA call, and the plain implementations of the GPU tests against hand-computed cases."""
import ctypes
import math

import numpy as np
import pytest

import ref_step as ref


@pytest.fixture(scope="module")
def b():
    from paper_2501_08090_b200 import build
    build.build()
    from paper_2501_08090_b200 import binding
    return binding


def test_null_handles_are_errors(b):
    def call(name):
        fn = getattr(b.lib, name)
        args = [0 if t in (ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_float) else None for t in fn.argtypes]
        return fn(*args)

    for name in ("kv8_append", "kv8_gather", "kv8_attention", "decode_attention_window", "kv_pages_assign", "kv_pages_release", "logits_process",
                 "kv8_pool_create"):
        assert call(name) == b.CKV_EINVAL, name


def test_cache_size(b):
    cfg = b.make_config(3, 8, 2, 128, 100, 4, 4)
    assert b.kv8_pool_bytes(cfg) == 3 * 100 * 2 * 2 * (16 * 128 + 4)
    assert 2 * b.kv8_pool_bytes(cfg) < 1.01 * b.kv_pool_bytes(cfg)
    cfg = b.make_config(1, 8, 2, 96, 100, 4, 4)
    assert b.kv8_pool_bytes(cfg) == 0 and "head_dim" in b.last_error()


def test_create_refuses_buffers_before_any_cuda_call(b):
    cfg = b.make_config(1, 8, 2, 128, 16, 4, 4)
    h = ctypes.c_void_p()
    c, w = b.kv8_pool_bytes(cfg), b.kv_workspace_bytes(cfg)
    for cache, cb, ws, wb, code, needle in ((None, c, 4096, w, b.CKV_EINVAL, "NULL"), (4096 + 16, c, 8192, w, b.CKV_EINVAL, "aligned"),
                                            (4096, c - 1, 8192, w, b.CKV_ENOMEM, "needed"), (4096, c, 8192, w - 1, b.CKV_ENOMEM, "workspace")):
        assert b.lib.kv8_pool_create(ctypes.byref(cfg), cache, cb, ws, wb, 0, ctypes.byref(h)) == code and not h.value
        assert needle in b.last_error() and "kv8_pool_create" in b.last_error()


def test_create_refuses_more_heads_than_a_pages_rows_are_counted_for(b):
    h = ctypes.c_void_p()
    for heads, needle in ((2048, "num_q_heads"), (2047, "NULL")):
        cfg = b.make_config(1, heads, heads, 64, 16, 4, 4)
        assert b.lib.kv8_pool_create(ctypes.byref(cfg), None, 1 << 40, None, 1 << 40, 0, ctypes.byref(h)) == b.CKV_EINVAL and not h.value
        assert needle in b.last_error()


@pytest.mark.parametrize("change,needle", [
    (dict(batch=0), "batch"), (dict(rows=0), "rows"), (dict(batch=1 << 20, rows=1 << 10), "rows"), (dict(vocab=0), "vocab"),
    (dict(vocab=262129), "vocab"), (dict(in_dtype=2), "dtype"), (dict(out_dtype=-1), "dtype"), (dict(logits=None), "NULL"), (dict(out=None), "NULL"),
    (dict(prompt=None), "history"), (dict(told=None), "history"), (dict(history_stride=-1), "history"), (dict(params=None), "params"),
    (dict(n_bias=-1), "n_bias"), (dict(bias=None), "bias"), (dict(ids=None), "bias"), (dict(logits_stride=99), "stride"), (dict(out_stride=99), "stride"),
    (dict(mask_stride=3), "mask"), (dict(logits=1 << 20 | 2), "aligned"), (dict(out=1 << 24 | 1), "aligned"),
    (dict(out=(1 << 20) + 400), "overlaps"), (dict(out=(1 << 20), out_dtype=1), "overlaps"), (dict(out=1 << 20, out_stride=104), "overlaps"),
    (dict(out=(1 << 20) - 2396), "overlaps")])
def test_logits_refusals(b, change, needle):
    a = dict(batch=2, rows=3, vocab=100, in_dtype=0, out_dtype=0, probs=1, logits=1 << 20, logits_stride=100, params=64, history=128, history_stride=5,
             prompt=256, told=512, drafts=1024, ids=2048, bias=4096, n_bias=4, mask=8192, mask_stride=4, out=1 << 24, out_stride=100, stream=None)
    a.update(change)
    assert b.lib.logits_process(*a.values()) == b.CKV_EINVAL
    assert needle in b.last_error()


def test_plain_quantisation_by_hand():
    rec, steps = np.zeros((2, 1, 2, 16, 4)), np.zeros((2, 1, 2))
    rows = np.zeros((1, 1, 2, 4))
    rows[0, 0, 0], rows[0, 0, 1] = [1.0, -0.5, 0.0078125, 0.0234375], [127.5, -127.5, 0.5, 1.5]
    ref.append8(rec, steps, 1, 0, rows)
    assert steps[1].tolist() == [[2.0 ** -6, 1.0]]
    assert rec[1, 0, 0, 0].tolist() == [64, -32, 0, 2] and rec[1, 0, 1, 0].tolist() == [127, -127, 0, 2]
    rows[0, 0, 0, 0] = 4.0
    ref.append8(rec, steps, 1, 1, rows)
    assert steps[1, 0, 0] == 2.0 ** -4 and rec[1, 0, 0, :2].tolist() == [[16, -8, 0, 0], [64, -8, 0, 0]]
    rows[0, 0, 1, 2] = math.nan
    ref.append8(rec, steps, 1, 2, rows)
    assert math.isnan(steps[1, 0, 1]) and rec[1, 0, 1, :3].tolist() == [[127, -127, 0, 2], [127, -127, 0, 2], [0, 0, 0, 0]]
    assert ref.need_step(np.array([2.0 ** -120])) == 2.0 ** -106 and not rec[0].any()
    ref.append8_tokens(rec, steps, [0, 1], 18, np.ones((3, 1, 2, 4)))
    assert rec[0, 0, 0, 15].tolist() == [64] * 4 and rec[1, 0, 0, :3].tolist() == [[64] * 4, [64] * 4, [64, -8, 0, 0]]
    assert steps.tolist() == [[[2.0 ** -6] * 2]] * 2


def test_plain_windows_by_hand():
    k, v = np.zeros((6, 2)), np.arange(12.0).reshape(6, 2)
    out, size, _ = ref.attend(np.ones((2, 1, 2)), k, v, 6, 2, 1)
    assert np.allclose(out[:, 0], [[14 / 3, 17 / 3], [6, 7]], rtol=1e-15) and np.array_equal(out, size)      # tokens 0, 3, 4 and 0, 4, 5
    assert ref.attend(np.ones((1, 1, 2)), k, v, 1, 0, 0)[0][0, 0].tolist() == [0, 1]


def test_plain_pages_by_hand():
    tables = [[5, 6, -1], [7, -1, -1], [-1, -1, -1]]
    free = [1, 2, 3, -7, -7, -7, -7, -7]
    out, count, step, start, slots, bad = ref.assign(tables, [20, 16, 0], [2, 17, 1], free, 3, 8)
    assert (out, count, step, start, bad) == ([22, 33, 1], 0, [22, 33, 1], [0, 2, 19, 20], False)
    assert tables == [[5, 6, -1], [7, 3, 2], [1, -1, -1]] and slots[:3] == [6 * 16 + 4, 6 * 16 + 5, 3 * 16] and slots[-1] == 16
    out, count, bad = ref.release(tables, out, [20, 16, 0], free, 0, 8)
    assert (out, count, bad) == ([20, 16, 0], 3, False) and free[:3] == [1, 2, 3]


def test_plain_logits_by_hand():
    x, p = ref.logits(np.array([2.0, -2.0, 1.0, 0.0]), [2.0, 0.25, 0.5, 1.0], prompt=[1], said=[0, 0, 9], bias=[(3, 5.0), (3, 1.0), (-1, 9.0)])
    assert x.tolist() == [1.0 - 1.0 - 0.25, -4.0, 1.0, 1.0] and abs(p.sum() - 1) < 1e-15
    x, p = ref.logits(np.array([2.0, 3.0, 3.0]), [1, 0, 0, 0.0], mask=np.array([True, True, True]))
    assert p.tolist() == [0, 1, 0]
    assert not ref.logits(np.ones(3), mask=np.zeros(3, bool))[1].any()
