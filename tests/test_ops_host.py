"""Host-only checks of the operators around a long decode step: argument checks that come before any
CUDA call, and the plain implementations of the GPU tests against hand-computed cases."""
import ctypes
import math

import numpy as np
import pytest

import ref_ops


@pytest.fixture(scope="module")
def b():
    from paper_2501_08090_b200 import build
    build.build()
    from paper_2501_08090_b200 import binding
    return binding


def test_null_handles_are_errors(b):
    assert b.lib.kv_append_rope(None, 0, 1, 1, None, None, None, None, 64, 0, 1.0, None, 0, None, 0, None, 0, None, 0, None) == b.CKV_EINVAL
    assert b.lib.kv_index_update(None, 0, 1, None, None, 0, None, 0, None) == b.CKV_EINVAL
    assert b.lib.kv_index_values(None, 0, None, 0, None, None) == b.CKV_EINVAL
    assert b.lib.decode_select_pages(None, 0, 1, None, None, None, None, 0, 4, 1, 1, None, None, None) == b.CKV_EINVAL
    assert b.lib.decode_attention_pages(None, 0, 1, 4, None, None, None, None, None) == b.CKV_EINVAL
    assert b.lib.decode_attention_sparse(None, 0, 1, None, None, None, None, 0, 4, 1, 1, None, None, None, None) == b.CKV_EINVAL


def test_index_size(b):
    cfg = b.make_config(3, 8, 2, 128, 100, 4, 4)
    assert b.kv_index_bytes(cfg) == 3 * 100 * 2 * (2 * 128 + 4)
    cfg = b.make_config(1, 8, 2, 96, 100, 4, 4)
    assert b.kv_index_bytes(cfg) == 0 and "head_dim" in b.last_error()


@pytest.mark.parametrize("change,needle", [
    (dict(batch=0), "batch"), (dict(batch=1 << 28), "batch"), (dict(max_draft=-1), "max_draft"), (dict(vocab=0), "vocab"),
    (dict(dtype=2), "dtype"), (dict(target=None), "NULL"), (dict(tokens=None), "NULL"), (dict(drafts=None), "NULL"),
    (dict(u_accept=None), "NULL"), (dict(u_sample=None), "NULL"), (dict(accepted=None), "NULL"),
    (dict(target_stride=99), "stride"), (dict(draft_stride=99), "stride"), (dict(target=4097), "aligned"), (dict(draft=8194), "aligned")])
def test_draft_verify_refusals(b, change, needle):
    a = dict(batch=2, max_draft=3, vocab=100, dtype=0, drafts=16, lens=None, target=4096, target_stride=100, draft=8192,
             draft_stride=100, u_accept=64, u_sample=96, tokens=128, accepted=256, stream=None)
    a.update(change)
    assert b.lib.draft_verify(*a.values()) == b.CKV_EINVAL
    assert needle in b.last_error()


def test_plain_rotation_by_hand():
    x = np.array([[1.0, 2.0, 3.0, 4.0, 5.0, 6.0]])
    out, size = ref_ops.rotate(x, 1, [math.pi / 2, math.pi], False)
    assert np.allclose(out, [[-3, -2, 1, -4, 5, 6]]) and size.tolist() == [[4, 6, 4, 6, 5, 6]]
    out, _ = ref_ops.rotate(x, 1, [math.pi / 2, math.pi], True, scale=2.0)
    assert np.allclose(out, [[-4, 2, -6, -8, 5, 6]])
    assert [t for t in ref_ops.new_tokens([7, 5], 3, [0, 2, 3])] == [(0, 0, 5), (1, 0, 6), (2, 1, 4)]


def test_plain_bounds_by_hand():
    lo, hi, step = ref_ops.key_bounds(np.array([[1.0, -0.51, 0.0], [0.3, 0.25, 0.0]]))
    assert step == 2.0 ** -6 and lo.tolist() == [19, -33, 0] and hi.tolist() == [64, 16, 0]
    lo, hi, step = ref_ops.key_bounds(np.array([[127.5, -1.0]]))
    assert step == 2.0 and hi.tolist() == [64, 0] and lo.tolist() == [63, -1]
    lo, hi, step = ref_ops.key_bounds(np.array([[np.inf, 0.0]]))
    assert step == 2.0 ** 121 and lo.tolist() == [-127, -127]


def test_plain_selection_by_hand():
    index = {(p, 0): (np.array([lo]), np.array([hi]), 1.0) for p, lo, hi in ((9, 0, 0), (8, -5, 1), (7, 2, 3), (6, -9, -5), (5, 0, 0))}
    tables = [9, 8, 7, 6, 5]
    assert ref_ops.select(index, tables, 80, np.array([[1.0]]), 0, 3, 1, 1) == [9, 7, 5]
    assert ref_ops.select(index, tables, 80, np.array([[-1.0]]), 0, 3, 1, 1) == [9, 6, 5]
    assert ref_ops.select(index, tables, 80, np.array([[-1.0]]), 0, 4, 1, 1) == [9, 8, 6, 5]
    assert ref_ops.select(index, tables, 80, np.array([[0.0]]), 0, 3, 1, 1) == [9, 8, 5]
    assert ref_ops.select(index, tables, 48, np.array([[1.0]]), 0, 3, 1, 1) == [9, 8, 7]


def test_plain_verification_by_hand():
    p = np.array([[0.5, 0.5, 0.0], [0.2, 0.2, 0.6]])
    q = np.array([[0.9, 0.1, 0.0]])
    assert ref_ops.verify([0], p, q, [0.5], 0.99) == (1, [0, 2])          # 0.45 < 0.5
    assert ref_ops.verify([0], p, q, [0.6], 0.0) == (0, [1])              # 0.54 >= 0.5; only token 1 has p > q
    assert ref_ops.verify([0], p, None, [0.5], 0.3) == (0, [1])           # 0.5 >= 0.5; p without token 0
    assert ref_ops.verify([], p[:1], None, [], 0.5) == (0, [1])
    assert ref_ops.verify([2], p, q, [0.0], 0.2) == (0, [1])              # p = 0: refused even at u = 0


def test_marshalling_refuses_what_the_library_cannot_see(b):
    """Checks of the tensors and numbers of a call, none of which reaches CUDA."""
    import torch
    m = b._marshal
    x = torch.zeros(2, 3, 4, dtype=torch.bfloat16)
    for bad in (x, None, 3, torch.zeros(2, 3)):
        with pytest.raises(ValueError) as e:
            m.on(0, bad, torch.bfloat16, "thing", 2, 3, 4)
        assert "thing" in str(e.value)
        with pytest.raises(ValueError) as e:
            m.rows_on(0, bad, "rows", 2, 3, 4)
        assert "rows" in str(e.value)
    with pytest.raises(TypeError):
        m.on(0, x)
    with pytest.raises(TypeError):
        m.draft_verify(1, 2, 3)
    ok = [2, 3, 100, 0, 16, None, 4096, 100, 8192, 100, 64, 96, 128, 256, None]
    assert m.draft_verify(*[-1 if i == 1 else v for i, v in enumerate(ok)]) == b.CKV_EINVAL and "max_draft" in b.last_error()
    for at, wrong, kind in ((0, 2 ** 31, OverflowError), (0, "two", TypeError), (4, "address", TypeError), (6, 1.5, TypeError)):
        with pytest.raises(kind):
            m.draft_verify(*[wrong if i == at else v for i, v in enumerate(ok)])
    assert m.kv_index_update(None, 0, 1, None, None, 0, None, 0, None) == b.CKV_EINVAL
