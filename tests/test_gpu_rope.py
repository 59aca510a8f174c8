"""The rotated append against its definition in 64 bits, over head layouts, rotations, ragged batches,
strides and far positions; what it must not touch; what it flags and refuses."""
import numpy as np
import pytest
import torch

from paper_2501_08090_b200 import workloads as wl

import ref_ops
from helpers import bits_to_dev, dev_to_bits, widen

pytestmark = pytest.mark.gpu

# A result is rounded once to bf16 (half a step: 2^-8 of the value).  Before that: the turn's fraction is
# rounded to fp32 (at most 2^-25 turns, 2^-22.3 radians), sincospif is within 2 units in the last
# place (2^-23), the scale and the two products round by 2^-24 each: under 2^-21 of |x| + |y| together.
HALF_STEP, ARITH = 2.0 ** -8, 2.0 ** -21


def setup(lens, Hq, Hkv, d, seed, spare=3):
    from paper_2501_08090_b200 import binding as b
    lens = np.asarray(lens, dtype=np.int32)
    pages = int(wl.pages_of(lens).sum()) + spare
    bt = wl.block_tables(lens, pages, seed)
    pool = wl.normal_bf16((pages, Hkv, 2, 16, d), seed, 1)
    cfg = b.make_config(1, Hq, Hkv, d, pages, bt.shape[1], lens.size)
    kp = b.KvPool(cfg, pool=bits_to_dev(pool.reshape(-1)))
    return kp, lens, bt, pool, torch.from_numpy(bt).cuda(), torch.from_numpy(lens).cuda()


def rows(n, heads, d, seed, stream):
    return wl.normal_bf16((n, heads, d), seed, stream)


def inv_freq(rotary, base=500000.0):
    half = rotary // 2
    return (base ** (-np.arange(half) / half)).astype(np.float32)


def expect(q, k, v, pool, bt, lens, freq, interleaved, new_start=None, scale=1.0):
    """(q_out, its tolerance, pool, its tolerance) in float64; rows of no request stay NaN / untouched."""
    out, tol = np.full(q.shape, np.nan), np.zeros(q.shape)
    ref = widen(pool)
    ptol = np.zeros(ref.shape)
    for i, r, pos in ref_ops.new_tokens(lens, q.shape[0], new_start):
        out[i], size = ref_ops.rotate(widen(q[i]), pos, freq, interleaved, scale)
        delta = ARITH * abs(scale) * size * (np.arange(q.shape[2]) < 2 * len(freq))
        tol[i] = HALF_STEP * (np.abs(out[i]) + delta) + delta
        page, slot = bt[r][pos // 16], pos % 16
        ref[page, :, 0, slot], size = ref_ops.rotate(widen(k[i]), pos, freq, interleaved, scale)
        delta = ARITH * abs(scale) * size * (np.arange(q.shape[2]) < 2 * len(freq))
        ptol[page, :, 0, slot] = HALF_STEP * (np.abs(ref[page, :, 0, slot]) + delta) + delta
        ref[page, :, 1, slot] = widen(v[i])
    return out, tol, ref, ptol


def run(lens, q_len, Hq, Hkv, d, rotary, interleaved, seed, new=None, scale=1.0, packed=False, pad=0, in_place=False):
    kp, lens, bt, pool, btd, sld = setup(lens, Hq, Hkv, d, seed)
    starts = None if new is None else np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    n = (len(lens) * q_len if new is None else int(starts[-1])) + pad
    q, k, v = rows(n, Hq, d, seed, 2), rows(n, Hkv, d, seed, 3), rows(n, Hkv, d, seed, 4)
    freq = inv_freq(rotary)
    want, tol, ref_pool, pool_tol = expect(q, k, v, pool, bt, lens, freq, interleaved, starts, scale)
    if packed:
        qkv = bits_to_dev(np.concatenate([q, k, v], axis=1))
        qd, kd, vd = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    else:
        qd, kd, vd = bits_to_dev(q), bits_to_dev(k), bits_to_dev(v)
    out = qd if in_place else torch.full((n, Hq, d), 7.0, dtype=torch.bfloat16, device="cuda")
    kp.kv_append_rope(0, btd, sld, qd, kd, vd, out, torch.from_numpy(freq).cuda(),
                      new_start=None if starts is None else torch.from_numpy(starts).cuda(), interleaved=interleaved, scale=scale)
    assert kp.check_status() == 0
    got, got_pool = widen(dev_to_bits(out)), widen(dev_to_bits(kp.pool)).reshape(ref_pool.shape)
    live = ~np.isnan(want)
    assert np.all(np.abs(got - want)[live] <= tol[live])
    untouched = widen(q) if in_place else np.full(q.shape, 7.0)
    assert np.array_equal(got[~live], untouched[~live])           # rows of no request
    assert np.all(np.abs(got_pool - ref_pool) <= pool_tol)        # values and everything else bit-exact (tolerance 0)
    if packed and not in_place:
        assert np.array_equal(dev_to_bits(kd), k) and np.array_equal(dev_to_bits(qd), q)
    kp.close()


@pytest.mark.parametrize("Hq,Hkv,d,rotary,interleaved", [
    (32, 8, 128, 128, False), (64, 8, 128, 128, True), (4, 1, 64, 64, False), (4, 1, 64, 16, True), (12, 4, 64, 32, False),
    (35, 5, 128, 64, False), (1, 1, 128, 16, False), (6, 6, 64, 64, True), (8, 2, 128, 112, True), (7, 1, 128, 48, False)])
@pytest.mark.parametrize("q_len", [1, 3])
def test_even_batches(Hq, Hkv, d, rotary, interleaved, q_len):
    run([q_len, 16, 17, 31, 33, 260], q_len, Hq, Hkv, d, rotary, interleaved, seed=Hq + rotary + q_len)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("packed,in_place,pad", [(False, False, 5), (True, False, 0), (True, True, 2), (False, True, 0)])
def test_ragged_prompts_padding_and_strides(interleaved, packed, in_place, pad):
    new = [0, 1, 16, 0, 0, 47, 3, 200, 0]
    lens = [9, 1, 16, 1, 33, 50, 515, 200, 64]
    run(lens, 0, 8, 2, 128, 96, interleaved, seed=3, new=new, packed=packed, in_place=in_place, pad=pad, scale=1.25)


def test_many_requests_are_searched_in_rounds():
    rng = np.random.default_rng(5)
    new = rng.integers(0, 4, size=1500)
    run(new + rng.integers(1, 40, size=1500), 0, 2, 1, 64, 64, False, seed=6, new=new)
    run([20] * 33, 0, 2, 1, 64, 64, True, seed=7, new=[1] * 32 + [4])


@pytest.mark.parametrize("interleaved,in_place", [(False, True), (True, False)])
def test_long_prompts_take_several_tokens_a_cta(interleaved, in_place):
    """Enough tokens for four a CTA: requests that begin and end inside a CTA, empty ones, padding, a ragged end."""
    new = [0, 2501, 1, 0, 2, 2, 1801, 0, 450]
    run([n + extra for n, extra in zip(new, (5, 0, 40, 1, 0, 700, 3, 9, 0))], 0, 3, 1, 64, 32, interleaved, seed=11, new=new,
        packed=True, in_place=in_place, pad=6)
    run([1201] * 4, 1201, 2, 2, 64, 64, interleaved, seed=12)


def test_far_positions_keep_their_angle():
    for L in (131072, 1000003):
        run([L], 1, 4, 1, 64, 64, False, seed=8)


def test_values_of_special_rows_pass_through():
    """Infinities and NaN among the values are copied bit for bit; a rotated NaN stays one."""
    kp, lens, bt, pool, btd, sld = setup([5], 2, 1, 64, 9)
    v = np.array([[[0x7f80, 0xff80, 0x7fc1, 0x0001] * 16]], dtype=np.uint16)
    k = np.full((1, 1, 64), 0x7fc0, dtype=np.uint16)
    q = rows(1, 2, 64, 9, 2)
    out = torch.empty(1, 2, 64, dtype=torch.bfloat16, device="cuda")
    kp.kv_append_rope(0, btd, sld, bits_to_dev(q), bits_to_dev(k), bits_to_dev(v), out, torch.from_numpy(inv_freq(64)).cuda())
    got = dev_to_bits(kp.pool).reshape(pool.shape)[bt[0][0], 0]
    assert np.array_equal(got[1, 4], v[0, 0]) and np.all(np.isnan(widen(got[0, 4])))
    kp.close()


def test_keys_and_values_alone():
    kp, lens, bt, pool, btd, sld = setup([40, 3], 8, 2, 128, 10)
    k, v = rows(2, 2, 128, 10, 3), rows(2, 2, 128, 10, 4)
    freq = inv_freq(128)
    q = np.zeros((2, 8, 128), dtype=np.uint16)
    _, _, ref, tol = expect(q, k, v, pool, bt, lens, freq, False)
    kp.kv_append_rope(0, btd, sld, None, bits_to_dev(k), bits_to_dev(v), None, torch.from_numpy(freq).cuda())
    assert np.all(np.abs(widen(dev_to_bits(kp.pool)).reshape(ref.shape) - ref) <= tol)
    kp.close()


def test_a_second_layer_and_a_captured_call():
    from paper_2501_08090_b200 import binding as b
    cfg = b.make_config(2, 4, 1, 64, 8, 4, 2)
    kp = b.KvPool(cfg)
    kp.pool.zero_()
    btd = torch.arange(8, dtype=torch.int32, device="cuda").view(2, 4)
    sld = torch.tensor([10, 33], dtype=torch.int32, device="cuda")
    q, k, v = (torch.randn(2, h, 64, device="cuda").to(torch.bfloat16) for h in (4, 1, 1))
    out, freq = torch.zeros_like(q), torch.from_numpy(inv_freq(64)).cuda()
    kp.kv_append_rope(1, btd, sld, q, k, v, out, freq)
    first, pool = out.clone(), kp.pool.clone()
    assert not kp.pool_view()[0].any() and kp.pool_view()[1].any()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kp.kv_append_rope(1, btd, sld, q, k, v, out, freq)
    out.zero_(); kp.pool.zero_()
    graph.replay()
    assert torch.equal(out, first) and torch.equal(kp.pool, pool)
    sld.copy_(torch.tensor([11, 1], dtype=torch.int32))                # lengths are read when it runs
    graph.replay()
    assert not torch.equal(out, first)
    assert kp.check_status() == 0
    del graph
    kp.close()


def test_rows_far_apart():
    """Tokens 2^30 elements apart: offsets beyond 32 bits."""
    kp, lens, bt, pool, btd, sld = setup([20, 33, 7], 4, 2, 64, 15)
    q, k, v = rows(3, 4, 64, 15, 2), rows(3, 2, 64, 15, 3), rows(3, 2, 64, 15, 4)
    freq = inv_freq(64)
    want, tol, ref, ptol = expect(q, k, v, pool, bt, lens, freq, False)
    far = torch.empty(2 * 2 ** 30 + 4096, dtype=torch.bfloat16, device="cuda")
    at = lambda heads, off: far[off:].as_strided((3, heads, 64), (2 ** 30, 64, 1))
    qd, kd, vd, out = at(4, 0), at(2, 256), at(2, 384), at(4, 512)
    qd.copy_(bits_to_dev(q)); kd.copy_(bits_to_dev(k)); vd.copy_(bits_to_dev(v))
    kp.kv_append_rope(0, btd, sld, qd, kd, vd, out, torch.from_numpy(freq).cuda())
    assert kp.check_status() == 0
    assert np.all(np.abs(widen(dev_to_bits(out)) - want) <= tol)
    assert np.all(np.abs(widen(dev_to_bits(kp.pool)).reshape(ref.shape) - ref) <= ptol)
    kp.close()


def test_inputs_written_by_the_kernel_just_before():
    """Queries, lists and lengths come from the kernel that directly precedes each call, many times over."""
    kp, lens, bt, pool, btd, sld = setup([300, 77], 8, 2, 128, 16)
    freq = torch.from_numpy(inv_freq(128)).cuda()
    q0, k0, v0 = (torch.randn(6, h, 128, device="cuda").to(torch.bfloat16) for h in (8, 2, 2))
    start0 = torch.tensor([0, 4, 6], dtype=torch.int32, device="cuda")
    want = torch.empty_like(q0)
    kp.kv_append_rope(0, btd, sld, q0, k0, v0, want, freq, new_start=start0)
    pool0 = kp.pool.clone()
    q, start, out, lens_d = torch.empty_like(q0), torch.empty_like(start0), torch.empty_like(want), torch.empty_like(sld)
    for i in range(200):
        q.zero_(); start.zero_(); lens_d.fill_(1)
        lens_d.copy_(sld)
        start.copy_(start0)
        torch.add(q0, 0, out=q)
        kp.kv_append_rope(0, btd, lens_d, q, k0, v0, out, freq, new_start=start)
        if i % 20 == 0:
            assert torch.equal(out, want) and torch.equal(kp.pool, pool0)
        out.zero_()
    assert kp.check_status() == 0
    kp.close()


def test_unusable_requests_and_pages_are_flagged():
    from paper_2501_08090_b200 import binding as b
    kp, lens, bt, pool, btd, sld = setup([20, 20, 20, 20, 20], 4, 2, 64, 12)
    sld.copy_(torch.tensor([20, 0, 1, 1000, 20], dtype=torch.int32))    # request 1 empty, 2 shorter than its 2 new tokens, 3 beyond the table
    btd[4, 1] = 10 ** 6                                                  # position 18 and 19 of request 4
    n = 10
    q, k, v = rows(n, 4, 64, 12, 2), rows(n, 2, 64, 12, 3), rows(n, 2, 64, 12, 4)
    freq = inv_freq(64)
    out = torch.full((n, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    kp.kv_append_rope(0, btd, sld, bits_to_dev(q), bits_to_dev(k), bits_to_dev(v), out, torch.from_numpy(freq).cuda())
    assert kp.check_status(raise_on_error=False) == b.STATUS_BAD_LENGTH | b.STATUS_BAD_PAGE
    got = widen(dev_to_bits(out))
    assert not got[2:8].any() and got[:2].all() and got[8:].all()       # zero rows; request 4's queries are turned all the same
    want, tol, ref, ptol = expect(q[:2], k[:2], v[:2], pool, bt[:1], np.array([20]), freq, False)
    assert np.all(np.abs(got[:2] - want) <= tol)
    assert np.all(np.abs(widen(dev_to_bits(kp.pool)).reshape(ref.shape) - ref) <= ptol)      # only request 0 was appended
    kp.close()


def test_lists_out_of_order_touch_nothing_they_should_not():
    kp, lens, bt, pool, btd, sld = setup([20, 20, 20], 4, 2, 64, 13)
    q, k, v = rows(12, 4, 64, 13, 2), rows(12, 2, 64, 13, 3), rows(12, 2, 64, 13, 4)
    freq = torch.from_numpy(inv_freq(64)).cuda()
    out = torch.full((12, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    for starts in ([0, 9, 3, 12], [5, 2, 1, 0], [-4, 2, 2 ** 31 - 1, 6], [-2 ** 31, 0, 5, 2 ** 31 - 1]):
        kp.kv_append_rope(0, btd, sld, bits_to_dev(q), bits_to_dev(k), bits_to_dev(v), out, freq,
                          new_start=torch.tensor(starts, dtype=torch.int32, device="cuda"))
        kp.check_status(raise_on_error=False)
    got = dev_to_bits(kp.pool).reshape(pool.shape)
    dead = np.setdiff1d(np.arange(pool.shape[0]), bt[bt >= 0])
    assert np.array_equal(got[dead], pool[dead])
    kp.close()


def test_refusals():
    from paper_2501_08090_b200 import binding as b
    kp, lens, bt, pool, btd, sld = setup([20, 20], 4, 2, 64, 14)
    bf = dict(dtype=torch.bfloat16, device="cuda")
    q, k, v, out = torch.zeros(2, 4, 64, **bf), torch.zeros(2, 2, 64, **bf), torch.zeros(2, 2, 64, **bf), torch.zeros(2, 4, 64, **bf)
    freq = torch.ones(32, device="cuda")
    before = kp.launch_count()
    for bad in (torch.ones(4, device="cuda"), torch.ones(36, device="cuda"), torch.ones(40, device="cuda")):     # rotary 8, 72, 80
        with pytest.raises(b.CkvError) as e:
            kp.kv_append_rope(0, btd, sld, q, k, v, out, bad)
        assert e.value.code == b.CKV_EINVAL and "rotary_dim" in str(e.value)
    with pytest.raises(b.CkvError):
        kp.kv_append_rope(1, btd, sld, q, k, v, out, freq)               # layer
    three = [torch.zeros(3, h, 64, **bf) for h in (4, 2, 2, 4)]
    with pytest.raises(b.CkvError):
        kp.kv_append_rope(0, btd, sld, *three, freq)                     # 3 tokens over 2 requests
    odd = torch.zeros(2 * 4 * 64 + 8 * 64, **bf)
    with pytest.raises(b.CkvError):                                      # misaligned start
        kp.kv_append_rope(0, btd, sld, odd[1:1 + 512].view(2, 4, 64), k, v, out, freq)
    with pytest.raises(b.CkvError):                                      # stride not a multiple of 8
        kp.kv_append_rope(0, btd, sld, odd.as_strided((2, 4, 64), (260, 64, 1)), k, v, out, freq)
    with pytest.raises(b.CkvError):                                      # in place with another stride
        kp.kv_append_rope(0, btd, sld, odd[:512].view(2, 4, 64), k, v, odd.as_strided((2, 4, 64), (264, 64, 1)), freq)
    for odd_kind in (lambda t: t.to_sparse(), lambda t: torch.nested.nested_tensor([t[0], t[1]])):
        with pytest.raises(ValueError) as e:
            kp.kv_append_rope(0, btd, sld, odd_kind(q), k, v, out, freq)
        assert "q must be" in str(e.value)
        with pytest.raises(ValueError):
            kp.kv_append_rope(0, btd, sld, q, k, v, out, odd_kind(torch.ones(2, 16, device="cuda")))
    for wrong in (q.float(), q[:, :3], q.transpose(1, 2).contiguous().transpose(1, 2), q.cpu()):
        with pytest.raises(ValueError):
            kp.kv_append_rope(0, btd, sld, wrong, k, v, out, freq)
    with pytest.raises(ValueError):
        kp.kv_append_rope(0, btd, sld, q, k, v, None, freq)
    with pytest.raises(ValueError):
        kp.kv_append_rope(0, btd, sld.long(), q, k, v, out, freq)
    with pytest.raises(ValueError):
        kp.kv_append_rope(0, btd[:, :1], sld, q, k, v, out, freq)
    with pytest.raises(ValueError):
        kp.kv_append_rope(0, btd, sld, q, k, v, out, freq, new_start=torch.zeros(2, dtype=torch.int32, device="cuda"))
    none = [torch.zeros(0, h, 64, **bf) for h in (4, 2, 2, 4)]
    kp.kv_append_rope(0, btd, sld, *none, freq)                          # no tokens: nothing to do
    assert kp.launch_count() == before
    kp.close()
