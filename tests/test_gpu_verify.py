"""Verification of drafted tokens against the definition in 64 bits: accepted counts and tokens exactly."""
import numpy as np
import pytest
import torch

import ref_ops

pytestmark = pytest.mark.gpu


def make(B, K, V, seed, dtype=torch.float32, draft=True, pad=0, sharp=2.0):
    g = torch.Generator().manual_seed(seed)
    logits = sharp * torch.randn(B, K + 1, V, generator=g)
    stride = V + pad
    target, q = torch.full((B, K + 1, stride), float("nan")).to(dtype), None
    target[..., :V] = torch.softmax(logits, -1).to(dtype)
    tilted = torch.softmax(logits[:, :K] + 0.7 * torch.randn(B, K, V, generator=g), -1)
    if draft:
        q = torch.full((B, K, stride), float("nan")).to(dtype)
        q[..., :V] = tilted.to(dtype)
    x = torch.multinomial(tilted.reshape(-1, V), 1, generator=g).view(B, K).int() if K else torch.zeros(B, 0, dtype=torch.int32)
    return target[..., :V], None if q is None else q[..., :V], x, torch.rand(B, K, generator=g), torch.rand(B, generator=g)


def on_gpu(t):
    """The tensor on the GPU with its strides."""
    if t is None:
        return None
    base = torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device="cuda") if t.numel() else t.cuda()
    base.copy_(t)
    return base


def check(target, q, x, ua, us, draft_lens=None):
    from paper_2501_08090_b200 import binding as b
    B, K = x.shape
    tokens = torch.full((B, K + 1), -9, dtype=torch.int32, device="cuda")
    accepted = torch.full((B,), -9, dtype=torch.int32, device="cuda")
    b.draft_verify(x.cuda(), on_gpu(target), on_gpu(q), ua.cuda(), us.cuda(), tokens, accepted,
                   draft_lens=None if draft_lens is None else torch.tensor(draft_lens, dtype=torch.int32, device="cuda"))
    tokens, accepted = tokens.tolist(), accepted.tolist()
    p64, q64 = target.double().numpy(), None if q is None else q.double().numpy()
    for r in range(B):
        n = K if draft_lens is None else min(max(draft_lens[r], 0), K)
        want_n, want = ref_ops.verify(x[r, :n], p64[r, :n + 1], None if q64 is None else q64[r, :n], ua[r], us[r])
        assert accepted[r] == want_n and tokens[r] == want + [-1] * (K + 1 - len(want)), (r, tokens[r], want)
    return tokens, accepted


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("V", [1, 2, 31, 128, 1000, 4099, 32000, 50257, 128256])
def test_vocabularies(V, draft, dtype):
    check(*make(6, 3, V, seed=V, dtype=dtype, draft=draft))


@pytest.mark.parametrize("B", [1, 2, 5, 40, 300])
@pytest.mark.parametrize("K", [0, 1, 7, 33, 70])
def test_batches_and_draft_lengths(B, K):
    V = 517 if B * K > 2000 else 8200
    check(*make(B, K, V, seed=B * 100 + K, draft=(B + K) % 2 == 0))
    if K:
        lens = [int(i) for i in np.random.default_rng(K).integers(-1, K + 2, size=B)]
        check(*make(B, K, V, seed=B * 100 + K + 50), draft_lens=lens)


@pytest.mark.parametrize("dtype,pad", [(torch.float32, 4), (torch.float32, 3), (torch.bfloat16, 8), (torch.bfloat16, 5)])
def test_rows_apart(dtype, pad):
    """Padded rows (the padding is NaN), on aligned strides and on others."""
    check(*make(9, 4, 6000, seed=pad, dtype=dtype, pad=pad))


def test_rows_far_apart():
    """Rows 2^29 elements apart: offsets beyond 32 bits."""
    target, q, x, ua, us = make(2, 2, 300, seed=21, dtype=torch.bfloat16)
    far = torch.empty(5 * 2 ** 29 + 2 ** 10, dtype=torch.bfloat16, device="cuda")
    p_far = far.as_strided((2, 3, 300), (3 * 2 ** 29, 2 ** 29, 1))
    q_far = far[512:].as_strided((2, 2, 300), (2 * 2 ** 29, 2 ** 29, 1))
    p_far.copy_(target); q_far.copy_(q)
    from paper_2501_08090_b200 import binding as b
    for u in (ua, torch.zeros_like(ua), torch.ones_like(ua)):
        tokens, accepted = torch.empty(2, 3, dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
        b.draft_verify(x.cuda(), p_far, q_far, u.cuda(), us.cuda(), tokens, accepted)
        want = check(target, q, x, u, us)
        assert tokens.tolist() == want[0] and accepted.tolist() == want[1]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [7, 8, 33, 256, 2049, 9000])
def test_rows_of_every_alignment(V, dtype):
    """Target and draft rows that start at every offset within 16 bytes, each against each."""
    target, q, x, ua, us = make(3, 2, V, seed=V, dtype=dtype)
    from paper_2501_08090_b200 import binding as b
    want = check(target, q, x, ua, us)
    step = 16 // target.element_size()
    dev = [t.cuda() for t in (x, ua, us)]
    stride = (V + 2 * step - 1) // step * step                             # every row at the same offset

    def place(t, off):
        base = torch.full((t.shape[0] * t.shape[1] * stride + 2 * step,), float("nan"), dtype=dtype, device="cuda")
        rows = base[off:].as_strided(t.shape, (t.shape[1] * stride, stride, 1))
        rows.copy_(t)
        return rows

    for i in range(step):
        for j in range(step):
            tokens, accepted = torch.empty(3, 3, dtype=torch.int32, device="cuda"), torch.empty(3, dtype=torch.int32, device="cuda")
            b.draft_verify(dev[0], place(target, i), place(q, j), dev[1], dev[2], tokens, accepted)
            assert tokens.tolist() == want[0] and accepted.tolist() == want[1], (i, j)


def test_infinite_weights():
    """An infinity in the deciding row gives -1; in the draft's row it only refuses its own token."""
    V = 500
    p, q = torch.full((3, 2, V), 1.0 / V), torch.full((3, 1, V), 0.5 / V)
    x = torch.full((3, 1), 4, dtype=torch.int32)
    ua = torch.tensor([[0.5], [0.999999], [0.5]])
    p[0, 1, 77] = float("inf")                                             # accepted; the next row decides
    p[1, 0, 77] = float("inf")
    q[1, 0, 4] = 1.0                                                       # refused
    q[2, 0, 4] = float("inf")
    q[2, 0, 5:] = 1.0                                                      # refused; tokens 0 .. 3 remain
    from paper_2501_08090_b200 import binding as b
    tokens, accepted = torch.empty(3, 2, dtype=torch.int32, device="cuda"), torch.empty(3, dtype=torch.int32, device="cuda")
    b.draft_verify(x.cuda(), p.cuda(), q.cuda(), ua.cuda(), torch.tensor([0.5, 0.5, 0.6]).cuda(), tokens, accepted)
    assert tokens.tolist() == [[4, -1], [-1, -1], [2, -1]] and accepted.tolist() == [1, 0, 0]


def test_every_border_of_a_small_distribution():
    """Eighths: each draw's goal falls on a border exactly, or half a step beside it."""
    V = 8
    p = torch.full((17, 1, V), 0.125)
    us = torch.tensor([i / 16 for i in range(16)] + [1 - 2.0 ** -24])
    tokens, _ = check(p, None, torch.zeros(17, 0, dtype=torch.int32), torch.zeros(17, 0), us)
    assert [t[0] for t in tokens] == [i // 2 for i in range(16)] + [7]


def test_the_draw_is_exact_over_a_long_flat_row():
    """2^17 equal weights and one heavy tail: sums in 32 bits would be off by many tokens."""
    V = 131072
    p = torch.full((64, 1, V), 1.0 / V)
    p[:, :, -1] = 0.25
    us = torch.rand(64, generator=torch.Generator().manual_seed(1))
    check(p, None, torch.zeros(64, 0, dtype=torch.int32), torch.zeros(64, 0), us)


def test_degenerate_rows():
    V, B = 300, 9
    p, q = torch.zeros(B, 2, V), torch.zeros(B, 1, V)
    x = torch.full((B, 1), 5, dtype=torch.int32)
    ua, us = torch.full((B, 1), 0.5), torch.full((B,), 0.5)
    p[0, :, 7] = 1; q[0, 0, 5] = 1                 # disjoint point masses: refused, 7 is drawn
    p[1, :, 5] = 1; q[1, 0, 5] = 1                 # the same point mass: accepted, 5 again
    p[2, 0, 5] = q[2, 0, 5] = 0.25; ua[2] = 1.0    # refused although p = q: nothing is left, drawn from p
    p[3, 0, 5] = 0.1; q[3, 0, 5] = 0.2; ua[3] = 0.9   # p below q everywhere: drawn from p
    p[5, 0, :] = float("nan"); q[5, 0, 5] = 1      # NaN: refused, a row without weight
    p[6, 0, 200] = float("nan"); p[6, 0, 201] = 0.5; q[6, 0, 5] = 1
    p[7, :, 299] = 1e-38; q[7, 0, 5] = 1           # the last token, a tiny weight
    p[8, 0, :] = 0.5; q[8, 0, :] = 0.25; us[8] = float("nan")      # accepted; the next row is empty
    tokens, accepted = check(p, q, x, ua, us)
    assert tokens[0] == [7, -1] and tokens[1] == [5, 5] and tokens[2] == [5, -1] and tokens[3] == [5, -1]
    assert tokens[4] == [-1, -1] and tokens[5] == [-1, -1] and tokens[6] == [201, -1] and tokens[7] == [299, -1]
    assert tokens[8] == [5, -1]


@pytest.mark.parametrize("draft", [True, False])
def test_drafts_outside_the_vocabulary_are_refused(draft):
    target, q, x, ua, us = make(4, 2, 100, seed=3, draft=draft)
    x[0, 0], x[1, 0], x[2, 1], x[3, 1] = -1, 100, 2 ** 31 - 1, -2 ** 31
    ua[:] = 0
    tokens, accepted = check(target, q, x, ua, us)
    assert accepted == [0, 0, 1, 1]


def test_results_follow_the_targets_distribution():
    """The point of the rule: whatever the draft, the first token is distributed as the target's.  20000 draws
    over 6 tokens; each count within 5 standard deviations."""
    N, V = 20000, 6
    g = torch.Generator().manual_seed(2)
    p = torch.tensor([0.05, 0.3, 0.15, 0.2, 0.25, 0.05])
    q = torch.tensor([0.4, 0.1, 0.1, 0.1, 0.1, 0.2])
    x = torch.multinomial(q.expand(N, V), 1, generator=g).int()
    from paper_2501_08090_b200 import binding as b
    tokens = torch.empty(N, 2, dtype=torch.int32, device="cuda")
    accepted = torch.empty(N, dtype=torch.int32, device="cuda")
    b.draft_verify(x.cuda(), p.expand(N, 2, V).contiguous().cuda(), q.expand(N, 1, V).contiguous().cuda(),
                   torch.rand(N, 1, generator=g).cuda(), torch.rand(N, generator=g).cuda(), tokens, accepted)
    count = torch.bincount(tokens[:, 0].long().cpu(), minlength=V).double()
    sigma = (N * p.double() * (1 - p.double())).sqrt()
    assert ((count - N * p.double()).abs() <= 5 * sigma).all()


def test_captured_and_on_another_stream():
    from paper_2501_08090_b200 import binding as b
    target, q, x, ua, us = (t.cuda() for t in make(5, 3, 20000, seed=4))
    want = [torch.empty(5, 4, dtype=torch.int32, device="cuda"), torch.empty(5, dtype=torch.int32, device="cuda")]
    got = [torch.empty_like(t) for t in want]
    b.draft_verify(x, target, q, ua, us, *want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    b.draft_verify(x, target, q, ua, us, *got, stream=side)
    side.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.draft_verify(x, target, q, ua, us, *got)
    keep = ua.clone()
    ua.fill_(1.0)
    graph.replay()
    assert not torch.equal(want[1], got[1])
    ua.copy_(keep)
    for _ in range(20):
        graph.replay()
    assert all(torch.equal(a, c) for a, c in zip(want, got))


def test_refusals():
    from paper_2501_08090_b200 import binding as b
    target, q, x, ua, us = (t.cuda() for t in make(2, 3, 64, seed=5))
    tokens, accepted = torch.zeros(2, 4, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    for bad in (dict(target_probs=target.half()), dict(draft_probs=q.bfloat16()), dict(target_probs=target[:, :3]),
                dict(draft_probs=q[:, :, :32]), dict(target_probs=target.transpose(1, 2).contiguous().transpose(1, 2)),
                dict(draft_tokens=x.long()), dict(u_accept=ua.double()), dict(u_sample=us[:1]), dict(tokens=tokens[:, :3]),
                dict(accepted=accepted.cpu()), dict(draft_lens=torch.zeros(3, dtype=torch.int32, device="cuda"))):
        args = dict(draft_tokens=x, target_probs=target, draft_probs=q, u_accept=ua, u_sample=us, tokens=tokens, accepted=accepted)
        args.update(bad)
        with pytest.raises(ValueError):
            b.draft_verify(**args)
    assert not tokens.any()
