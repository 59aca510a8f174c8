"""The operators together, as a self-speculative decode step uses them: rotated prompts enter the
cache, its pages are indexed, tokens are drafted with page-sparse attention, checked in one multi-token
pass over the whole context, and verified; rejected drafts are overwritten by the next step."""
import numpy as np
import pytest
import torch

from oracle import oracle
from oracle.oracle import PoolShape
from paper_2501_08090_b200 import workloads as wl

import ref_ops
from helpers import assert_close, bits_to_dev, dev_to_bits, widen

pytestmark = pytest.mark.gpu

HQ, HKV, D, V, DRAFTS = 8, 2, 64, 211, 3


class Model:
    """One attention layer between an embedding and a vocabulary projection (random weights)."""

    def __init__(self, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.embed = torch.randn(V, (HQ + 2 * HKV) * D, generator=g, device="cuda").to(torch.bfloat16)
        self.head = 0.6 * torch.randn(HQ * D, V, generator=g, device="cuda")
        self.freq = (10000.0 ** (-torch.arange(D // 2, device="cuda") / (D // 2))).float()

    def qkv(self, tokens):
        x = self.embed[tokens.long()].view(-1, HQ + 2 * HKV, D)
        return x[:, :HQ], x[:, HQ:HQ + HKV], x[:, HQ + HKV:]

    def probs(self, attended):
        return torch.softmax(attended.float().flatten(-2) @ self.head, -1)


def test_self_speculative_decoding_step_by_step():
    from paper_2501_08090_b200 import binding as b
    model = Model(1)
    prompt = [700, 45, 333, 1]
    B, steps = len(prompt), 14
    room = [n + steps * (DRAFTS + 1) + DRAFTS for n in prompt]
    pages = sum(-(-n // 16) for n in room) + 2
    bt = wl.block_tables(np.array(room, dtype=np.int32), pages, 3)
    cfg = b.make_config(1, HQ, HKV, D, pages, bt.shape[1], B)
    kp = b.KvPool(cfg)
    kp.pool.fill_(float("nan"))                                       # slots that nothing wrote stay visible
    index = kp.make_index()
    btd = torch.from_numpy(bt).cuda()
    gen = torch.Generator(device="cuda").manual_seed(2)
    text = [torch.randint(0, V, (n,), generator=gen, device="cuda").tolist() for n in prompt]

    # prompts, all but their last token
    fed = [t[:-1] for t in text]
    flat = torch.tensor([x for t in fed for x in t], device="cuda")
    start = torch.tensor([0] + [len(t) for t in fed], device="cuda").cumsum(0).to(torch.int32)
    lens = torch.tensor([max(1, len(t)) for t in fed], dtype=torch.int32, device="cuda")
    q, k, v = model.qkv(flat)
    kp.kv_append_rope(0, btd, lens, q, k, v, torch.empty_like(q), model.freq, new_start=start)
    have = torch.tensor([len(t) for t in fed], dtype=torch.int32, device="cuda")

    budget = 8
    picked = torch.empty(B, HKV, budget, dtype=torch.int32, device="cuda")
    picked_lens = torch.empty(B, dtype=torch.int32, device="cuda")
    last = torch.tensor([t[-1] for t in text], dtype=torch.int32, device="cuda")
    kp.kv_index_update(0, btd, (have + 1).int(), index)               # position `have` is not written yet: NaN there is no matter, its page is recent
    total_accepted = 0
    for step in range(steps):
        drafts, draft_p = [], []
        token = last
        for i in range(DRAFTS):                                       # sparse drafting, one token at a time
            now = (have + 1 + i).int()
            q, k, v = model.qkv(token)
            turned = torch.empty(B, HQ, D, dtype=torch.bfloat16, device="cuda")
            kp.kv_append_rope(0, btd, now, q, k, v, turned, model.freq)
            kp.kv_index_update(0, btd, now, index, last_tokens=1)
            out = torch.empty(B, HQ, D, dtype=torch.bfloat16, device="cuda")
            kp.decode_attention_sparse(0, btd, now, turned, index, picked, picked_lens, out, sink=1, recent=2)
            p = model.probs(out)
            token = torch.multinomial(p, 1, generator=gen)[:, 0].int()
            drafts.append(token)
            draft_p.append(p)
        drafts = torch.stack(drafts, 1).contiguous()
        # the whole-context pass over the last accepted token and the drafts
        now = (have + DRAFTS + 1).int()
        q, k, v = model.qkv(torch.cat((last[:, None], drafts), 1).flatten())
        turned = torch.empty(B * (DRAFTS + 1), HQ, D, dtype=torch.bfloat16, device="cuda")
        kp.kv_append_rope(0, btd, now, q, k, v, turned, model.freq)
        kp.kv_index_update(0, btd, now, index, last_tokens=DRAFTS + 1)
        out = torch.empty_like(turned)
        kp.decode_attention_multi(0, DRAFTS + 1, btd, now, turned, out)
        target = model.probs(out).view(B, DRAFTS + 1, V)
        ua, us = torch.rand(B, DRAFTS, generator=gen, device="cuda"), torch.rand(B, generator=gen, device="cuda")
        tokens = torch.empty(B, DRAFTS + 1, dtype=torch.int32, device="cuda")
        accepted = torch.empty(B, dtype=torch.int32, device="cuda")
        stacked = torch.stack(draft_p, 1).contiguous()
        b.draft_verify(drafts, target.contiguous(), stacked, ua, us, tokens, accepted)
        assert kp.check_status() == 0

        # every part against its definition: attention over what the pool holds, verification of the given rows
        pool = dev_to_bits(kp.pool)
        ref = oracle.decode_attention_multi(pool, PoolShape(1, pages, HQ, HKV, 16, D), 0, DRAFTS + 1, bt, now.cpu().numpy(),
                                            dev_to_bits(turned).reshape(B, DRAFTS + 1, HQ, D))
        assert_close(dev_to_bits(out).reshape(ref.shape), ref, "step %d" % step)
        got = tokens.tolist()
        for r in range(B):
            n, want = ref_ops.verify(drafts[r].tolist(), target[r].double().cpu().numpy(), stacked[r].double().cpu().numpy(),
                                     ua[r].tolist(), float(us[r]))
            assert int(accepted[r]) == n and got[r] == want + [-1] * (DRAFTS + 1 - len(want))
            text[r] += want
        total_accepted += int(accepted.sum())
        have = (have + 1 + accepted).int()
        last = torch.tensor([t[-1] for t in text], dtype=torch.int32, device="cuda")
    assert total_accepted > 0

    # the cache holds exactly the accepted text, each key at its own position
    pool = widen(dev_to_bits(kp.pool)).reshape(pages, HKV, 2, 16, D)
    for r in range(B):
        _, k, v = model.qkv(torch.tensor(text[r][:-1], device="cuda"))
        assert len(text[r]) - 1 == int(have[r])
        for pos in sorted({0, 1, prompt[r], int(have[r]) // 2, int(have[r]) - 1} & set(range(int(have[r])))):
            want, size = ref_ops.rotate(k[pos].double().cpu().numpy(), pos, model.freq.cpu().numpy(), False)
            page, slot = bt[r][pos // 16], pos % 16
            delta = 2.0 ** -21 * size
            assert np.all(np.abs(pool[page, :, 0, slot] - want) <= 2.0 ** -8 * (np.abs(want) + delta) + delta)
            assert np.array_equal(pool[page, :, 1, slot], v[pos].double().cpu().numpy())
    # and the index its keys' bounds, page by page, as if built at once
    fresh = kp.make_index()
    kp.kv_index_update(0, btd, have, fresh)
    kp.kv_index_update(0, btd, have, index, last_tokens=DRAFTS + 16)
    for r in range(B):
        ids = torch.from_numpy(bt[r][:(int(have[r]) + 15) // 16].astype(np.int64)).cuda()
        n = pages * HKV * 2 * D
        for view in (lambda t: t[:n].view(pages, -1), lambda t: t[n:].view(pages, -1)):
            assert torch.equal(view(fresh)[ids], view(index)[ids])
    kp.close()
