"""Keys with an infinity: a score of minus infinity is a weight of 0, wherever in the context it lies and
however the context is split over warps, CTAs and launches."""
import numpy as np
import pytest
import torch

import ref_ops
from helpers import assert_close, bits_to_dev, dev_to_bits, widen
from paper_2501_08090_b200 import workloads as wl

pytestmark = pytest.mark.gpu

CHANNEL = 5


def away(kind, L):
    """Which of the context's tokens score minus infinity."""
    i = np.arange(L)
    return {"last token": i == L - 1, "first tile": i < 32, "all but the last token": i < L - 1, "every other tile": i // 32 % 2 == 0,
            "all but one in the middle": i != L // 2, "none": i < 0}[kind] & (L > 1)


KINDS = ["last token", "first tile", "all but the last token", "every other tile", "all but one in the middle", "none"]


class Batch:
    """Contexts of which some tokens' keys hold -inf in a channel where every query is positive, or +inf where
    every query is negative."""

    def __init__(self, kind, Hq, Hkv, d, seed, lens=(1, 33, 32, 65, 100, 1000, 4001)):
        from paper_2501_08090_b200 import binding as b
        rng = np.random.default_rng(seed)
        self.Hq, self.Hkv, self.d, self.lens = Hq, Hkv, d, np.array(lens, dtype=np.int32)
        pages = int(wl.pages_of(self.lens).sum()) + 2
        self.bt = wl.block_tables(self.lens, pages, seed)
        self.pool = wl.normal_bf16((pages, Hkv, 2, 16, d), seed, 1)
        self.q = wl.normal_bf16((len(lens), Hq, d), seed, 2)
        for r, L in enumerate(lens):
            negative = rng.random(Hkv) < 0.5
            for h in range(Hkv):
                rows = slice(h * Hq // Hkv, (h + 1) * Hq // Hkv)
                self.q[r, rows, CHANNEL] = 0xbf80 if negative[h] else 0x3f80
                for t in np.nonzero(away(kind, L))[0]:
                    self.pool[self.bt[r][t // 16], h, 0, t % 16, CHANNEL] = 0x7f80 if negative[h] else 0xff80
        cfg = b.make_config(1, Hq, Hkv, d, pages, self.bt.shape[1], len(lens))
        self.kp = b.KvPool(cfg, pool=bits_to_dev(self.pool.reshape(-1)))
        self.btd, self.sld, self.qd = torch.from_numpy(self.bt).cuda(), torch.from_numpy(self.lens).cuda(), bits_to_dev(self.q)
        self.out = torch.full((len(lens), Hq, d), float("nan"), dtype=torch.bfloat16, device="cuda")

    def check(self, what, pages_of=None):
        pool, q, G = widen(self.pool), widen(self.q), self.Hq // self.Hkv
        assert self.kp.check_status() == 0
        for r, L in enumerate(int(x) for x in self.lens):
            for h in range(self.Hkv):
                pages = [int(x) for x in self.bt[r][:-(-L // 16)]] if pages_of is None else pages_of(r, h)
                tokens = L - 16 * (-(-L // 16) - len(pages))
                with np.errstate(invalid="ignore"):
                    ref = ref_ops.attend(pool, pages, tokens, q[r, h * G:(h + 1) * G], h)
                if np.isnan(ref).all():                              # no token has any weight: 0 / 0, as by the formula
                    assert torch.isnan(self.out[r, h * G:(h + 1) * G]).all(), (what, r, h)
                    continue
                assert_close(dev_to_bits(self.out[r, h * G:(h + 1) * G]), ref, "%s: request %d kv head %d" % (what, r, h))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("Hq,Hkv,d", [(8, 2, 128), (4, 1, 64), (14, 2, 128)])
def test_over_page_lists(kind, Hq, Hkv, d):
    """Whole contexts as lists: one CTA to a cluster a pair."""
    c = Batch(kind, Hq, Hkv, d, seed=31)
    for budget in (c.bt.shape[1], c.bt.shape[1] + 700):
        lists = torch.full((len(c.lens), Hkv, budget), -1, dtype=torch.int32, device="cuda")
        lists[:, :, :c.bt.shape[1]] = c.btd.unsqueeze(1)
        c.out.fill_(float("nan"))
        c.kp.decode_attention_pages(0, lists, c.sld, c.qd, c.out)
        c.check("budget %d" % budget)
    c.kp.close()


@pytest.mark.parametrize("kind", ["last token", "all but the last token", "every other tile"])
@pytest.mark.parametrize("lens", [(1000, 333, 16 * 21 + 1), (4001, 1000, 16 * 201 + 1)])        # one kernel selects and attends, or three
def test_selected_by_their_bounds(kind, lens):
    """Attention over selected pages, pages with an infinity among them."""
    c = Batch(kind, 8, 2, 128, seed=32, lens=lens)
    index = c.kp.make_index()
    c.kp.kv_index_update(0, c.btd, c.sld, index)
    pages = torch.empty(len(lens), 2, 20, dtype=torch.int32, device="cuda")
    got_lens = torch.empty(len(lens), dtype=torch.int32, device="cuda")
    c.kp.decode_attention_sparse(0, c.btd, c.sld, c.qd, index, pages, got_lens, c.out, sink=1, recent=2)
    chosen = pages.cpu().numpy()
    c.check("sparse", lambda r, h: [int(x) for x in chosen[r, h] if x >= 0])
    c.kp.close()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("Hq,Hkv,d", [(8, 2, 128), (4, 1, 64), (14, 2, 128)])
def test_over_whole_contexts(kind, Hq, Hkv, d):
    """decode_attention with the context whole in one warp, in a CTA, and cut over many."""
    c = Batch(kind, Hq, Hkv, d, seed=33)
    default = c.kp.get_partition()
    for spans in (default, 1, 3, 100):
        c.kp.set_partition(spans)
        c.out.fill_(float("nan"))
        c.kp.decode_attention(0, c.btd, c.sld, c.qd, c.out)
        c.check("%d spans" % spans)
    c.kp.close()


@pytest.mark.parametrize("kind", KINDS)
def test_of_a_fused_step(kind):
    """decode_step, whose new key is the last token's."""
    c = Batch(kind, 8, 2, 128, seed=34)
    pool = c.kp.pool_view()[0]
    last = [(int(c.bt[r][(L - 1) // 16]), (int(L) - 1) % 16) for r, L in enumerate(c.lens)]
    k, v = (torch.stack([pool[p, :, kv, s] for p, s in last]).contiguous() for kv in (0, 1))
    for p, s in last:
        pool[p, :, :, s] = float("nan")                                  # the step stores it
    torch.cuda.synchronize()
    c.kp.decode_step(0, c.btd, c.sld, c.qd, k, v, c.out)
    c.check("decode_step")
    c.kp.close()


@pytest.mark.parametrize("q_len", [2, 5])
@pytest.mark.parametrize("kind", ["first tile", "every other tile", "none"])
def test_of_several_new_tokens(kind, q_len):
    """decode_attention_multi: each new token's own context."""
    lens = (65, 100, 1000, 4001)
    c = Batch(kind, 8, 2, 128, seed=35, lens=lens)
    q = wl.normal_bf16((len(lens), q_len, 8, 128), 35, 3)
    q[..., CHANNEL] = c.q[:, None, :, CHANNEL]
    out = torch.full((len(lens), q_len, 8, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    c.kp.decode_attention_multi(0, q_len, c.btd, c.sld, bits_to_dev(q), out)
    assert c.kp.check_status() == 0
    pool, q = widen(c.pool), widen(q)
    for r, L in enumerate(lens):
        pages = [int(x) for x in c.bt[r][:-(-L // 16)]]
        for i in range(q_len):
            for h in range(2):
                ref = ref_ops.attend(pool, pages, L - q_len + 1 + i, q[r, i, h * 4:h * 4 + 4], h)
                assert_close(dev_to_bits(out[r, i, h * 4:h * 4 + 4]), ref, "request %d token %d kv head %d" % (r, i, h))
    c.kp.close()
