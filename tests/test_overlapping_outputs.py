"""Results written over a call's own inputs are refused: blocks of one request would still be reading them."""
import pytest


@pytest.fixture(scope="module")
def b():
    from paper_2501_08090_b200 import build
    build.build()
    from paper_2501_08090_b200 import binding
    return binding


# batch 2, 3 drafts: drafts 24 bytes, tokens 32, lengths and accepted 8, u_accept 24, u_sample 8
@pytest.mark.parametrize("change", [
    dict(tokens=4096), dict(tokens=4096 + 20), dict(tokens=4096 - 28), dict(accepted=4096), dict(accepted=4096 + 20),
    dict(accepted=5120), dict(tokens=5120 - 28), dict(accepted=5120 - 4), dict(tokens=6144), dict(accepted=6144 + 20),
    dict(tokens=7168 - 28), dict(accepted=7168 + 4), dict(tokens=8192, accepted=8192 + 28), dict(tokens=8192, accepted=8192 - 4)])
def test_draft_verify(b, change):
    a = dict(batch=2, max_draft=3, vocab=100, dtype=0, drafts=4096, lens=5120, target=1 << 20, target_stride=100, draft=1 << 21,
             draft_stride=100, u_accept=6144, u_sample=7168, tokens=9216, accepted=10240, stream=None)
    a.update(change)
    assert b.lib.draft_verify(*a.values()) == b.CKV_EINVAL
    assert "overlap" in b.last_error()


@pytest.mark.gpu
def test_draft_verify_in_place_of_the_drafts(b):
    """One request whose drafts are the first entries of the tokens' array: a contiguous slice."""
    import torch
    from test_gpu_verify import make
    target, q, x, ua, us = (t.cuda() for t in make(1, 3, 500, seed=1))
    tokens, accepted = torch.zeros(1, 4, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    tokens[:, :3] = x
    with pytest.raises(b.CkvError) as e:
        b.draft_verify(tokens[:, :3], target, q, ua, us, tokens, accepted)
    assert "overlap" in str(e.value) and torch.equal(tokens[:, :3], x)
    with pytest.raises(b.CkvError):
        b.draft_verify(x, target, q, ua, us, tokens, accepted, draft_lens=accepted)
    both = torch.zeros(5, dtype=torch.int32, device="cuda")
    b.draft_verify(x, target, q, ua, us, both[:4].view(1, 4), both[4:])               # side by side is fine
    b.draft_verify(x, target, q, ua, us, tokens, accepted)
    assert both.tolist() == tokens[0].tolist() + accepted.tolist()


@pytest.mark.gpu
@pytest.mark.parametrize("width", [70, 600])                                           # one kernel scores and selects, or two
def test_page_selection(b, width):
    import torch
    from test_gpu_sparse import Case
    c = Case([900, 1000], 4, 1, 64, seed=3, width=width)
    c.update()
    pages, lens, out = c.out(9)
    n = c.kp.launch_count()
    joint = torch.zeros(2 * 9 + 2, dtype=torch.int32, device="cuda")
    for bad in (dict(lens=c.sld), dict(lens=c.btd.view(-1)[5:7]), dict(pages=c.btd.view(-1)[:18].view(2, 1, 9)),
                dict(pages=joint[:18].view(2, 1, 9), lens=joint[17:19])):
        args = {"pages": pages, "lens": lens, **bad}
        for call in (lambda: c.kp.decode_select_pages(0, c.btd, c.sld, c.qd, c.index, args["pages"], args["lens"]),
                     lambda: c.kp.decode_attention_sparse(0, c.btd, c.sld, c.qd, c.index, args["pages"], args["lens"], out)):
            with pytest.raises(b.CkvError) as e:
                call()
            assert e.value.code == b.CKV_EINVAL and "overlap" in str(e.value)
    assert c.kp.launch_count() == n
    c.kp.decode_select_pages(0, c.btd, c.sld, c.qd, c.index, joint[:18].view(2, 1, 9), joint[18:])
    c.check(9, 1, 2)
    c.close()
