"""draft_verify with one row of probabilities a request: torch gives the stride of a dimension of size 1 no
meaning, the rows lie as far apart as the requests do."""
import pytest
import torch

from test_gpu_verify import make

pytestmark = pytest.mark.gpu


def verified(target, q, x, ua, us):
    from paper_2501_08090_b200 import binding as b
    tokens = torch.full((x.shape[0], x.shape[1] + 1), -9, dtype=torch.int32, device="cuda")
    accepted = torch.full((x.shape[0],), -9, dtype=torch.int32, device="cuda")
    b.draft_verify(x, target, q, ua, us, tokens, accepted)
    return tokens.tolist(), accepted.tolist()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B", [1, 7])
def test_no_drafts_and_rows_of_a_larger_array(B, dtype):
    target, _, x, ua, us = (None if t is None else t.cuda() for t in make(B, 0, 1003, seed=1, dtype=dtype, draft=False))
    want = verified(target.contiguous(), None, x, ua, us)
    steps = torch.full((B, 5, 1003), float("nan"), dtype=dtype, device="cuda")           # a sequence's positions, the last one taken
    steps[:, -1:] = target
    assert verified(steps[:, -1:], None, x, ua, us) == want
    padded = torch.full((B, 1100), float("nan"), dtype=dtype, device="cuda")             # a padded vocabulary
    padded[:, :1003] = target[:, 0]
    assert verified(padded[:, :1003].unsqueeze(1), None, x, ua, us) == want
    for stride in (0, 1, 1003, 10 ** 12):                                               # whatever the dimension of size 1 says
        assert verified(padded.as_strided((B, 1, 1003), (1100, stride, 1)), None, x, ua, us) == want


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B", [1, 7])
def test_one_draft_and_rows_of_a_larger_array(B, dtype):
    target, q, x, ua, us = (t.cuda() for t in make(B, 1, 1003, seed=2, dtype=dtype))
    want = verified(target.contiguous(), q.contiguous(), x, ua, us)
    drafted = torch.full((B, 4, 1003), float("nan"), dtype=dtype, device="cuda")
    drafted[:, 2:3] = q
    assert verified(target, drafted[:, 2:3], x, ua, us) == want
    padded = torch.full((B, 1024), float("nan"), dtype=dtype, device="cuda")
    padded[:, :1003] = q[:, 0]
    for stride in (0, 5, 1003, 10 ** 12):
        assert verified(target, padded.as_strided((B, 1, 1003), (1024, stride, 1)), x, ua, us) == want


def test_rows_on_one_another_stay_refused():
    from paper_2501_08090_b200 import binding as b
    target, q, x, ua, us = (t.cuda() for t in make(3, 1, 64, seed=3))
    for bad in (dict(target=target[:1].expand(3, 2, 64)), dict(q=q[:1].expand(3, 1, 64))):
        with pytest.raises((ValueError, b.CkvError)):
            verified(**{**dict(target=target, q=q, x=x, ua=ua, us=us), **bad})
