"""Page selection where long contexts lie far apart among short ones: what is chosen, and that the time of a
selection does not grow with the short requests that a warp has no work in."""
import numpy as np
import pytest
import torch

from test_gpu_sparse import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("long_at", [[0], [399], [0, 399], [31, 32, 96, 97, 330], [1, 33, 34, 200]])
@pytest.mark.parametrize("Hq,Hkv,d", [(2, 1, 64), (8, 2, 128)])
def test_long_requests_far_apart(long_at, Hq, Hkv, d):
    lens = np.random.default_rng(len(long_at)).integers(1, 16 * 9, size=400)
    for i, r in enumerate(long_at):
        lens[r] = 3000 + 700 * i
    c = Case(lens, Hq, Hkv, d, seed=40 + len(long_at), width=400)
    c.update()
    c.check(9, 1, 2, requests=sorted(set(long_at + [0, 5, 31, 63, 399])))
    c.close()


def test_time_does_not_follow_the_place_of_the_long_request():
    """One context of 8000 pages and 7999 of one page: first among them or last, the same work.  The bound is
    three times; with warps that walk over the requests behind their last tile it was twenty."""
    from paper_2501_08090_b200 import binding as b
    B, width = 8000, 8192
    kp = b.KvPool(b.make_config(1, 4, 1, 64, width, width, B))
    kp.pool.normal_()
    index = kp.make_index()
    order = torch.randperm(width, device="cuda").int()
    kp_lens = torch.full((B,), 16, dtype=torch.int32, device="cuda")
    tables = torch.zeros(B, width, dtype=torch.int32, device="cuda")
    q = torch.randn(B, 4, 64, device="cuda").to(torch.bfloat16)
    pages = torch.empty(B, 1, 64, dtype=torch.int32, device="cuda")
    lens = torch.empty(B, dtype=torch.int32, device="cuda")
    best = {}
    for place in (0, B - 1):
        kp_lens.fill_(16)
        kp_lens[place] = 8000 * 16
        tables[place] = order
        kp.kv_index_update(0, tables, kp_lens, index)
        times = []
        for _ in range(12):
            start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            start.record()
            for _ in range(8):
                kp.decode_select_pages(0, tables, kp_lens, q, index, pages, lens)
            end.record()
            torch.cuda.synchronize()
            times.append(start.elapsed_time(end))
        best[place] = min(times)
    assert kp.check_status() == 0
    assert best[0] < 3 * best[B - 1], best
    kp.close()
