"""The memory for a page selection's scores: apart from the workspace, so that a handle which never selects does
not hold it."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def b():
    from paper_2501_08090_b200 import build
    build.build()
    from paper_2501_08090_b200 import binding
    return binding


def test_the_workspace_holds_no_scores(b):
    """What a wider table adds to the workspace are the staged tables of the largest batch, 4 bytes an entry."""
    narrow, wide = (b.make_config(1, 32, 8, 128, 1000, pages, 512) for pages in (64, 8192))
    assert b.kv_workspace_bytes(wide) - b.kv_workspace_bytes(narrow) == 512 * (8192 - 64) * 4


def test_sizes_and_null_handles(b):
    assert b.kv_select_bytes(b.make_config(3, 8, 2, 128, 100, 9, 4)) == 4 * 2 * 12 * 4
    assert b.kv_select_bytes(b.make_config(1, 64, 8, 128, 100, 8192, 8192)) == 4 << 26
    assert b.kv_select_bytes(b.make_config(1, 8, 2, 96, 100, 9, 4)) == 0 and "head_dim" in b.last_error()
    assert b.lib.ckv_set_select_scratch(None, None, 0) == b.CKV_EINVAL


@pytest.mark.gpu
def test_selection_needs_room_for_its_scores(b):
    from test_gpu_sparse import Case
    c = Case([3000, 517, 90, 2048], 8, 2, 128, seed=61, width=400)
    c.update()
    c.check(20, 1, 2)
    need = 4 * 2 * 400 * 4
    assert b.kv_select_bytes(c.kp.cfg) == need
    pages, lens, out = c.out(20)
    scratch = torch.empty(need + 4, dtype=torch.uint8, device="cuda")
    assert b.lib.ckv_set_select_scratch(c.kp._h, scratch.data_ptr() + 4, need) == b.CKV_EINVAL and "aligned" in b.last_error()
    for ptr, size in ((None, need), (scratch.data_ptr(), need - 4)):
        assert b.lib.ckv_set_select_scratch(c.kp._h, ptr, size) == b.CKV_OK
        n = c.kp.launch_count()
        for call in (lambda: c.kp.decode_select_pages(0, c.btd, c.sld, c.qd, c.index, pages, lens, sink=1, recent=2),
                     lambda: c.kp.decode_attention_sparse(0, c.btd, c.sld, c.qd, c.index, pages, lens, out, sink=1, recent=2)):
            with pytest.raises(b.CkvError) as e:
                call()
            assert e.value.code == b.CKV_ENOMEM and "scratch" in str(e.value)
        assert c.kp.launch_count() == n
    # a smaller batch needs less
    c.kp.decode_select_pages(0, c.btd[:3].contiguous(), c.sld[:3].contiguous(), c.qd[:3].contiguous(), c.index, pages[:3], lens[:3])
    assert b.lib.ckv_set_select_scratch(c.kp._h, scratch.data_ptr(), need) == b.CKV_OK
    c.check(20, 1, 2)
    # neither a budget that holds every page nor few short tables write scores
    assert b.lib.ckv_set_select_scratch(c.kp._h, None, 0) == b.CKV_OK
    c.check(400, 1, 2)
    c.close()
    short = Case([3000, 517], 8, 2, 128, seed=62, width=200)
    short.update()
    want = short.out(20)
    args = (0, short.btd, short.sld, short.qd, short.index)
    short.kp.decode_attention_sparse(*args, *want)
    assert b.lib.ckv_set_select_scratch(short.kp._h, None, 0) == b.CKV_OK
    got = short.out(20)
    short.kp.decode_attention_sparse(*args, *got)
    assert all(torch.equal(x, y) for x, y in zip(want, got))
    short.close()


@pytest.mark.gpu
def test_a_first_selection_inside_a_capture(b):
    """A handle whose first selection is captured: the memory outlives the capture and other graphs."""
    from test_gpu_sparse import Case
    c = Case([3000, 517, 90, 2048], 8, 2, 128, seed=63, width=400)
    c.update()
    want = c.out(20)
    c.kp.decode_attention_sparse(0, c.btd, c.sld, c.qd, c.index, *want)
    kp = b.KvPool(c.kp.cfg, pool=c.kp.pool)
    assert kp.workspace.numel() == b.kv_workspace_bytes(kp.cfg)
    got = c.out(20)
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    for g in graphs:
        with torch.cuda.graph(g):
            kp.decode_attention_sparse(0, c.btd, c.sld, c.qd, c.index, *got)
    for g in (*graphs, *graphs):
        for t in got:
            t.zero_()
        g.replay()
        assert all(torch.equal(x, y) for x, y in zip(want, got))
    del graphs, g
    torch.cuda.empty_cache()
    filler = [torch.ones(1 << 20, device="cuda") for _ in range(8)]
    kp.decode_attention_sparse(0, c.btd, c.sld, c.qd, c.index, *got)
    assert all(torch.equal(x, y) for x, y in zip(want, got)) and all(bool((t == 1).all()) for t in filler)
    assert kp.check_status() == 0
    kp.close()
    c.close()


@pytest.mark.gpu
def test_a_first_selection_on_another_stream_takes_nothing_that_is_in_use(b):
    """Memory that was given back while work queued on the current stream still reads it."""
    from test_gpu_sparse import Case
    c = Case([3000, 517, 90, 2048], 8, 2, 128, seed=64, width=400)
    c.update()
    want = c.out(20)
    c.kp.decode_attention_sparse(0, c.btd, c.sld, c.qd, c.index, *want)
    kp, side, got = b.KvPool(c.kp.cfg, pool=c.kp.pool), torch.cuda.Stream(), c.out(20)
    held = torch.ones(b.kv_select_bytes(kp.cfg) // 4, dtype=torch.int32, device="cuda")
    copy = torch.empty_like(held)
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)
    copy.copy_(held)
    del held
    kp.decode_attention_sparse(0, c.btd, c.sld, c.qd, c.index, *got, stream=side)
    torch.cuda.synchronize()
    assert bool((copy == 1).all())
    assert all(torch.equal(x, y) for x, y in zip(want, got))
    kp.close()
    c.close()
