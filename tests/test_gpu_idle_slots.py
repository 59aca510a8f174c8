"""Requests of length 0 -- idle slots of a fixed batch -- beside long contexts, whose work is cut into even spans: their
rows are cleared and flagged, the others' are as without them, and the launch does not wait for one warp that clears them all."""
import numpy as np
import pytest
import torch

import test_gpu_cache8
import test_gpu_window
from test_gpu_cache8 import queries, tables_for, to_dev

pytestmark = pytest.mark.gpu


def attend(c, lens, q, out):
    if isinstance(c, test_gpu_window.Cache):
        c.kp.decode_attention_window(0, c.btd, lens, q, out, window=10 ** 6)
    else:
        c.kp.kv8_attention(0, c.btd, lens, q, out)


@pytest.mark.parametrize("kind", [test_gpu_cache8.Cache, test_gpu_window.Cache])
@pytest.mark.parametrize("layout,q_len,idle", [((8, 1, 128), 2, 700), ((4, 1, 64), 1, 1), ((6, 2, 64), 3, 8000), ((32, 8, 128), 1, 33)])
def test_rows_of_idle_slots(kind, layout, q_len, idle):
    rng = np.random.default_rng(1)
    B = idle + 3
    live = np.sort(rng.permutation(B)[:3])
    lens = rng.choice([0, q_len - 1, -5, 10 ** 9], B)
    lens[live] = [5000, 9000, q_len]
    bt, n = tables_for([x if i in live else 0 for i, x in enumerate(lens)], 9000, 2)
    c = kind(layout, bt, n, seed=3)
    q = queries(B, q_len, c.H, c.D, 4)
    sl = torch.tensor(lens.tolist(), dtype=torch.int32, device="cuda")
    out = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
    before = c.kp.launch_count()
    attend(c, sl, to_dev(q), out)
    assert c.kp.launch_count() - before == 2 * -(-q_len // (8 // (c.H // c.K)))          # spans and their fold, a block of tokens each
    assert c.kp.check_status(raise_on_error=False) == c.b.STATUS_BAD_LENGTH
    at = torch.from_numpy(live).cuda()
    gone = torch.ones(B, dtype=torch.bool, device="cuda")
    gone[at] = False
    assert not out[gone].any()
    c.btd, alone = c.btd[at].contiguous(), torch.empty_like(out[at])
    attend(c, sl[at].contiguous(), to_dev(q[live]), alone)
    assert c.kp.check_status() == 0 and (out[at].float() - alone.float()).abs().max() <= 2.0 ** -8 * alone.float().abs().max()      # cut at other places
    c.kp.close()


@pytest.mark.parametrize("kind", [test_gpu_cache8.Cache, test_gpu_window.Cache])
@pytest.mark.parametrize("batch,lens", [(1, [0]), (70, [0]), (2000, [0, -1]), (65, [0] * 64 + [1]), (65, [1] + [0] * 64)])
def test_all_slots_idle_or_all_but_one(kind, batch, lens):
    lens = (lens * batch)[:batch]
    bt, n = tables_for(lens, 9000, 7)
    c = kind((8, 2, 64), bt, n, seed=8)
    q = torch.zeros(batch, 8, 64, dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(q, 5.0)
    before = c.kp.launch_count()
    attend(c, torch.tensor(lens, dtype=torch.int32, device="cuda"), q, out)
    assert c.kp.launch_count() - before == 2 and c.kp.check_status(raise_on_error=False) == c.b.STATUS_BAD_LENGTH
    live = torch.tensor(lens) == 1
    assert not out[~live.cuda()].any()
    for r in torch.nonzero(live).flatten().tolist():         # one token: its value
        v = c.values(r, 1)[0, :, 1] if kind is test_gpu_cache8.Cache else c.pool[bt[r, 0], :, 1, 0]
        assert torch.equal(out[r].double().cpu(), torch.from_numpy(v).repeat_interleave(4, 0))
    c.kp.close()


@pytest.mark.parametrize("kind", [test_gpu_cache8.Cache, test_gpu_window.Cache])
def test_time_of_idle_slots(kind):
    """4000 of them, 32 heads x 128: 33 MB of zeros, 5 us at the memory's rate; one warp took 500."""
    B = 4003
    lens = [40000, 40000, 40000] + [0] * 4000
    bt, n = tables_for(lens[:1], 9000, 5)
    bt = np.concatenate([bt] * 3 + [np.full((4000, 9000), -1, np.int32)])
    c = kind((32, 8, 128), bt, n, seed=6)
    q = torch.zeros(B, 32, 128, dtype=torch.bfloat16, device="cuda")
    out, sl = torch.empty_like(q), torch.tensor(lens, dtype=torch.int32, device="cuda")

    def time(batch):
        tables, times = c.btd, []
        c.btd, args = tables[:batch], (sl[:batch], q[:batch], out[:batch])
        for _ in range(8):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            attend(c, *args)
            b.record()
            torch.cuda.synchronize()
            times.append(a.elapsed_time(b) * 1e3)
        c.btd = tables
        return min(times)

    few, many = time(3), time(B)
    print("%.1f us, with idle slots %.1f" % (few, many))
    assert many < few + 150
    c.kp.close()
