"""Rotation by angles whose cosine or sine is next to 0: it keeps its relative accuracy, in both caches' appends."""
import numpy as np
import pytest
import torch

from paper_2501_08090_b200 import binding as b

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache", [b.KvPool, b.Kv8Pool])
@pytest.mark.parametrize("n", [1, 40])
def test_cosines_and_sines_next_to_zero(cache, n):
    """Frequencies, fp32, that bring one position to within their rounding of whole quarters of a turn; n > 1: as one prompt's last rows."""
    D, half, pos = 128, 64, 4097
    kp = cache(b.make_config(1, 1, 1, D, 300, 300, 1))
    freq = np.float32(2 * np.pi * (np.arange(half) + 1) / 4 / pos)
    table = torch.arange(300, dtype=torch.int32, device="cuda").view(1, 300)
    q = torch.zeros(n, 1, D, dtype=torch.bfloat16, device="cuda")
    q[..., :half] = 1.0                                      # turned: cosines, then sines
    k = torch.zeros_like(q)
    out = torch.empty_like(q)
    sl = torch.tensor([pos + 1], dtype=torch.int32, device="cuda")
    f = torch.from_numpy(freq).cuda()
    if cache is b.KvPool:
        kp.kv_append_rope(0, table, sl, q, k, k, out, f)
    else:
        kp.kv8_append(0, table, sl, k, k, q=q, q_out=out, inv_freq=f)
    angle = (pos - np.arange(n)[::-1]).astype(np.float64)[:, None] * freq.astype(np.float64)   # 13 + 24 bits: exact
    want = np.concatenate([np.cos(angle), np.sin(angle)], 1)
    # angles of up to 101 radians: numpy's own are good to 2^-53 of themselves, the turns' two roundings to 2^-52 of 16 turns
    off, most = np.abs(out[:, 0].double().cpu().numpy() - want), np.abs(want) * (2.0 ** -8 + 2.0 ** -21) + 17 * 2 * np.pi * 2.0 ** -52
    assert np.abs(want[-1]).min() < 1e-6 and np.sum(np.abs(want[-1]) < 1e-4) >= half           # there is something to see
    assert np.all(off <= most), (off / most).max()
    assert kp.check_status() == 0
    kp.close()
