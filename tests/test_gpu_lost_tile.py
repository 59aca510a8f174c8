"""A warp whose wait for a tile has run out must not leave a row of the output as an earlier call left it: it writes NaN.
No wait runs out here: a kernel of one warp takes the attention kernels' own last step with `alive` false and true."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2501_08090_b200 import build

pytestmark = pytest.mark.gpu

SOURCE = """
#include "ckv_cache_attn.cuh"

template <int D, bool k8>
__global__ void last_step(ckv::CacheAttnParams p, bool alive)
{
    ckv::PairPart<D, k8> part;
    part.m0 = part.m1 = 3.f;
    part.l0 = part.l1 = 2.f;
    for (int c = 0; c < D / 16; ++c)
        for (int i = 0; i < 4; ++i) part.o[c][i] = k8 ? 64.f : 2.f;     // an 8-bit part's l is kept 2^-5 smaller
    part.store_out(p, 1, 1, threadIdx.x, alive);
}

// out: 2 requests, 2 new tokens, 2 kv heads of 3 heads each
extern "C" int run(int d, int k8, int alive, void *out)
{
    ckv::CacheAttnParams p{};
    p.out = (uint16_t *)out;
    p.q_len = p.q_pass = 2;
    p.num_kv_heads = 2;
    p.group = 3;
    if (d == 64) k8 ? last_step<64, true><<<1, 32>>>(p, alive) : last_step<64, false><<<1, 32>>>(p, alive);
    else k8 ? last_step<128, true><<<1, 32>>>(p, alive) : last_step<128, false><<<1, 32>>>(p, alive);
    return cudaDeviceSynchronize();
}
"""


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    at = tmp_path_factory.mktemp("last_step")
    (at / "last_step.cu").write_text(SOURCE)
    subprocess.run([build._nvcc()] + build.NVCC_FLAGS + ["-o", str(at / "last_step.so"), str(at / "last_step.cu")], check=True, capture_output=True)
    return ctypes.CDLL(os.fspath(at / "last_step.so")).run


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("k8", [0, 1])
def test_rows_are_nan_where_tiles_were_lost(run, d, k8):
    for alive, value in ((1, 1.0), (0, float("nan"))):
        out = torch.full((2, 2, 6, d), 9.0, dtype=torch.bfloat16, device="cuda")
        want = out.float()
        want[1, :, 3:] = value
        torch.cuda.synchronize()
        assert run(d, k8, alive, ctypes.c_void_p(out.data_ptr())) == 0
        assert torch.equal(out.float().nan_to_num(7.0), want.nan_to_num(7.0)) and torch.equal(out.isnan(), want.isnan())
