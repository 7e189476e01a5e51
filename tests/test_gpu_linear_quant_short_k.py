"""8-bit projections whose K is less than one step of the tiles: no whole step, the cut one alone."""
import numpy as np
import pytest

import quant_ref as R
from paper_2601_20655_amd import binding as B
from test_gpu_linear_quant import operands
from test_quant_short_k_host import LENGTHS, SHORT

pytestmark = pytest.mark.gpu


def rows_in_noise(a, pad, seed):
    """a [M, K] int8 on the device; what lies between the rows is random, so that no byte of it goes unnoticed."""
    import torch

    M, K = a.shape
    gen = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.randint(-128, 128, (M, (K + 15) // 16 * 16 + pad), generator=gen, device="cuda", dtype=torch.int8)
    buf[:, :K] = torch.from_numpy(a).cuda()
    return buf[:, :K]


@pytest.mark.parametrize("i", range(len(SHORT)), ids=["%s_%dx%d" % s for s in SHORT])
def test_less_than_a_step(i):
    """Unit scales: the sums of at most 127 products of at most 2^14 are exact in fp32, and with scales of 1 bit for bit.  In 16
    bits the same numbers rounded once.  Then scales and a bias."""
    import torch

    _, M, N = SHORT[i]
    for K in LENGTHS:
        x, xs, w, ws, bias = operands(M, N, K, seed=i + K)
        xd, wd = rows_in_noise(x, 16 * (i % 3), 1), rows_in_noise(w, 16 * ((i + 1) % 3), 2)
        ones = [torch.ones(n, device="cuda") for n in (M, N)]
        per = 8
        buf = torch.full((M + 2, (N + per - 1) // per * per + 2 * per), -77.0, device="cuda")
        y = buf[1:M + 1, per:per + N]
        B.dit_linear_quant_forward(xd, ones[0], wd, ones[1], out=y)
        assert np.array_equal(y.cpu().numpy(), x.astype(np.float32) @ w.astype(np.float32).T), K
        y16 = B.dit_linear_quant_forward(xd, ones[0], wd, ones[1])
        assert torch.equal(y16, y.bfloat16()), K
        guard = buf.clone()
        guard[1:M + 1, per:per + N] = -77.0
        assert (guard == -77.0).all().item(), K
        if K in (34, 127):
            sx, sw, b = (torch.from_numpy(t).cuda() for t in (xs, ws, bias))
            B.dit_linear_quant_forward(xd, sx, wd, sw, b.bfloat16(), out=y)
            R.check_linear(y.cpu().numpy(), x, xs, w, ws, bias, False, "%dx%dx%d" % (M, N, K))


@pytest.mark.parametrize("M,N,K", [(1, 15360, 5120), (1, 20480, 5120), (16, 15360, 5120), (16, 20480, 5120), (9, 24576, 1000)])
def test_several_workgroups_a_unit(M, N, K):
    """The few rows' kernel with two or three workgroups a compute unit."""
    import torch

    x, xs, w, ws, bias = operands(M, N, K, seed=M + N)
    sx, sw, b = (torch.from_numpy(t).cuda() for t in (xs, ws, bias))
    y = B.dit_linear_quant_forward(rows_in_noise(x, 0, 3), sx, rows_in_noise(w, 16, 4), sw, b.bfloat16(), out_dtype=torch.float32)
    R.check_linear(y.cpu().numpy(), x, xs, w, ws, bias, False, "%dx%dx%d" % (M, N, K))
