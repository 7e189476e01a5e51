"""8-bit projections of more tiles than one launch takes, by tokens and by features: rows repeat, and so do the results."""
import pytest

from paper_2601_20655_amd import binding as B
from test_gpu_quant_long_calls import BASE, repeat, same

pytestmark = pytest.mark.gpu


def operands(M, N, K, gen):
    import torch

    x = torch.randint(-128, 128, (M, (K + 15) // 16 * 16), generator=gen, device="cuda", dtype=torch.int8)
    w = torch.randint(-128, 128, (N, (K + 15) // 16 * 16), generator=gen, device="cuda", dtype=torch.int8)
    return x, torch.rand(M, generator=gen, device="cuda"), w, torch.rand(N, generator=gen, device="cuda")


@pytest.mark.parametrize("M,N,K", [(540000011, 8, 16), (540000011, 5, 11), ((1 << 30) + 100, 5, 16), ((1 << 30) + 7000, 8, 11)])
def test_more_tokens_than_a_launch_takes(M, N, K):
    import torch

    gen = torch.Generator(device="cuda").manual_seed(N)
    x, xs, w, ws = operands(BASE, N, K, gen)
    bias = torch.randn(N, generator=gen, device="cuda").bfloat16()
    want = B.dit_linear_quant_forward(x[:, :K], xs, w[:, :K], ws, bias)
    y = torch.full((M, 8), 7.0, dtype=torch.bfloat16, device="cuda")
    B.dit_linear_quant_forward(repeat(x, M)[:, :K], repeat(xs, M), w[:, :K], ws, bias, out=y[:, :N])
    for at in range(0, M, BASE << 20):  # (piece by piece: less memory)
        same(y[at:at + (BASE << 20), :N].contiguous(), want.contiguous())
    assert (y[:, N:] == 7.0).all().item()


@pytest.mark.parametrize("M", [1, 2])
def test_more_features_than_a_slice_takes(M):
    import torch

    N, K = (1 << 30) + 61 * 5 + 3, 16
    gen = torch.Generator(device="cuda").manual_seed(M)
    x, xs, w, ws = operands(M, BASE, K, gen)
    bias = torch.randn(BASE, generator=gen, device="cuda").bfloat16()
    want = B.dit_linear_quant_forward(x, xs, w, ws, bias)
    y = B.dit_linear_quant_forward(x, xs, repeat(w, N), repeat(ws, N), repeat(bias, N))
    for m in range(M):
        same(y[m], want[m])
