"""More rows (and features) than one launch of 2^32 work items takes: rows repeat, and so do the results."""
import pytest

from paper_2601_20655_amd import binding as B

pytestmark = pytest.mark.gpu

ROWS, BASE = (1 << 26) + 37, 61


def repeat(t, n):
    """Rows 0 .. n - 1 of t over and over, without an index as large as the result."""
    import torch

    out = torch.empty((n,) + t.shape[1:], dtype=t.dtype, device=t.device)
    whole = n // len(t)
    out[:whole * len(t)].view((whole,) + t.shape).copy_(t)
    out[whole * len(t):] = t[:n - whole * len(t)]
    return out


def same(got, few):
    whole = len(got) // len(few)
    a = got[:whole * len(few)].view((whole,) + few.shape)
    assert (a == few).all().item() and (got[whole * len(few):] == few[:len(got) - whole * len(few)]).all().item()


@pytest.mark.parametrize("N", [8, 5])
def test_more_rows_than_a_launch_takes(N):
    import torch

    gen = torch.Generator(device="cuda").manual_seed(N)
    few = torch.randn((BASE, 8), generator=gen, device="cuda").bfloat16()
    x = repeat(few, ROWS)
    q = torch.full((ROWS, 16), 77, dtype=torch.int8, device="cuda")
    scale = torch.empty(ROWS, device="cuda")
    B.dit_quant_rows_forward(x[:, :N], q=q[:, :N], scale=scale)
    q0, s0 = B.dit_quant_rows_forward(few[:, :N])
    same(q[:, :N].contiguous(), q0.contiguous())
    same(scale, s0)
    assert (q[:, N:] == 77).all().item()
    back = torch.full((ROWS, 8), -5.0, dtype=torch.bfloat16, device="cuda")
    B.dit_dequant_rows_forward(q[:, :N], scale, out=back[:, :N])
    same(back[:, :N].contiguous(), B.dit_dequant_rows_forward(q0, s0).contiguous())
    assert (back[:, N:] == -5.0).all().item()
    g = 1 + 0.25 * torch.randn(N, generator=gen, device="cuda")
    B.dit_rms_norm_quant_forward(x[:, :N], g, residual=x[:, :N], h_out=back[:, :N], q=q[:, :N], scale=scale)
    q0, s0, h0 = B.dit_rms_norm_quant_forward(few[:, :N], g, residual=few[:, :N])
    same(q[:, :N].contiguous(), q0.contiguous())
    same(scale, s0)
    same(back[:, :N].contiguous(), h0.contiguous())
