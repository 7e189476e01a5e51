"""The norm with a residual whose sum is not wanted: the same 8-bit rows, and nothing else written."""
import numpy as np
import pytest

from paper_2601_20655_amd import binding as B
from test_gpu_rows_quant import check_guard, dev_rows, guarded_q, rows_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,N", [(1, 1), (3, 100), (65, 5120), (1041, 4999), (2, 20484), (27500, 5121)])
@pytest.mark.parametrize("r_bf16", [True, False])
def test_sum_not_wanted(M, N, r_bf16):
    import torch

    rng = np.random.default_rng(N)
    base = rows_of(rng, min(M, 1041), N, True), rows_of(rng, min(M, 1041), N, r_bf16)
    x, r = (dev_rows(np.resize(t, (M, N)), bf16) for t, bf16 in zip(base, (True, r_bf16)))
    g = torch.from_numpy((1 + 0.25 * rng.standard_normal(N)).astype(np.float32)).cuda()
    q0, s0, _ = B.dit_rms_norm_quant_forward(x, g, residual=r)
    keep = x.clone(), r.clone()
    q, buf = guarded_q(M, N)
    got = B.dit_rms_norm_quant_forward(x, g, residual=r, q=q, want_h=False)
    assert len(got) == 2 and torch.equal(got[0], q0) and torch.equal(got[1], s0)
    assert torch.equal(x, keep[0]) and torch.equal(r, keep[1])
    check_guard(buf, M, N)


def test_sum_given_and_not_wanted():
    import torch

    x = torch.ones((4, 64), device="cuda")
    with pytest.raises(ValueError):
        B.dit_rms_norm_quant_forward(x, residual=x, h_out=torch.empty_like(x), want_h=False)
    assert len(B.dit_rms_norm_quant_forward(x, want_h=False)) == 2 and len(B.dit_rms_norm_quant_forward(x)) == 2
