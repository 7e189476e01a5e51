"""8-bit rows as their formula has them, operation by operation in fp32: bit for bit, and how near the GELU is."""
import numpy as np
import pytest

import quant_ref as R
from paper_2601_20655_amd import binding as B
from test_gpu_rows_quant import dev_rows, rows_of

pytestmark = pytest.mark.gpu

F = np.float32


def formula(t):
    amax = np.abs(t).max(axis=1)
    inverse = F(127) * (F(1) / amax)
    return np.rint(t * inverse[:, None]).astype(np.int8), amax / F(127)


@pytest.mark.parametrize("M,N", [(5000, 1), (4000, 64), (1100, 520), (700, 1001), (65, 5121), (3, 40001)])
@pytest.mark.parametrize("bf16", [True, False])
def test_rows_are_the_formula_in_fp32(M, N, bf16):
    rng = np.random.default_rng(N)
    x = rows_of(rng, M, N, bf16)
    q, scale = B.dit_quant_rows_forward(dev_rows(x, bf16))
    want_q, want_scale = formula(x)
    assert np.array_equal(q.cpu().numpy(), want_q)
    assert np.array_equal(scale.cpu().numpy(), want_scale)


@pytest.mark.parametrize("M,N", [(4000, 64), (1100, 520), (65, 5121)])
@pytest.mark.parametrize("residual", ["none", "bf16", "f32"])
def test_norm_integers_are_the_formula_in_fp32(M, N, residual):
    import torch

    rng = np.random.default_rng(N + 1)
    x = rows_of(rng, M, N, True)
    r = None if residual == "none" else rows_of(rng, M, N, residual == "bf16")
    g = (1 + 0.25 * rng.standard_normal(N)).astype(F)
    q = B.dit_rms_norm_quant_forward(dev_rows(x, True), torch.from_numpy(g).cuda(), 1e-6,
                                     residual=None if r is None else dev_rows(r, residual == "bf16"))[0]
    assert np.array_equal(q.cpu().numpy(), formula((x if r is None else x + r) * g)[0])


@pytest.mark.parametrize("N", [1, 9, 600])
def test_gelu_is_within_its_bound(N):
    """Rows that hold one number and zeros: the scale is |gelu(x)| / 127.  The GELU is x / (1 + e), e = exp(-v), v = 2u.  An
    error of d in v changes 1 / (1 + e) by d e / (1 + e)^2 = (d / v) (v e / (1 + e)^2), the last factor at most 0.23; d / v is at most
    nine roundings (x x, the sum, its product with x, six in the constants).  The exponential and the reciprocal (an ulp, two
    roundings, each), the sum and the product: six more.  Nine units of 2^-24 of |x| in all; the header says sixteen.  And
    one for the quotient by 127."""
    rng = np.random.default_rng(N)
    x = np.concatenate([np.linspace(-9, 9, 4001), np.exp(rng.uniform(-60, 60, 1000)), -np.exp(rng.uniform(-60, 2, 1000))]).astype(F)
    rows = np.zeros((len(x), N), F)
    rows[np.arange(len(x)), rng.integers(0, N, len(x))] = x
    _, scale = B.dit_quant_rows_forward(dev_rows(rows, False), act="gelu")
    got, want = scale.cpu().numpy().astype(np.float64) * 127, np.abs(R.gelu(x.astype(np.float64)))
    assert np.all(np.abs(got - want) <= 16 * R.U * np.abs(x) + R.U * want + 2.0 ** -120)
