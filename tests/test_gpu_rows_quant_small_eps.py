"""The norm's 8-bit rows where eps does not outweigh what is lost of small squares (bounds: quant_ref.check_rows and
norm_scale_rel), eps = 0 included."""
import numpy as np
import pytest

import quant_ref as R
from paper_2601_20655_amd import binding as B
from paper_2601_20655_amd import workloads as wl
from test_gpu_rows_quant import check_guard, dev_rows, guarded_q, rows_of

pytestmark = pytest.mark.gpu

# magnitudes of rows: squares that are ordinary, denormal and zero in fp32, down to numbers that are denormal themselves
GAINS = np.array([1.0, 1e-4, 1e15, 1e-18, 1e-20, 1e-22, 1e-25, 1e-30, 1e-37, 1e-39, 1e-41, 3e-44], dtype=np.float64)
EPS = [0.0, 1e-45, 1e-38, 2.0 ** -110, 2.0 ** -101, 2.0 ** -100, 1e-12]


def rows_of_gains(rng, M, N, bf16):
    x = (rng.standard_normal((M, N)) * GAINS[np.arange(M) % len(GAINS)][:, None]).astype(np.float32)
    x[:, rng.random(N) < 0.01] *= 20
    return wl.bf16_bits_to_f32(wl.f32_to_bf16_bits(x)) if bf16 else x


def counts(t, eps):
    """Rows that do not count as zeros.  From eps = 2^-100 on they are those whose max |t| is 2^-120 or more."""
    return np.abs(t).max(axis=1) >= 2.0 ** -120 if eps >= 2.0 ** -100 else np.abs(t).max(axis=1) > 0


@pytest.mark.parametrize("M,N", [(12, 1), (13, 8), (24, 77), (12, 512), (25, 1001), (12, 2056), (36, 5120), (12, 20484), (12, 65536),
                                 (1031, 520), (1025, 4999)])
@pytest.mark.parametrize("x_bf16,residual,gamma", [(False, "none", False), (True, "none", True), (True, "bf16", True),
                                                   (True, "f32", True), (False, "f32", False)])
def test_small_eps(M, N, x_bf16, residual, gamma):
    import torch

    rng = np.random.default_rng(17 * N + M)
    x = rows_of_gains(rng, M, N, x_bf16)
    r = None if residual == "none" else rows_of_gains(rng, M, N, residual == "bf16")
    g = (1 + 0.25 * rng.standard_normal(N)).astype(np.float32) if gamma else None
    for eps in EPS:
        q, buf = guarded_q(M, N)
        got = B.dit_rms_norm_quant_forward(dev_rows(x, x_bf16), torch.from_numpy(g).cuda() if gamma else None, eps,
                                           residual=None if r is None else dev_rows(r, residual == "bf16"), q=q)
        eps = float(np.float32(eps))  # (as the call takes it)
        h, t, _ = R.norm_rows(x, g, r, 1.0)
        n = counts(t, eps)
        qn, sn = q.cpu().numpy(), got[1].cpu().numpy()
        assert not qn[~n].any() and not sn[~n].any()
        factor = 1.0 / np.sqrt(np.mean(h[n] * h[n], axis=1) + eps)
        R.check_rows(qn[n], sn[n], t[n], factor, scale_rel=R.norm_scale_rel(N), what="%dx%d eps %g" % (M, N, eps))
        check_guard(buf, M, N)
        if r is not None:  # the sum goes out as it is
            want = x + r
            if residual == "bf16":
                want = wl.bf16_bits_to_f32(wl.f32_to_bf16_bits(want))
            assert np.array_equal(got[2].float().cpu().numpy(), want)


@pytest.mark.parametrize("eps", [0.0, 1e-40])
@pytest.mark.parametrize("N", [40, 5120, 20481])
def test_rows_that_cannot_be_quantised(N, eps):
    """Zeros, NaN and infinities, a sum of squares that overflows, and rows around them: as with an ordinary eps."""
    rng = np.random.default_rng(N)
    x = rows_of(rng, 10, N, False, gain=np.float32(1e-24))
    x[1] = 0
    x[2, N // 2] = np.nan
    x[4, N - 1] = np.inf
    x[5] = -0.0
    x[6] = 1e25
    x[8, 0] = -np.inf
    q, scale = (t.cpu().numpy() for t in B.dit_rms_norm_quant_forward(dev_rows(x, False), None, eps))
    bad, good = [1, 2, 4, 5, 6, 8], [0, 3, 7, 9]
    assert not q[bad].any() and np.all(scale[[1, 5]] == 0) and np.all(np.isnan(scale[[2, 4, 6, 8]]))
    h, t, factor = R.norm_rows(x[good], None, None, float(np.float32(eps)))
    R.check_rows(q[good], scale[good], t, factor, scale_rel=R.norm_scale_rel(N))


def test_ordinary_rows_have_the_same_bits():
    """Scaling by a power of two rounds nothing: rows whose squares eps does not touch have the same bits for any small eps."""
    rng = np.random.default_rng(2)
    x = dev_rows(rows_of(rng, 300, 2056, False, gain=np.float32(0.01)), False)
    got = [B.dit_rms_norm_quant_forward(x, None, eps) for eps in (0.0, 2.0 ** -110, 2.0 ** -101, 2.0 ** -99, 2.0 ** -60)]
    for q, scale in got[1:]:
        assert (q == got[0][0]).all().item() and (scale == got[0][1]).all().item()
