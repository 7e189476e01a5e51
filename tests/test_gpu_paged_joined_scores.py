"""Attention over a paged cache whose keys are taken in pieces, at large scores: the pieces' weights are those of the differences of
their maxima, however large these are."""
import numpy as np
import pytest

from paged_util import Cache, host, randn
from paper_2601_20655_amd import binding as B
from test_paged_host import plan

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,page", [(128, 64), (128, 60), (64, 48)])
@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("N", [1, 30, 100])
def test_maxima_of_pieces(N, kind, D, page):
    """Scores 2^23 .. 2^24 and up to six more (whole numbers, exact in fp32), halved, at every 128th key; the others have no weight."""
    import torch

    keys = 8300
    c = Cache([keys], 1, D, page, kind, "head", N)
    p = plan(N, 1, 1, 1, D, c.table.shape[1] * page, 0, page % 16 == 0)
    assert (p.few_each if p.few else 2) > 1 and (p.big_each if p.big else 2) > 1
    a = 128 + np.arange(N) % 128
    q = torch.zeros((N, 1, D), dtype=torch.bfloat16, device="cuda")
    q[:, 0, 0] = torch.from_numpy(2.0 * a).cuda().bfloat16()
    q[:, 0, 1] = 1
    n = np.arange(5, keys, 128)
    more = 3 * (n // 128) % 7
    at, slot = torch.from_numpy(c.table[0, n // page]).long().cuda(), torch.from_numpy(n % page).cuda()
    c.k.zero_()
    c.k[at, slot, 0, 0] = 2.0 ** 15
    c.k[at, slot, 0, 1] = torch.from_numpy(more).cuda().to(c.k.dtype)
    out, lse = B.dit_attn_paged_forward(q, *c.args([N]), scale=0.5, out=torch.empty((N, 1, D), device="cuda"), want_lse=True)
    v = c.v[at, slot, 0].double().cpu().numpy()
    w = np.exp(0.5 * (more - more.max()))
    # P rounded to its type; exponents of differences below 2^3, sums of 65 terms
    tol = ({"f16": 2.0 ** -11, "bf16": 2.0 ** -8}[kind] + 2.0 ** -17) * (w @ np.abs(v) / w.sum())
    assert np.all(np.abs(host(out)[:, 0] - w @ v / w.sum()) <= tol)
    # (log2(e), its products with the scale and m, log(2) and the last product)
    want = 0.5 * (a * 65536.0 + more.max()) + np.log(w.sum())
    assert np.all(np.abs(host(lse)[0] - want) <= 2.0 ** -21 * (1 + np.abs(want)))
