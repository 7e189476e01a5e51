"""Attention over fp16 pages of one key with nearly all the weight and many of very little: what the many have together counts."""
import numpy as np
import pytest

from paged_util import Cache, host, randn
from paper_2601_20655_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,D,page", [(1, 128, 64), (1, 64, 60), (24, 128, 64), (40, 64, 48), (100, 128, 64), (100, 128, 60), (300, 64, 48)])
@pytest.mark.parametrize("keys", [700, 40000])
@pytest.mark.parametrize("halvings", [18.0, 25.3, 30.0])
def test_many_small_weights(N, D, page, keys, halvings):
    """One key of weight 1 whose row of V is 0; the others of 2^-halvings each, their rows of V near 1.  Where it is: first, last, inside."""
    import torch

    for place in (0, keys - 1, keys // 2 + 37):
        c = Cache([keys], 1, D, page, "f16", "head", keys)
        c.v.copy_(1 + 0.25 * c.v)
        c.k[..., 0] = 0
        gap = float(np.float16(halvings * np.log(2)))
        at, slot = c.table[0, place // page], place % page
        c.k[at, slot, 0, 0] = gap
        c.v[at, slot] = 0
        q = torch.zeros((N, 1, D), dtype=torch.bfloat16, device="cuda")
        q[:, 0, 0] = 1
        out, lse = B.dit_attn_paged_forward(q, *c.args([N]), scale=1.0, out=torch.empty((N, 1, D), device="cuda"), want_lse=True)
        n = np.arange(keys)
        v = host(c.v)[c.table[0, n // page], n % page, 0].astype(np.float64)
        w = np.where(n == place, 1.0, np.exp(-gap))
        total = w.sum()
        # a probability: half a step of fp16, or 2^-32 of the largest; exponents up to 2^5 rounded, sums over the keys
        tol = ((w * 2.0 ** -11 + 2.0 ** -32) @ np.abs(v) + (2.0 ** -18 + (keys + 64) * 2.0 ** -24) * (w @ np.abs(v))) / total
        assert np.all(np.abs(host(out)[:, 0] - w @ v / total) <= tol), (place, np.abs(host(out)[:, 0] / (w @ v / total) - 1).max())
        want = gap + np.log(total)
        assert np.all(np.abs(host(lse)[0] - want) <= (keys + 64) * 2.0 ** -24 + 2.0 ** -18 + 2.0 ** -21 * (1 + want)), place


@pytest.mark.parametrize("N,D,page", [(1, 128, 64), (100, 128, 64), (100, 128, 60), (100, 64, 48)])
@pytest.mark.parametrize("step", [8.5, 12.0, 15.75])
def test_scores_a_step_of_fp32_apart(N, D, page, step):
    """Scores of 2^30 and, behind them, of 2^30 + 128, the next number but none: a weight 2^-step of the other."""
    import torch

    keys, scale = 653, float(np.float32(step / 128 * np.log(2)))
    c = Cache([keys], 1, D, page, "f16", "head", keys)
    n = np.arange(keys)
    at, slot = torch.from_numpy(c.table[0, n // page]).long().cuda(), torch.from_numpy(n % page).cuda()
    more = np.where(n % 150 == 149, 128.0, 0.0)
    c.k.zero_()
    c.k[at, slot, 0, 0] = 2.0 ** 15
    c.k[at, slot, 0, 1] = torch.from_numpy(more).cuda().half()
    q = torch.zeros((N, 1, D), dtype=torch.bfloat16, device="cuda")
    q[:, 0, 0], q[:, 0, 1] = 2.0 ** 15, 1
    out, lse = B.dit_attn_paged_forward(q, *c.args([N]), scale=scale, max_kv=1, out=torch.empty((N, 1, D), device="cuda"), want_lse=True)
    v = c.v[at, slot, 0].double().cpu().numpy()
    w = np.exp(scale * (more - 128))
    total = w.sum()
    # a probability: half a step of fp16; exponents up to 2^4 rounded, sums over the keys
    tol = (2.0 ** -11 + 2.0 ** -18 + (keys + 64) * 2.0 ** -24) * (w @ np.abs(v)) / total
    assert np.all(np.abs(host(out)[:, 0] - w @ v / total) <= tol)
    want = scale * (2.0 ** 30 + 128) + np.log(total)
    assert np.all(np.abs(host(lse)[0] - want) <= 2.0 ** -21 * want)
