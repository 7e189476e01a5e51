"""Attention over a paged cache of rows all of whose scores are below -10^30, and of rows without a key at a very large scale."""
import numpy as np
import pytest

from paged_util import Cache, host
from paper_2601_20655_amd import binding as B

pytestmark = pytest.mark.gpu


def one_hot(keys, N, D, page, q_power, k_sign_power):
    """Exact scores (128 + t) 2^q_power times -(128 + (37 n) mod 100) 2^k_power, of one channel.  (cache, q, numbers of k, V's rows)"""
    import torch

    c = Cache([keys], 1, D, page, "bf16", "head", 3)
    n = np.arange(keys)
    numbers = 128 + 37 * n % 100
    at, slot = torch.from_numpy(c.table[0, n // page]).long().cuda(), torch.from_numpy(n % page).cuda()
    c.k.zero_()
    c.k[at, slot, 0, 0] = torch.from_numpy(-numbers * 2.0 ** k_sign_power).cuda().bfloat16()
    q = torch.zeros((N, 1, D), dtype=torch.bfloat16, device="cuda")
    q[:, 0, 0] = torch.from_numpy((128.0 + np.arange(N) % 100) * 2.0 ** q_power).cuda().bfloat16()
    return c, q, numbers, c.v[at, slot, 0].double().cpu().numpy()


@pytest.mark.parametrize("D,page", [(128, 64), (128, 60), (64, 48)])
@pytest.mark.parametrize("N", [1, 30, 100])
@pytest.mark.parametrize("keys,max_kv", [(90, 1), (653, 1), (8300, 0)])
def test_rows_of_very_low_scores(N, D, page, keys, max_kv):
    """-2^109 .. -2^110: the keys of the largest number share the weight."""
    import torch

    c, q, numbers, v = one_hot(keys, N, D, page, 45, 50)
    out, lse = B.dit_attn_paged_forward(q, *c.args([N]), max_kv=max_kv, out=torch.empty((N, 1, D), device="cuda"), want_lse=True)
    best = v[numbers == numbers.min()]
    # equal weights, powers of two: what is left are sums over the keys and pieces, 1 / sum and the product
    tol = (len(best) + 68) * 2.0 ** -24 * np.abs(best).mean(0)
    assert np.all(np.abs(host(out)[:, 0] - best.mean(0)) <= tol)
    # (seven roundings at the most: the scale's root and quotient, log2(e), two products, log(2), a product)
    want = -(128.0 + np.arange(N) % 100) * 2.0 ** 95 * numbers.min() / np.sqrt(D) + np.log(len(best))
    assert np.all(np.abs(host(lse)[0] - want) <= 2.0 ** -21 * (1 + np.abs(want)))


@pytest.mark.parametrize("D,page", [(128, 64), (128, 60), (64, 48)])
@pytest.mark.parametrize("N", [20, 200])
@pytest.mark.parametrize("scale", [1.0, 1e9, 1e36])
def test_rows_without_a_key_at_any_scale(N, D, page, scale):
    """kv_len is half the new tokens: the first half lie ahead of the first key and see nothing; the others one key by far the best."""
    import torch

    keys = N // 2
    c, q, numbers, v = one_hot(keys, N, D, page, 0, 0)
    out, lse = B.dit_attn_paged_forward(q, *c.args([N]), frame=1, scale=scale, out=torch.empty((N, 1, D), device="cuda"), want_lse=True)
    out, lse = host(out)[:, 0], host(lse)[0]
    assert np.all(out[:N - keys] == 0) and np.all(np.isneginf(lse[:N - keys]))
    for i in range(keys):
        best = v[:i + 1][numbers[:i + 1] == numbers[:i + 1].min()]
        assert np.all(np.abs(out[N - keys + i] - best.mean(0)) <= 8 * 2.0 ** -24 * np.abs(best).mean(0)), i
