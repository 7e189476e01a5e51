"""Attention over a paged cache where a row's maximum becomes very large, or stops being it, in the middle of its keys.

The large scores are exact: one channel of q, a number of 8 bits, times one of k, a power of two.  So keys of equal large scores have the
same weight, all others none, and the output is the mean of their rows of V.

lse, scale m + log(sum): the scale's root and quotient, log2(e), their product, that with m, log(2) and the last product are seven roundings at
the most, below 2^-21 of it."""
import numpy as np
import pytest

from paged_util import Cache, dtype, host, randn
from paper_2601_20655_amd import binding as B
from test_gpu_paged_wide import wide

pytestmark = pytest.mark.gpu


def rows(N, H, D, power, kind):
    """Queries whose channel 0 is (128 .. 255) 2^(power of q), and what the large keys' is; the other channels N(0, 1)."""
    import torch

    of_k = min(power, 15 if kind == "f16" else 120)
    a = (128.0 + np.arange(N) % 128) * 2.0 ** (power - of_k)
    q = randn(power + N, (N, H, D), "f32")
    q[:, :, 0] = torch.from_numpy(a.astype(np.float32)).cuda()[:, None]
    return q.to(torch.bfloat16), 2.0 ** of_k, a


def call(c, q, **kw):
    import torch

    N, H, D = q.shape
    out, lse = B.dit_attn_paged_forward(q, *c.args([N]), frame=0, out=torch.empty((N, H, D), device="cuda"), want_lse=True, **kw)
    return host(out).astype(np.float64), host(lse).astype(np.float64)


def set_channel(c, keys, value, others=None):
    for n in keys:
        page, slot = c.table[0, n // c.k.shape[1]], n % c.k.shape[1]
        if others is not None:
            c.k[page, slot] = others
        c.k[page, slot, :, 0] = value


# where the first large key is: in the second half of a tile of 64 keys, in the first, its last key; where equal ones follow
PLACES = [(168, 261), (133, 178), (255, 447), (160, 161, 330, 600), (40, 639)]


@pytest.mark.parametrize("kind,power", [("f16", 12), ("f16", 19), ("f16", 23), ("bf16", 12), ("bf16", 19), ("bf16", 60)])
@pytest.mark.parametrize("D,page", [(128, 64), (128, 60), (64, 48), (64, 60)])
@pytest.mark.parametrize("N", [1, 40, 100])
def test_a_maximum_that_jumps(kind, power, D, page, N):
    """Ordinary keys, then a very large one, and equal ones behind it.  Keys in one piece (max_kv: 1)."""
    for places in PLACES:
        c = Cache([653], 1, D, page, kind, "head", power)
        q, large, a = rows(N, 1, D, power, kind)
        c.k[..., 0] = 0
        set_channel(c, places, large, 0.0)
        out, lse = call(c, q, max_kv=1)
        v = np.stack([host(c.v)[c.table[0, n // page], n % page, 0] for n in places]).astype(np.float64)
        # equal weights, powers of two: what is left are the sums over the keys, 1 / sum and the product
        tol = (len(places) + 4) * 2.0 ** -24 * np.abs(v).mean(0)
        assert np.all(np.abs(out[:, 0] - v.mean(0)) <= tol), (places, np.abs(out[:, 0] - v.mean(0)).max())
        want = a * large / np.sqrt(D) + np.log(len(places))
        assert np.all(np.abs(lse[0] - want) <= 2.0 ** -21 * (1 + np.abs(want))), places


@pytest.mark.parametrize("kind,power", [("f16", 19), ("f16", 23), ("bf16", 19), ("bf16", 60)])
@pytest.mark.parametrize("D,page", [(128, 64), (64, 48), (64, 60)])
def test_maxima_that_jump_in_wide_tiles(kind, power, D, page):
    """The same by tiles of 256 rows, over keys in pieces: pairs of large keys everywhere."""
    lens, new = [70000], [300]
    c, H = wide(lens, D, page, kind, "head", power, 1, new)
    q, large, a = rows(new[0], H, D, power, kind)
    places = [64 * t + x for t in range(2, 1090, 7) for x in (44, 130)]
    import torch

    at = torch.tensor(places)
    pages, slots = torch.from_numpy(c.table[0])[at // page].long(), at % page
    c.k[..., 0] = 0
    zero = torch.zeros((len(places),) + tuple(c.k.shape[2:]), dtype=dtype(kind), device="cuda")
    zero[..., 0] = large
    c.k[pages.cuda(), slots.cuda()] = zero
    out, lse = call(c, q)
    v = c.v[pages.cuda(), slots.cuda()].double().cpu().numpy()
    tol = (len(places) + 4) * 2.0 ** -24 * np.abs(v).mean(0)
    assert np.all(np.abs(out - v.mean(0)) <= tol)
    want = a * large / np.sqrt(D) + np.log(len(places))
    assert np.all(np.abs(lse - want) <= 2.0 ** -21 * (1 + np.abs(want)))


@pytest.mark.parametrize("kind,power", [("f16", 19), ("bf16", 19), ("bf16", 60)])
@pytest.mark.parametrize("D,page", [(128, 64), (128, 60), (64, 48)])
@pytest.mark.parametrize("N", [1, 100])
@pytest.mark.parametrize("last", [31, 70, 127, 200])
def test_a_maximum_that_comes_back(kind, power, D, page, N, last):
    """The first keys' scores are very low, those behind them ordinary: the first ones have no weight."""
    import torch

    keys = 653
    c = Cache([keys], 1, D, page, kind, "head", power)
    q, large, _ = rows(N, 1, D, power, kind)
    c.k[..., 0] = 0
    set_channel(c, range(last), -large)
    out, lse = call(c, q, max_kv=1)
    n = np.arange(last, keys)
    k, v = (host(x)[c.table[0, n // page], n % page, 0].astype(np.float64) for x in (c.k, c.v))
    x = (q[:, 0].half() if kind == "f16" else q[:, 0]).double().cpu().numpy()
    s = x @ k.T / np.sqrt(D)
    w = np.exp(s - s.max(1, keepdims=True))
    total = w.sum(1, keepdims=True)
    # a score: D + 8 roundings of the sum of |q k|; P: half a step of its type; sums over the keys
    err = (np.abs(x) @ np.abs(k).T).max(1, keepdims=True) / np.sqrt(D) * (D + 8) * 2.0 ** -24 + (keys + 64) * 2.0 ** -24
    tol = ({"f16": 2.0 ** -11, "bf16": 2.0 ** -8}[kind] + 2 * err + 2.0 ** -20) * (w @ np.abs(v) / total)
    assert np.all(np.abs(out[:, 0] - w @ v / total) <= tol)
    want = s.max(1) + np.log(total[:, 0])
    assert np.all(np.abs(lse[0] - want) <= err[:, 0] + 2.0 ** -21 * (1 + np.abs(want)))
    assert torch.isfinite(c.k.float()).all()
