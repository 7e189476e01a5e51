"""Attention over a paged cache by the tiles of 256 rows that long caches take (a table with room for many pages, whatever there is
in them, chooses those), and of 128 rows over rows that lie anywhere, against 64-bit softmaxes."""
import numpy as np
import pytest

from paged_util import Cache, host, randn
from test_gpu_paged_attn import check, run
from test_paged_host import plan
import paged_ref as R

pytestmark = pytest.mark.gpu

ROOM = 3_000_000  # keys


def wide(lens, D, page, kind, layout, seed, G, new, **kw):
    """A cache, and query heads (G a key head), as few as get those tiles."""
    import torch  # noqa: F401  (the HIP runtime that the library is to share, ahead of the library)

    runs = page % 16 == 0
    columns = max(-(-n // page) for n in lens) + ROOM // page
    for Hk in range(1, 17):
        p = plan(sum(new) + 2, len(lens), G * Hk, Hk, D, columns * page, 0, runs)
        if p.big and (p.big_waves, p.big_qb) == ((8, 2) if runs or D == 64 else (8, 1)):
            return Cache(lens, Hk, D, page, kind, layout, seed, extra_pages=ROOM // page, **kw), G * Hk
    raise AssertionError("no such heads")


# on, one short of and one past a tile of rows, of keys, a page; tiles in several pieces, of which the last are empty
SHAPES = [([129], [129]), ([200], [201]), ([255], [300]), ([256], [256]), ([257], [1000]), ([300], [5000]), ([40, 500, 5], [40, 1210, 640]),
          ([3, 0, 1, 740], [3, 9, 130, 2333])]


@pytest.mark.parametrize("new,lens", SHAPES, ids=["-".join(map(str, a + b)) for a, b in SHAPES])
@pytest.mark.parametrize("D,G,page,layout,kind", [(128, 1, 64, "head", "bf16"), (64, 2, 48, "token", "f16"),
                                                  (128, 3, 20, "padded", "f16"), (64, 1, 100, "head", "bf16"),
                                                  (128, 1, 1000, "token", "bf16"), (64, 1, 7, "token", "f16")])
@pytest.mark.parametrize("frame,window", [(0, 0), (1, 0), (40, 5)])
def test_shapes(new, lens, D, G, page, layout, kind, frame, window):
    seed = sum(new) + sum(lens) + page
    c, H = wide(lens, D, page, kind, layout, seed, G, new)
    check(c, randn(seed, (sum(new) + 2, H, D), "bf16"), new, "f32" if seed % 2 else "bf16", frame=frame, window=window)


@pytest.mark.parametrize("page", [5, 16, 64, 100])
@pytest.mark.parametrize("D,kind", [(128, "bf16"), (64, "f16")])
def test_dropped_pages(page, D, kind):
    """Pages that are not there: early, inside, a whole request's, and a sixteen-tile group's."""
    new, lens = [90, 3, 300], [2600, 3, 1300]
    c, H = wide(lens, D, page, kind, "head", page, 2, new, drop=(0, 2, 3))
    c.table[0, 1100 // page:2300 // page] = -1
    c.table[1, :] = 2 ** 31 - 1
    c.table[2, (lens[2] - 1) // page] = -7
    q = randn(page, (sum(new) + 2, H, D), "bf16")
    for frame, window in ((0, 0), (1, 0), (20, 2)):
        check(c, q, new, "bf16", frame=frame, window=window, what="frame %d" % frame)


@pytest.mark.parametrize("bad", ["nan", "inf"])
@pytest.mark.parametrize("D,page", [(128, 64), (128, 60), (64, 60), (64, 64)])
def test_masked_keys_may_hold_anything(bad, D, page):
    new, lens, frame = [270], [1100], 90
    c, H = wide(lens, D, page, "bf16", "head", 3, 1, new)
    q = randn(1, (sum(new), H, D), "bf16")
    want, want_lse = run(c, q, new, "f32", 0, frame=frame)
    at = 1079  # the last key of a frame; the tokens of the frame before do not see it
    c.k[c.table[0, at // page], at % page, :, 7] = float(bad)
    c.v[c.table[0, at // page], at % page, :, 33] = float(bad)
    got, lse = run(c, q, new, "f32", 0, frame=frame)
    hidden = np.array([R.seen(830 + i, 1100, frame, 0)[1] <= at for i in range(270)])
    assert hidden.any() and not hidden.all()
    assert np.allclose(got[hidden], want[hidden], rtol=0, atol=2.0 ** -6) and np.array_equal(lse[:, hidden], want_lse[:, hidden])
    assert not np.any(np.isfinite(got[~hidden][:, :, 33]))


def test_maxima_that_move():
    """Keys whose scores grow along the sequence: every tile raises its rows' maxima."""
    c, H = wide([3000], 128, 64, "bf16", "head", 1, 1, [280])
    import torch

    for at in range(3000):
        c.k[c.table[0, at // 64], at % 64] *= 0.02 + at / 500
    check(c, randn(2, (282, H, 128), "bf16"), [280], "f32", frame=1, scale=1.0)
    assert torch.isfinite(c.k.float()).all()


def test_deterministic():
    new, lens = [300, 240], [6000, 2000]
    for page in (64, 100):
        c, H = wide(lens, 128, page, "bf16", "head", 1, 2, new)
        q = randn(2, (sum(new), H, 128), "bf16")
        first = run(c, q, new, "f32", 0, frame=30)
        for _ in range(3):
            assert all(np.array_equal(a, b) for a, b in zip(first, run(c, q, new, "f32", 0, frame=30)))
