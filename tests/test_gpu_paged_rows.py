"""Rows normalised and rotated by given positions (dit_qk_rope_forward), and appended to pages (dit_kv_append_forward)."""
import numpy as np
import pytest

import paged_ref as R
from paged_util import Cache, dtype, host, ints, randn
from paper_2601_20655_amd import binding as B

pytestmark = pytest.mark.gpu
EPS = 1e-6


def positions(N, seed, far=3000):
    rng = np.random.default_rng([seed, 9])
    return rng.integers(-far, far, size=(N, 3)).astype(np.int32)


def norm_of(norm, H, Hk, D, seed, eps=EPS, gamma=True):
    if norm is None:
        return None, None, None
    rng = np.random.default_rng([seed, 4])
    g = [(1 + 0.25 * rng.standard_normal(h * D)).astype(np.float32) if gamma else None for h in (H, Hk)]
    import torch

    return (norm, eps) + tuple(None if x is None else torch.from_numpy(x).cuda() for x in g), g[0], g[1]


def check(got, x, pos, split, kind, norm, gamma, eps=EPS, base=10000.0, what=""):
    y, mag = R.rows(host(x), pos, split, base, norm, gamma, eps)
    bound = 0.0 if pos is None else R.angle_bound(pos, split, base)
    R.check_rows(host(got), y, mag, kind, norm, bound, what)


SPLITS = {128: [(44, 42, 42), (128, 0, 0), (0, 2, 126), (64, 64, 0)], 64: [(22, 20, 22), (64, 0, 0), (2, 0, 62), (0, 0, 64)]}


@pytest.mark.parametrize("N,H,Hk,D", [(1, 1, 1, 64), (1, 40, 8, 128), (2, 3, 3, 128), (7, 9, 3, 64), (33, 5, 1, 128), (257, 12, 12, 128),
                                      (130, 17, 17, 64), (1024, 3, 2, 128), (5, 96, 96, 128)])
@pytest.mark.parametrize("norm", [None, "head", "token"])
@pytest.mark.parametrize("x,out", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f16"), ("f32", "bf16")])
def test_rows(N, H, Hk, D, norm, x, out):
    """One projection's output holds q and k rows; outputs inside a guard."""
    import torch

    seed = N + 7 * H + D
    qk = randn(seed, (N, H + Hk + 1, D), x)
    q, k = qk[:, :H], qk[:, H:H + Hk]
    pos, split = positions(N, seed), SPLITS[D][seed % 4]
    args, gq, gk = norm_of(norm, H, Hk, D, seed, gamma=seed % 3 > 0)
    buf = torch.full((N + 2, H + Hk, D + 8), -77.0, dtype=dtype(out), device="cuda")
    qo, ko = buf[1:N + 1, :H, :D], buf[1:N + 1, H:, :D]
    got = B.dit_qk_rope_forward(q, k, ints(pos), split, q_out=qo, k_out=ko, norm=args)
    assert got[0].data_ptr() == qo.data_ptr() and got[1].data_ptr() == ko.data_ptr()
    check(qo, q, pos, split, out, norm, gq, what="q")
    check(ko, k, pos, split, out, norm, gk, what="k")
    b = host(buf)
    assert np.all(b[0] == -77) and np.all(b[-1] == -77) and np.all(b[:, :, D:] == -77)


@pytest.mark.parametrize("which", ["q", "k"])
@pytest.mark.parametrize("norm", [None, "head", "token"])
def test_one_of_them_head_major(which, norm):
    """Only q or only k, [heads, N, D] in memory, allocated output."""
    N, H, D = 37, 6, 64
    x = randn(3, (H, N, D), "bf16").transpose(0, 1)
    pos = positions(N, 2)
    args, gq, gk = norm_of(norm, H, H, D, 1)
    if args is not None:
        args = args[:2] + ((args[2], None) if which == "q" else (None, args[3]))
    q, k = (x, None) if which == "q" else (None, x)
    got = B.dit_qk_rope_forward(q, k, ints(pos), (22, 20, 22), norm=args)
    assert got[1 if which == "q" else 0] is None
    check(got[0 if which == "q" else 1], x, pos, (22, 20, 22), "bf16", norm, gq if which == "q" else gk)


@pytest.mark.parametrize("norm", ["head", "token"])
def test_without_positions(norm):
    N, H, D = 65, 4, 128
    q, k = randn(1, (N, H, D), "f32"), randn(2, (N, H, D), "f32")
    args, gq, gk = norm_of(norm, H, H, D, 1)
    qo, ko = B.dit_qk_rope_forward(q, k, None, norm=args)
    check(qo, q, None, None, "f32", norm, gq)
    check(ko, k, None, None, "f32", norm, gk)


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("norm", [None, "head", "token"])
def test_in_place(x, norm):
    N, H, Hk, D = 300, 12, 5, 128
    q, k = randn(1, (N, H, D), x), randn(2, (N, Hk, D), x)
    pos = positions(N, 1)
    args, _, _ = norm_of(norm, H, Hk, D, 1)
    want = B.dit_qk_rope_forward(q, k, ints(pos), (44, 42, 42), norm=args)
    got = B.dit_qk_rope_forward(q, k, ints(pos), (44, 42, 42), q_out=q, k_out=k, norm=args)
    assert got[0].data_ptr() == q.data_ptr()
    assert np.array_equal(host(q), host(want[0])) and np.array_equal(host(k), host(want[1]))


@pytest.mark.parametrize("base", [10000.0, 1e6, 3.0, 0.5])
def test_far_positions(base):
    """Positions up to the ends of 32 bits, 32-bit rows."""
    rng = np.random.default_rng(0)
    pos = np.concatenate([rng.integers(-2 ** 31, 2 ** 31, size=(40, 3)), [[2 ** 31 - 1] * 3, [-2 ** 31] * 3, [0] * 3]]).astype(np.int32)
    if base < 1:
        pos = pos // 2 ** 12  # (angles of 2^31 2^63: the bound says nothing of them)
    x = randn(5, (len(pos), 2, 128), "f32")
    for split in SPLITS[128]:
        got, _ = B.dit_qk_rope_forward(x, None, ints(pos), split, rope_base=base)
        check(got, x, pos, split, "f32", None, None, base=base)


@pytest.mark.parametrize("norm", ["head", "token"])
@pytest.mark.parametrize("eps", [0.0, 1e-38, 1e-6])
def test_rows_whose_squares_leave_fp32(norm, eps):
    """Rows of 1e-30, 1e-22, 1, 1e22 and 1e30, and of zeros with an eps."""
    N, H, D = 5, 3, 64
    x = host(randn(1, (N, H, D), "f32")) * np.array([1e-30, 1e-22, 1, 1e22, 1e30], dtype=np.float32)[:, None, None]
    import torch

    args, g, _ = norm_of(norm, H, H, D, 1, eps)
    got, _ = B.dit_qk_rope_forward(torch.from_numpy(x).cuda(), None, None, norm=args[:3] + (None,))
    y, mag = R.rows(x, None, None, 1.0, norm, g, eps)
    tol = R.rows_tolerance(y, mag, "f32", norm)
    # (1e-38 and 1e-6 against squares of 1e-60: what is left is below any number that fp32 keeps whole)
    assert np.all(np.abs(host(got) - y) <= tol + 2.0 ** -148)
    if eps:
        zero, _ = B.dit_qk_rope_forward(torch.zeros((N, H, D), device="cuda"), None, None, norm=args[:3] + (None,))
        assert np.all(host(zero) == 0)


@pytest.mark.parametrize("norm", [None, "head", "token"])
def test_no_row_reaches_another(norm):
    """A NaN and an infinity stay in their pair, head or token."""
    N, H, D = 40, 8, 128
    x = randn(1, (N, H, D), "bf16")
    pos = ints(positions(N, 3))
    args, _, _ = norm_of(norm, H, H, D, 1)
    want = host(B.dit_qk_rope_forward(x, None, pos, (44, 42, 42), norm=args and args[:3] + (None,))[0])
    x[11, 3, 6], x[30, 7, 127] = float("nan"), float("inf")
    got = host(B.dit_qk_rope_forward(x, None, pos, (44, 42, 42), norm=args and args[:3] + (None,))[0])
    touched = np.zeros((N, H, D), bool)
    for t, h, c in ((11, 3, 6), (30, 7, 127)):
        touched[(t, h, slice(c // 2 * 2, c // 2 * 2 + 2)) if norm is None else (t, h) if norm == "head" else t] = True
    assert np.array_equal(got[~touched], want[~touched])
    assert np.all(np.isnan(got[11, 3, 6:8]))


# ---- to pages ----

def expected_pages(c, k, v, q_start, kind):
    """The caches after the call: the rows of every token that has a slot."""
    kc, vc = host(c.k).copy(), host(c.v).copy()
    where = np.zeros(kc.shape[:2], bool)
    for r in range(len(c.lens)):
        new = q_start[r + 1] - q_start[r]
        for i in range(new):
            at = c.lens[r] - new + i
            if at < 0 or at // kc.shape[1] >= c.table.shape[1]:
                continue
            page = c.table[r, at // kc.shape[1]]
            if 0 <= page < kc.shape[0]:
                kc[page, at % kc.shape[1]] = k[q_start[r] + i]
                vc[page, at % kc.shape[1]] = v[q_start[r] + i]
                where[page, at % kc.shape[1]] = True
    return kc, vc, where


@pytest.mark.parametrize("page,layout", [(1, "token"), (16, "head"), (48, "token"), (64, "head"), (100, "padded"), (2000, "head")])
@pytest.mark.parametrize("D,H,Hk", [(128, 10, 2), (64, 3, 3), (128, 0, 4)])
@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("norm", [None, "head", "token"])
def test_append(page, layout, D, H, Hk, kind, norm):
    """Ragged requests, one without new tokens, two tokens behind the last request, dropped pages, q beside."""
    import torch

    new, lens = [1, 0, 33, 7, 130], [1, 50, 33, 77, 401]
    N = sum(new) + 2
    seed = page + D + H
    c = Cache(lens, Hk, D, page, kind, layout, seed, drop=(1, 3) if page < 64 else ())
    rows = randn(seed, (N, H + 2 * Hk, D), "bf16")
    q, k, v = rows[:, :H] if H else None, rows[:, H:H + Hk], rows[:, H + Hk:]
    pos, split = positions(N, seed), SPLITS[D][seed % 4]
    args, gq, gk = norm_of(norm, max(H, 1), Hk, D, seed)
    if args is not None and not H:
        args = args[:2] + (None, args[3])
    pages = c.args(new)
    y, mag = R.rows(host(k), pos, split, 10000.0, norm, gk, EPS)
    bound = R.angle_bound(pos, split, 10000.0)
    tol = R.rows_tolerance(y, mag, kind, norm, bound)
    kw, vw, where = expected_pages(c, y, host(v), c.q_start, kind)
    kt, _, _ = expected_pages(c, tol, host(v), c.q_start, kind)
    q_out = torch.full((N, H, D), -77.0, dtype=torch.bfloat16, device="cuda") if H else None
    got = B.dit_kv_append_forward(k, v, *pages, pos=ints(pos), split=split, q=q, q_out=q_out, norm=args)
    kg, vg = host(c.k).astype(np.float64), host(c.v)
    assert np.array_equal(kg[~where], kw[~where]) and where.any()
    assert np.all(np.abs(kg - kw)[where] <= kt[where])
    assert np.array_equal(vg, vw.astype(np.float16).astype(np.float32) if kind == "f16" else vw)
    if H:
        n = sum(new)
        check(got[:n], q[:n], pos[:n], split, "bf16", norm, gq)
        assert np.all(host(q_out)[n:] == -77)
    else:
        assert got is None


def test_append_many_requests():
    """1,000 requests, some without a token: the search for a token's request over more entries than a wavefront has lanes."""
    rng = np.random.default_rng(1)
    new = rng.integers(0, 4, size=1000)
    new[:3] = 0
    new[-2:] = 0
    lens = new + rng.integers(0, 20, size=1000)
    c = Cache(lens, 1, 64, 8, "bf16", "head", 1)
    N = int(new.sum())
    k, v = randn(1, (N, 1, 64), "bf16"), randn(2, (N, 1, 64), "bf16")
    pages = c.args(new)
    kw, vw, _ = expected_pages(c, host(k), host(v), c.q_start, "bf16")
    B.dit_kv_append_forward(k, v, *pages)
    assert np.array_equal(host(c.k), kw) and np.array_equal(host(c.v), vw)


@pytest.mark.parametrize("table", [8, 64, 65, 4097])
def test_request_search_sizes(table):
    """One token a request, as many requests as entries of a search step and one more."""
    c = Cache([3] * table, 1, 64, 4, "f16", "token", 2)
    k, v = randn(1, (table, 1, 64), "f32"), randn(2, (table, 1, 64), "f32")
    pages = c.args([1] * table)
    kw, vw, where = expected_pages(c, host(k), host(v), c.q_start, "f16")
    B.dit_kv_append_forward(k, v, *pages)
    assert where.sum() == table
    assert np.array_equal(host(c.k), kw.astype(np.float16)) and np.array_equal(host(c.v), vw.astype(np.float16))


def test_counts_out_of_range():
    """Tokens before place 0 or behind the table write nothing; counts that make no sense reach no other memory."""
    import torch

    c = Cache([64, 64], 2, 128, 16, "bf16", "head", 3, extra_pages=0)
    k, v = randn(1, (12, 2, 128), "bf16"), randn(2, (12, 2, 128), "bf16")
    before = host(c.k).copy()
    args = list(c.args([4, 8]))
    for lens in ([2, 66], [-5, 2 ** 31 - 1], [0, -2 ** 31]):
        c.lens = np.array(lens)
        kw, vw, _ = expected_pages(c, host(k), host(v), c.q_start, "bf16")
        args[4] = ints(lens)
        B.dit_kv_append_forward(k, v, *args)
        assert np.array_equal(host(c.k), kw) and np.array_equal(host(c.v), vw)
    assert not np.array_equal(host(c.k), before)
    for starts in ([0, -7, 2 ** 31 - 1], [5, 3, 1], [2 ** 31 - 1] * 3, [-2 ** 31, 0, 12]):
        args[3], args[4] = ints(starts), ints([64, 64])
        B.dit_kv_append_forward(k, v, *args)
    torch.cuda.synchronize()


def test_fp16_saturates():
    import torch

    c = Cache([4], 1, 64, 16, "f16", "head", 1)
    k = torch.full((4, 1, 64), 1e30, dtype=torch.bfloat16, device="cuda")
    B.dit_kv_append_forward(k, -k, *c.args([4]))
    page = int(c.table[0, 0])
    assert torch.all(c.k[page, :4] == 65504) and torch.all(c.v[page, :4] == -65504)


def test_no_tokens():
    import torch

    c = Cache([4], 1, 64, 16, "f16", "head", 1)
    k = torch.empty((0, 1, 64), dtype=torch.bfloat16, device="cuda")
    before = host(c.k).copy()
    assert B.dit_kv_append_forward(k, k, *c.args([0])) is None
    q, _ = B.dit_qk_rope_forward(k, None, None)
    assert q.shape == k.shape and np.array_equal(host(c.k), before)
