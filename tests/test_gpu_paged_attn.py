"""Attention of chunks of new tokens over a paged cache (dit_attn_paged_forward) against 64-bit softmaxes."""
import numpy as np
import pytest

import paged_ref as R
from paged_util import Cache, dtype, host, ints, randn
from paper_2601_20655_amd import binding as B

pytestmark = pytest.mark.gpu


def run(c, q, new, out="bf16", tail=2, **kw):
    """The call, with `tail` rows behind the last request that have to stay as they are; (out, lse) on the host."""
    import torch

    N, H, D = q.shape
    assert N == sum(new) + tail
    buf = torch.full((N, H, D), -77.0, dtype=dtype(out), device="cuda")
    lse = torch.full((H, N), -77.0, device="cuda")
    got = B.dit_attn_paged_forward(q, *c.args(new), out=buf, lse=lse, **kw)
    assert got[0].data_ptr() == buf.data_ptr()
    o, l = host(buf), host(lse)
    assert np.all(o[N - tail:] == -77) and np.all(l[:, N - tail:] == -77)
    return o[:N - tail], l[:, :N - tail]


def check(c, q, new, out="bf16", what="", tail=2, q_rounded=None, frame=0, window=0, scale=None, **kw):
    n = sum(new)
    got, lse = run(c, q, new, out, tail, frame=frame, window=window, scale=scale or 0.0, **kw)
    x = host(q)[:n] if q_rounded is None else q_rounded
    ref = R.attend(x, host(c.k), host(c.v), c.table, c.q_start, c.lens, frame, window, scale, R.HALF[c.kind])
    R.check_attn(got, lse, ref, out, what)
    return got, lse


# one token; a short chunk; on, one short of and one past a tile of keys, a page and a tile of rows; several requests
SHAPES = [([1], [1]), ([1], [64]), ([1], [65]), ([2], [33]), ([1], [1000]), ([16], [16]), ([17], [129]), ([64], [64]), ([128], [200]),
          ([129], [257]), ([300], [300]), ([1, 1, 1], [5, 700, 64]), ([3, 0, 1, 40], [3, 9, 130, 333]), ([1, 200, 5], [77, 210, 640])]


@pytest.mark.parametrize("new,lens", SHAPES, ids=["-".join(map(str, a + b)) for a, b in SHAPES])
@pytest.mark.parametrize("D,H,Hk,page,layout,kind", [(128, 2, 2, 64, "head", "bf16"), (64, 6, 2, 48, "token", "f16"),
                                                     (128, 5, 1, 16, "padded", "f16"), (64, 3, 3, 100, "head", "bf16"),
                                                     (128, 8, 1, 1000, "token", "bf16")])
@pytest.mark.parametrize("frame", [0, 1, 7])
def test_shapes(new, lens, D, H, Hk, page, layout, kind, frame):
    seed = sum(new) + sum(lens) + page
    c = Cache(lens, Hk, D, page, kind, layout, seed)
    q = randn(seed, (sum(new) + 2, H, D), "bf16")
    check(c, q, new, "f32" if seed % 2 else "bf16", frame=frame)


@pytest.mark.parametrize("frame,window", [(1, 1), (1, 5), (1, 64), (7, 1), (7, 3), (64, 1), (64, 2), (100, 2), (1000, 1)])
@pytest.mark.parametrize("D,kind", [(128, "f16"), (64, "bf16")])
@pytest.mark.parametrize("hint", [0, 1])
def test_windows(frame, window, D, kind, hint):
    new, lens = [1, 5, 150, 1], [400, 300, 411, 64]
    c = Cache(lens, 2, D, 48, kind, "head", frame + window)
    q = randn(frame, (sum(new) + 2, 4, D), "bf16")
    check(c, q, new, "f32", frame=frame, window=window, max_q=150 * hint, max_kv=411 * hint)


@pytest.mark.parametrize("page", [5, 16, 48, 64, 128])
@pytest.mark.parametrize("D,kind", [(128, "bf16"), (64, "f16")])
@pytest.mark.parametrize("new", [[1, 1, 1], [90, 3, 40]], ids=["tokens", "chunks"])
def test_dropped_pages(page, D, kind, new):
    """Pages that are not there, the first, the last and all of a request's among them; what the other pages' unused slots and
    page 0 hold (NaN) does not matter."""
    import torch

    lens = [300, 3, 129]
    c = Cache(lens, 2, D, page, kind, "head", page, drop=(0, 2, 3))
    c.table[1, :] = -1
    c.table[2, (lens[2] - 1) // page] = -7
    used = np.zeros((c.pool, page), bool)
    for r, n in enumerate(lens):
        for at in range(n):
            p = c.table[r, at // page]
            if 0 <= p < c.pool:
                used[p, at % page] = True
    unused = torch.from_numpy(~used).cuda()
    c.k[unused] = float("nan")
    c.v[unused] = float("nan")
    q = randn(page, (sum(new) + 2, 4, D), "bf16")
    for frame, window in ((0, 0), (1, 0), (20, 2)):
        check(c, q, new, "bf16", frame=frame, window=window, what="frame %d" % frame)


@pytest.mark.parametrize("bad", ["nan", "inf", "-inf"])
@pytest.mark.parametrize("where", ["k", "v", "kv"])
@pytest.mark.parametrize("new", [[1, 2], [40, 150], [150, 3]], ids=str)
@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_masked_keys_may_hold_anything(bad, where, new, kind):
    """A key that some rows see and some do not holds a NaN or an infinity: those that do not are as without it."""
    lens = [260, 200]
    c = Cache(lens, 1, 128, 64, kind, "head", 3)
    q = randn(1, (sum(new), 2, 128), "bf16")
    frame = 5
    want, want_lse = run(c, q, new, "f32", 0, frame=frame)
    for r in range(2):  # the last token but one of the chunk's last frame but one
        at = lens[r] // frame * frame - 1 if new[r] > 5 else lens[r] - 1
        page, slot = c.table[r, at // 64], at % 64
        if "k" in where:
            c.k[page, slot, 0, 77] = float(bad)
        if "v" in where:
            c.v[page, slot, 0, 33] = float(bad)
    got, lse = run(c, q, new, "f32", 0, frame=frame)
    hidden = np.zeros(sum(new), bool)
    for r in range(2):
        at = lens[r] // frame * frame - 1 if new[r] > 5 else lens[r] - 1
        for i in range(new[r]):
            hidden[c.q_start[r] + i] = R.seen(lens[r] - new[r] + i, lens[r], frame, 0)[1] <= at
    # (the rows that do not see it take another path to the same sums)
    assert np.allclose(got[hidden], want[hidden], rtol=0, atol=2.0 ** -9 if kind == "f16" else 2.0 ** -6)
    assert np.array_equal(lse[:, hidden], want_lse[:, hidden])
    if where == "v":
        others = [x for x in range(128) if x != 33]
        assert not np.any(np.isfinite(got[~hidden][:, :, 33])) and np.all(np.isfinite(got[~hidden][:, :, others]))
    if bad == "nan" and "k" in where:
        assert np.all(np.isnan(got[~hidden])) and np.all(np.isnan(lse[:, ~hidden]))


@pytest.mark.parametrize("q_type", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("new", [[3], [70]], ids=str)
def test_query_types(q_type, kind, new):
    """Rounded to the cache's type where theirs is another; fp16 saturates."""
    import torch

    c = Cache([150], 1, 64, 32, kind, "head", 2)
    q = randn(1, (sum(new), 3, 64), q_type)
    if kind == "f16" and q_type != "f16":
        q[0, 0, 5] = 1e6
        c.k[..., 5] = 0  # (finite scores all the same)
    rounded = q.float().clamp(-65504, 65504).half() if kind == "f16" else q.bfloat16()
    check(c, q, new, "f32", tail=0, q_rounded=host(rounded), frame=1)


@pytest.mark.parametrize("scale", [0.01, 1.0, 3.0])
def test_scale_and_peaky_rows(scale):
    """Softmaxes that are nearly one-hot, whose maximum moves from tile to tile."""
    c = Cache([1000, 500], 1, 128, 64, "f16", "head", 5)
    q = randn(5, (70 + 1, 2, 128), "bf16")
    check(c, q, [70, 1], "f32", tail=0, scale=scale, frame=0)
    c = Cache([1000, 500], 1, 128, 64, "bf16", "head", 6)
    check(c, q, [70, 1], "f32", tail=0, scale=scale, frame=1)


def test_extreme_scores():
    """Scores of +-1e9: one key has all the weight; all scores equal: all have the same."""
    import torch

    for new in ([1], [100]):
        c = Cache([300], 1, 64, 32, "bf16", "head", 7)
        q = randn(1, (new[0], 1, 64), "bf16") * 1e5
        c.k.mul_(1e4)
        out, _ = run(c, q, new, "f32", 0)
        k, _ = R.gather(host(c.k), c.table, 0, 300)
        v, _ = R.gather(host(c.v), c.table, 0, 300)
        best = (host(q)[:, 0].astype(np.float64) @ k[:, 0].astype(np.float64).T).argmax(1)
        assert np.array_equal(out[:, 0], v[best, 0])
        c.k.zero_()
        check(c, q, new, "f32", tail=0)
        torch.cuda.synchronize()


@pytest.mark.parametrize("G", [1, 2, 3, 7, 16, 17, 40])
@pytest.mark.parametrize("new", [[1, 1], [2, 9], [13, 1]], ids=str)
def test_heads_that_share_keys(G, new):
    c = Cache([200, 450], 2, 64, 64, "bf16", "token", G)
    q = randn(G, (sum(new) + 2, 2 * G, 64), "bf16")
    check(c, q, new, "bf16", frame=1)


@pytest.mark.parametrize("max_q,max_kv", [(0, 0), (1, 1), (1, 5000), (2 ** 31 - 1, 2 ** 31 - 1), (150, 640), (33, 64)])
def test_hints_do_not_matter(max_q, max_kv):
    """Right whatever the host says of the counts."""
    new, lens = [1, 150, 5, 33], [640, 333, 5, 64]
    c = Cache(lens, 2, 128, 64, "bf16", "head", 1)
    q = randn(2, (sum(new) + 2, 4, 128), "bf16")
    check(c, q, new, "bf16", frame=1, max_q=max_q, max_kv=max_kv)


def test_strided_rows_and_in_place():
    """q in a projection's output, head-major output; out over q."""
    import torch

    new, lens = [5, 60], [77, 130]
    c = Cache(lens, 2, 128, 64, "bf16", "head", 1)
    wide = randn(2, (65, 8, 128), "bf16")
    q = wide[:, 2:6]
    args = c.args(new)
    want = host(B.dit_attn_paged_forward(q, *args, frame=1))
    out = torch.empty((4, 65, 128), dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    assert np.array_equal(host(B.dit_attn_paged_forward(q, *args, frame=1, out=out)), want)
    before = host(wide)
    B.dit_attn_paged_forward(q, *args, frame=1, out=q)
    assert np.array_equal(host(q), want)
    assert np.array_equal(host(wide)[:, :2], before[:, :2]) and np.array_equal(host(wide)[:, 6:], before[:, 6:])


def test_many_requests():
    """200 requests of very different lengths, some without tokens, some without keys' pages."""
    rng = np.random.default_rng(3)
    new = rng.integers(0, 4, size=200)
    new[50] = 60
    lens = np.maximum(new, (np.exp(rng.uniform(0, 7, size=200))).astype(int))
    c = Cache(lens, 1, 64, 16, "f16", "head", 3, drop=(2,))
    q = randn(3, (int(new.sum()) + 2, 2, 64), "bf16")
    for hint in (0, 60):
        check(c, q, list(new), "bf16", frame=1, max_q=hint)


def test_counts_out_of_range():
    """Counts that make no sense reach no memory outside the tensors; rows are finite or left alone."""
    import torch

    c = Cache([64, 100], 1, 64, 16, "bf16", "head", 3, extra_pages=0)
    q = randn(1, (12, 2, 64), "bf16")
    args = list(c.args([4, 8]))
    for starts in ([0, -7, 2 ** 31 - 1], [5, 3, 1], [2 ** 31 - 1] * 3, [-2 ** 31, 0, 12], [0, 12, 0], [0, 12, 12]):
        for lens in ([64, 100], [-1, 2 ** 31 - 1], [0, 0], [2, 3], [2 ** 31 - 1, -2 ** 31]):
            for frame, window in ((0, 0), (1, 0), (3, 2), (2 ** 31 - 1, 2 ** 31 - 1)):
                args[3], args[4] = ints(starts), ints(lens)
                out = torch.zeros((12, 2, 64), dtype=torch.bfloat16, device="cuda")
                B.dit_attn_paged_forward(q, *args, frame=frame, window=window, out=out)
                assert torch.isfinite(out).all()


def test_more_new_tokens_than_tokens():
    """kv_len below the number of new tokens: the first ones lie before place 0 and, causal, see nothing."""
    c = Cache([3, 40], 1, 64, 16, "bf16", "head", 3)
    q = randn(1, (70, 2, 64), "bf16")
    for frame in (0, 1, 4):
        check(c, q, [20, 50], "f32", tail=0, frame=frame)


def test_deterministic():
    new, lens = [1, 1, 40], [3000, 100, 2000]
    c = Cache(lens, 2, 128, 64, "bf16", "head", 1)
    q = randn(2, (sum(new), 10, 128), "bf16")
    args = c.args(new)
    first = B.dit_attn_paged_forward(q, *args, frame=1, want_lse=True)
    for _ in range(4):
        again = B.dit_attn_paged_forward(q, *args, frame=1, want_lse=True)
        assert all(np.array_equal(host(a), host(b)) for a, b in zip(first, again))


def test_cache_beyond_32_bit_offsets():
    """Pages past 2^32 bytes and 2^32 elements of the first."""
    import torch

    page, Hk, D = 256, 8, 128
    pages = 2 ** 32 // (page * Hk * D) + 40  # more than 2^32 elements
    cache = [torch.zeros((pages, Hk, page, D), dtype=torch.bfloat16, device="cuda").transpose(1, 2) for _ in range(2)]
    ids = [0, pages - 1, pages // 2 + 7, 3, pages - 30]
    new, lens = [600, 1], [900, 300]
    table = np.full((2, 5), -1, np.int32)
    table[0, :4], table[1, :2] = ids[:4], [ids[4], ids[0] + 1]
    rows = [randn(i, (1200, Hk, D), "bf16") for i in (1, 2)]
    args = (cache[0], cache[1], ints(table), ints([0, 900, 1200]), ints(lens))
    B.dit_kv_append_forward(rows[0], rows[1], *args)
    for r, first in ((0, 0), (1, 900)):
        for at in (0, 255, 256, lens[r] - 1):
            assert torch.equal(cache[0][int(table[r, at // page]), at % page], rows[0][first + at])
            assert torch.equal(cache[1][int(table[r, at // page]), at % page], rows[1][first + at])
    q = randn(3, (601, Hk, D), "bf16")
    got, lse = B.dit_attn_paged_forward(q, cache[0], cache[1], ints(table), ints([0, 600, 601]), ints(lens), want_lse=True, frame=1)
    # the same rows in a small cache
    small = [torch.zeros((7, page, Hk, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for s, x in zip(small, rows):
        s.view(7 * page, Hk, D)[:900] = x[:900]
        s.view(7 * page, Hk, D)[1024:1324] = x[900:]
    table2 = np.array([[0, 1, 2, 3, -1], [4, 5, -1, -1, -1]], np.int32)
    want, want_lse = B.dit_attn_paged_forward(q, small[0], small[1], ints(table2), ints([0, 600, 601]), ints(lens), want_lse=True,
                                              frame=1)
    assert torch.equal(got, want) and torch.equal(lse, want_lse)


def test_no_tokens():
    import torch

    c = Cache([4], 1, 64, 16, "f16", "head", 1)
    q = torch.empty((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    out, lse = B.dit_attn_paged_forward(q, *c.args([0]), want_lse=True)
    assert out.shape == (0, 2, 64) and lse.shape == (2, 0)


def test_one_request_of_almost_all_keys():
    """500 requests of one token, planned with 22 pieces each, of which one has 2^31 - 65,536 keys (a page of 65,536, over and
    over): it gets some 11,000 pieces.  Its sum of exponentials is 32,767 times the page's."""
    import torch

    n, page, D, columns = 500, 65536, 64, 32767
    k, v = (randn(i, (2, page, 1, D), "bf16") for i in (1, 2))
    table = np.full((n, columns), 1, np.int32)
    table[7] = 0
    lens = np.full(n, 3)
    lens[7] = columns * page
    q = randn(3, (n, 1, D), "bf16")
    out, lse = B.dit_attn_paged_forward(q, k, v, ints(table), ints(np.arange(n + 1)), ints(lens), frame=0, max_q=1, want_lse=True,
                                        out=torch.empty((n, 1, D), device="cuda"))
    s = k[0, :, 0].double() @ q[7, 0].double() / 8
    p = (s - s.max()).exp()
    want = (p @ v[0, :, 0].double()) / p.sum()
    # P rounded by 2^-9 of itself (half a step), sums over 2^17 keys a piece and lane and over the pieces
    assert (out[7, 0].double() - want).abs().max() <= (2.0 ** -8 + 2.0 ** -10) * (p @ v[0, :, 0].double().abs() / p.sum()).max()
    assert abs(float(lse[0, 7]) - float(s.max() + p.sum().log()) - np.log(columns)) <= 2.0 ** -9
    s = (k[1, :3, 0].double() @ q[:, 0].double().T).T / 8
    want = s.softmax(1) @ v[1, :3, 0].double()
    others = [r for r in range(n) if r != 7]
    assert (out[others, 0].double() - want[others]).abs().max() <= (2.0 ** -8 + 2.0 ** -18) * v[1, :3].abs().max().double()
