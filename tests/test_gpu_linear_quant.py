"""The projection of 8-bit rows (dit_linear_quant_forward) against exact integer sums, scaled and biased in 64 bits."""
import numpy as np
import pytest

import quant_ref as R
from paper_2601_20655_amd import binding as B
from paper_2601_20655_amd import workloads as wl

pytestmark = pytest.mark.gpu


def int8_rows(a, pad=0, fill=55):
    """a [M, K] int8 on the device, rows starting on multiples of 16 bytes, what lies between them filled with `fill`."""
    import torch

    M, K = a.shape
    buf = torch.full((M, (K + 15) // 16 * 16 + 16 * pad), fill, dtype=torch.int8, device="cuda")
    buf[:, :K] = torch.from_numpy(a).cuda()
    return buf[:, :K]


def operands(M, N, K, seed, lo=-128, hi=128):
    rng = np.random.default_rng(seed)
    x = rng.integers(lo, hi, size=(M, K)).astype(np.int8)
    w = rng.integers(lo, hi, size=(N, K)).astype(np.int8)
    xs = np.exp(0.5 * rng.standard_normal(M)).astype(np.float32) * np.float32(0.02)
    ws = np.exp(0.5 * rng.standard_normal(N)).astype(np.float32) * np.float32(0.02 * K ** -0.5)
    bias = wl.bf16_bits_to_f32(wl.f32_to_bf16_bits(rng.standard_normal(N).astype(np.float32)))
    return x, xs, w, ws, bias


def run(x, xs, w, ws, bias, out, pad=0):
    """The call on padded operands, its output inside a guard that is checked."""
    import torch

    M, N = x.shape[0], w.shape[0]
    dt = torch.float32 if out == "f32" else torch.bfloat16
    per = 4 if out == "f32" else 8
    buf = torch.full((M + 2, (N + per - 1) // per * per + 2 * per), -77.0, dtype=dt, device="cuda")
    y = buf[1:M + 1, per:per + N]
    cu = [None if a is None else torch.from_numpy(a).cuda() for a in (xs, ws, bias)]
    got = B.dit_linear_quant_forward(int8_rows(x, pad), cu[0], int8_rows(w, pad), cu[1],
                                     None if bias is None else cu[2].bfloat16(), out=y)
    torch.cuda.synchronize()
    assert got.data_ptr() == y.data_ptr()
    b = buf.float().cpu().numpy()
    assert np.all(b[0] == -77) and np.all(b[M + 1] == -77) and np.all(b[:, :per] == -77) and np.all(b[:, per + N:] == -77)
    return b[1:M + 1, per:per + N]


# one of everything; on, one short of and one past the 16, 32, 64, 128 and 256 that tiles are made of, in each direction
SHAPES = [(1, 1, 1), (1, 8, 64), (2, 3, 5), (16, 16, 16), (17, 15, 127), (1, 5120, 128), (1, 1000, 1000), (5, 777, 129),
          (15, 260, 2048), (16, 4099, 640), (31, 264, 64), (32, 96, 4096), (33, 72, 1001), (63, 130, 384), (64, 2560, 512),
          (65, 129, 255), (100, 3001, 257), (128, 128, 128), (130, 3664, 704), (255, 256, 256), (256, 256, 384),
          (257, 257, 128), (300, 520, 1919), (513, 1000, 640), (600, 520, 192), (769, 2311, 1001), (1031, 3592, 256),
          (1250, 4104, 272), (2783, 144, 128), (3502, 1560, 130), (2500, 3336, 1152)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_shapes(M, N, K, out):
    x, xs, w, ws, bias = operands(M, N, K, seed=M + 3 * N + 7 * K)
    use = bias if (M + N) % 3 else None
    y = run(x, xs, w, ws, use, out, pad=(M + K) % 3)
    R.check_linear(y, x, xs, w, ws, use, out == "bf16", "%dx%dx%d" % (M, N, K))


@pytest.mark.parametrize("i", range(len(R.KERNELS)), ids=["%s_%dx%dx%d" % k for k in R.KERNELS])
def test_every_kernel(i):
    """Each kernel on more blocks of K than its stages hold (test_quant_host.py checks that the shapes run on these kernels),
    in both output types; unit scales and integers, so that a fragment read before its stage has arrived cannot hide."""
    _, M, N, K = R.KERNELS[i]
    x, xs, w, ws, bias = operands(M, N, K, seed=i, lo=-8, hi=9)
    for out in ("f32", "bf16"):
        y = run(x, xs, w, ws, bias, out, pad=i % 3)
        R.check_linear(y, x, xs, w, ws, bias, out == "bf16", R.KERNELS[i][0])
    ones = [np.ones(n, np.float32) for n in (M, N)]
    assert np.array_equal(run(x, ones[0], w, ones[1], None, "f32"), x.astype(np.float32) @ w.astype(np.float32).T)


@pytest.mark.parametrize("M", [1, 4, 16, 17, 40, 64, 300])
@pytest.mark.parametrize("K", [5120, 20480])
def test_long_sums(M, K):
    """All operands -128, the largest sums there are, on some rows and channels; random elsewhere."""
    x, xs, w, ws, bias = operands(M, 136, K, seed=M + K)
    x[M // 2] = -128
    w[::5] = -128
    w[1::7] = 127
    y = run(x, xs, w, ws, bias, "f32")
    R.check_linear(y, x, xs, w, ws, bias, False, "M=%d K=%d" % (M, K))


@pytest.mark.parametrize("M", [1, 20, 200])
def test_longest_sum(M):
    """K = 131,071: 128 * 128 * K is the last below 2^31."""
    K = 131071
    x, xs, w, ws, bias = operands(M, 20, K, seed=M)
    x[0] = -128
    w[3] = -128
    y = run(x, xs, w, ws, bias, "f32")
    R.check_linear(y, x, xs, w, ws, bias, False, "M=%d" % M)


@pytest.mark.parametrize("K", [128, 256, 384, 200])
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_many_tiles(K, out):
    """More 256 x 256 tiles than compute units with one to three steps each, ragged both ways; exact: unit scales and
    sums of at most 8 significant bits (bf16) or 24 (fp32)."""
    import torch

    M, N = 6000, 6149
    rng = np.random.default_rng(K)
    hi = 9 if out == "f32" else 2
    x = (rng.integers(-hi + 1, hi, size=(M, K)) * (rng.random((M, K)) < (1.0 if out == "f32" else 0.3))).astype(np.int8)
    w = (rng.integers(-hi + 1, hi, size=(N, K)) * (rng.random((N, K)) < (1.0 if out == "f32" else 0.3))).astype(np.int8)
    bias = rng.integers(-8, 9, size=N).astype(np.float32)
    y = run(x, np.ones(M, np.float32), w, np.ones(N, np.float32), bias, out)
    ref = x.astype(np.float32) @ w.astype(np.float32).T + bias
    if out == "bf16":
        assert np.abs(ref).max() <= 256
    assert np.array_equal(y, ref)


def test_rows_do_not_depend_on_their_neighbours():
    """The same rows in calls of 1, 16, 40, 300 and 3,000 rows (every kernel and tile): the same bits."""
    import torch

    M, N, K = 3000, 2572, 1280
    x, xs, w, ws, bias = operands(M, N, K, seed=4)
    xd, wd = int8_rows(x), int8_rows(w)
    s, t, b = torch.from_numpy(xs).cuda(), torch.from_numpy(ws).cuda(), torch.from_numpy(bias).cuda().bfloat16()
    full = B.dit_linear_quant_forward(xd, s, wd, t, b, out_dtype=torch.float32)
    for m in (1, 16, 40, 300):
        for r in (0, 1234, M - m):
            assert torch.equal(B.dit_linear_quant_forward(xd[r:r + m], s[r:r + m], wd, t, b, out_dtype=torch.float32),
                               full[r:r + m]), (m, r)


@pytest.mark.parametrize("M", [3, 48, 700])
def test_scales_that_are_not_numbers(M):
    """A NaN scale makes its row (its channel) NaN and touches nothing else; a zero scale leaves the bias."""
    import torch

    x, xs, w, ws, bias = operands(M, 300, 256, seed=M)
    xs[1], ws[7], xs[2], ws[100] = np.nan, np.nan, 0, 0
    y = run(x, xs, w, ws, bias, "f32")
    assert np.isnan(y[1]).all() and np.isnan(y[:, 7]).all()
    keep = np.ones(M, bool)
    keep[1] = False
    cols = np.ones(300, bool)
    cols[7] = False
    sub = y[keep][:, cols]
    R.check_linear(sub, x[keep], xs[keep], w[cols], ws[cols], bias[cols], False, "M=%d" % M)
    assert np.array_equal(y[2][cols], bias[cols])


@pytest.mark.parametrize("M", [2, 40, 300, 3000])
def test_scales_whose_product_is_no_normal_number(M):
    """Scales of 2^-75 and 2^-60: their product underflows fp32, sums of a million times as much do not."""
    x, xs, w, ws, _ = operands(M, 520, 640, seed=M)
    xs, ws = np.full(M, 2.0 ** -75, np.float32), np.full(520, 2.0 ** -60, np.float32)
    x[0] = w[0] = 127
    y = run(x, xs, w, ws, None, "f32")
    keep = np.abs(x.astype(np.float64) @ w.astype(np.float64).T) >= 2.0 ** 14  # (normal results)
    ref = (x.astype(np.float64) @ w.astype(np.float64).T) * 2.0 ** -135
    assert np.all(np.abs(y[keep] - ref[keep]) <= 4 * R.U * np.abs(ref[keep])) and y[0, 0] > 0


def test_offsets_beyond_32_bits():
    """Rows of x and y 2^17 bytes and elements apart, 33,000 of them; rows of w as far apart."""
    import torch

    M, N, K, ld = 33000, 72, 144, 1 << 17
    gen = torch.Generator(device="cuda").manual_seed(3)
    xd = torch.randint(-128, 128, (M, K), generator=gen, device="cuda", dtype=torch.int8)
    wd = torch.randint(-128, 128, (N, K), generator=gen, device="cuda", dtype=torch.int8)
    s, t = torch.rand(M, generator=gen, device="cuda"), torch.rand(N, generator=gen, device="cuda")
    x = torch.empty((M, ld), dtype=torch.int8, device="cuda")[:, :K]
    y = torch.empty((M, ld), dtype=torch.bfloat16, device="cuda")[:, :N]
    x.copy_(xd)
    B.dit_linear_quant_forward(x, s, wd, t, out=y)
    assert torch.equal(y, B.dit_linear_quant_forward(xd, s, wd, t))
    # and x as the weights of 72 tokens
    yt = B.dit_linear_quant_forward(wd, t, x, s, out_dtype=torch.float32)
    assert torch.equal(yt, B.dit_linear_quant_forward(wd, t, xd, s, out_dtype=torch.float32))


def test_own_stream_and_graph():
    """On a stream that is not the current one; captured and replayed on new rows, other work between the replays."""
    import torch

    M, N, K = 200, 520, 640
    x, xs, w, ws, bias = operands(M, N, K, seed=8)
    wd, s, t = int8_rows(w), torch.from_numpy(xs).cuda(), torch.from_numpy(ws).cuda()
    xin = [int8_rows(operands(M, N, K, seed=20 + i)[0]) for i in range(3)]
    xd = torch.zeros_like(xin[0])
    few = xd[:3]
    y, yf = (torch.zeros((m, N), dtype=torch.float32, device="cuda") for m in (M, 3))

    def calls(stream=None):
        B.dit_linear_quant_forward(xd, s, wd, t, out=y, stream=stream)
        B.dit_linear_quant_forward(few, s[:3], wd, t, out=yf, stream=stream)

    want = []
    for i in range(3):
        xd.copy_(xin[i])
        calls()
        torch.cuda.synchronize()
        want.append((y.clone(), yf.clone()))
    side = torch.cuda.Stream()
    xd.copy_(xin[0])
    torch.cuda.synchronize()
    calls(side)
    torch.cuda.synchronize()
    assert torch.equal(y, want[0][0]) and torch.equal(yf, want[0][1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for i in (1, 2, 0, 2):
        xd.copy_(xin[i])
        y.zero_()
        yf.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[i][0]) and torch.equal(yf, want[i][1])


@pytest.mark.parametrize("M", [1, 64, 1000])
def test_quantised_rows_through_the_projection(M):
    """Norm, 8-bit rows, 8-bit weights, product: against the same product of the values that the 8-bit rows stand for."""
    import torch

    gen = torch.Generator(device="cuda").manual_seed(M)
    K, N = 1536, 1000
    x = torch.randn((M, K), generator=gen, device="cuda").bfloat16()
    r = torch.randn((M, K), generator=gen, device="cuda").bfloat16()
    wf = torch.randn((N, K), generator=gen, device="cuda") * K ** -0.5
    wq, ws = B.dit_quant_rows_forward(wf)
    q, s, _ = B.dit_rms_norm_quant_forward(x, residual=r)
    y = B.dit_linear_quant_forward(q, s, wq, ws, out_dtype=torch.float32)
    R.check_linear(y.cpu().numpy(), q.cpu().numpy(), s.cpu().numpy(), wq.cpu().numpy(), ws.cpu().numpy(), None, False)
    # and near the product of the numbers themselves: each side off by at most half a scale a number, 1/254 of the row's
    # largest (about 4.5 standard deviations of 1): 2 x 4.5/254/sqrt(3), four standard deviations of the sum's error
    h = (x.double() + r.double()).cpu().numpy()
    ref = (h / np.sqrt((h * h).mean(1, keepdims=True))) @ wf.double().cpu().numpy().T
    assert np.sqrt(np.mean((y.cpu().numpy() - ref) ** 2)) < 2 * 4.5 / 254 / 3 ** 0.5


@pytest.mark.parametrize("M,N,K,bf16,ld", [(27500, 5120, 384, True, 5120), (27500, 5120, 384, True, 5128), (27500, 5121, 200, True, None),
                                           (27500, 5120, 2048, True, 5120), (27500, 5121, 2040, True, None),
                                           (13800, 5120, 384, False, 5124), (13800, 5121, 200, False, None),
                                           (27500, 5128, 2000, False, None)])
def test_output_larger_than_the_caches(M, N, K, bf16, ld):
    """61 rows over and over: integer sums are exact and the rest is done number by number, so the bits are those of a call on
    the 61 alone (another kernel)."""
    import torch

    gen = torch.Generator(device="cuda").manual_seed(N + K)
    of = torch.arange(M, device="cuda") % 61

    def rows(n):
        r = torch.empty((n, (K + 15) // 16 * 16), dtype=torch.int8, device="cuda")[:, :K]
        return r.copy_(torch.randint(-127, 128, (n, K), generator=gen, device="cuda", dtype=torch.int8))

    few, w = rows(61), rows(N)
    x = torch.empty((M, few.stride(0)), dtype=torch.int8, device="cuda")[:, :K].copy_(few[of])
    xs, ws = torch.rand(61, generator=gen, device="cuda"), torch.rand(N, generator=gen, device="cuda")
    bias = torch.randn(N, generator=gen, device="cuda").bfloat16()
    dt = torch.bfloat16 if bf16 else torch.float32
    buf = None if ld is None else torch.full((M, ld), 7.0, dtype=dt, device="cuda")
    y = B.dit_linear_quant_forward(x, xs[of], w, ws, bias, out=None if buf is None else buf[:, :N], out_dtype=dt if buf is None else None)
    want = B.dit_linear_quant_forward(few, xs, w, ws, bias, out_dtype=dt)
    assert torch.equal(y, want[of])
    assert buf is None or torch.all(buf[:, N:] == 7.0)
