"""8-bit rows (dit_quant_rows_forward, dit_rms_norm_quant_forward, dit_dequant_rows_forward) against the same in 64 bits.
The bounds are derived in quant_ref.check_rows and norm_scale_rel."""
import numpy as np
import pytest

import quant_ref as R
from paper_2601_20655_amd import binding as B
from paper_2601_20655_amd import workloads as wl

pytestmark = pytest.mark.gpu

# one token to many, one column to the most there may be; odd, on and next to multiples of what a lane, a wavefront and a
# workgroup take at once
SHAPES = [(1, 1), (3, 7), (1, 8), (5, 64), (2, 129), (7, 511), (4, 512), (3, 513), (9, 1000), (1, 1024), (2, 1537),
          (33, 2048), (6, 2056), (17, 2567), (300, 3000), (5, 4096), (1, 4999), (70, 5120), (2, 5121), (3, 7777), (4, 8192),
          (2, 10240), (3, 12289), (5, 20480), (1, 32768), (2, 40001), (2, 65535), (3, 65536)]


def dev_rows(a, bf16, pad=0):
    """a [M, N] float32 on the device as bf16 or float32 rows that start on multiples of 16 bytes, `pad` spare pieces a row."""
    import torch

    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    dt = torch.bfloat16 if bf16 else torch.float32
    per = 8 if bf16 else 4
    M, N = a.shape
    buf = torch.full((M, (N + per - 1) // per * per + per * pad), 999.0, dtype=dt, device="cuda")
    buf[:, :N] = t.to(dt)
    return buf[:, :N]


def rows_of(rng, M, N, bf16, gain=None):
    x = rng.standard_normal((M, N)).astype(np.float32)
    x *= np.exp(0.5 * rng.standard_normal((M, 1))).astype(np.float32) if gain is None else gain
    x[:, rng.random(N) < 0.01] *= 20
    if bf16:
        x = wl.bf16_bits_to_f32(wl.f32_to_bf16_bits(x))
    return x


def guarded_q(M, N, offset=0):
    """An int8 [M, N] view with a guard around it, and the whole buffer."""
    import torch

    ld = (N + 15) // 16 * 16 + 32
    buf = torch.full((M + 2, ld), 77, dtype=torch.int8, device="cuda")
    return buf[1:M + 1, 16:16 + N], buf


def check_guard(buf, M, N):
    b = buf.cpu().numpy()
    assert np.all(b[0] == 77) and np.all(b[M + 1] == 77) and np.all(b[:, :16] == 77) and np.all(b[:, 16 + N:] == 77)


@pytest.mark.parametrize("M,N", SHAPES)
@pytest.mark.parametrize("bf16", [True, False])
def test_quant_rows(M, N, bf16):
    rng = np.random.default_rng(7 * N + M)
    x = rows_of(rng, M, N, bf16)
    q, buf = guarded_q(M, N)
    _, scale = B.dit_quant_rows_forward(dev_rows(x, bf16, pad=1), q=q)
    R.check_rows(q.cpu().numpy(), scale.cpu().numpy(), x.astype(np.float64), 1.0, what="%dx%d" % (M, N))
    check_guard(buf, M, N)


@pytest.mark.parametrize("M,N", SHAPES)
@pytest.mark.parametrize("bf16", [True, False])
def test_quant_rows_gelu(M, N, bf16):
    """GELU in fp32: its argument, tanh, 1 + tanh and the products, sixteen units of 2^-24 of |x| (it does not shrink with
    the result where 1 + tanh cancels)."""
    rng = np.random.default_rng(11 * N + M)
    x = rows_of(rng, M, N, bf16)
    x[:, 0] = np.abs(x[:, 0]) + np.float32(0.5)  # (some number well away from zero in every row)
    if bf16:
        x = wl.bf16_bits_to_f32(wl.f32_to_bf16_bits(x))
    q, buf = guarded_q(M, N)
    _, scale = B.dit_quant_rows_forward(dev_rows(x, bf16), act="gelu", q=q)
    t = R.gelu(x.astype(np.float64))
    slack = 16 * R.U * np.abs(x).max(axis=1) / np.abs(t).max(axis=1)
    R.check_rows(q.cpu().numpy(), scale.cpu().numpy(), t, 1.0, q_slack=127 * slack, scale_rel=slack.max(),
                 what="%dx%d" % (M, N))
    check_guard(buf, M, N)


@pytest.mark.parametrize("M,N", SHAPES)
@pytest.mark.parametrize("x_bf16,residual,gamma", [(True, "bf16", True), (True, "f32", True), (False, "f32", True),
                                                   (False, "bf16", False), (True, "none", True), (False, "none", False)])
def test_norm_quant(M, N, x_bf16, residual, gamma):
    import torch

    rng = np.random.default_rng(13 * N + M)
    x = rows_of(rng, M, N, x_bf16)
    r = None if residual == "none" else rows_of(rng, M, N, residual == "bf16", gain=np.float32(3))
    g = (1 + 0.25 * rng.standard_normal(N)).astype(np.float32) if gamma else None
    q, buf = guarded_q(M, N)
    got = B.dit_rms_norm_quant_forward(dev_rows(x, x_bf16), torch.from_numpy(g).cuda() if gamma else None, 1e-6,
                                       residual=None if r is None else dev_rows(r, residual == "bf16", pad=2), q=q)
    h, t, factor = R.norm_rows(x, g, r, 1e-6)
    R.check_rows(q.cpu().numpy(), got[1].cpu().numpy(), t, factor, scale_rel=R.norm_scale_rel(N), what="%dx%d" % (M, N))
    check_guard(buf, M, N)
    if r is not None:  # one fp32 addition, one rounding to the stream's type: bit for bit
        want = x + r
        if residual == "bf16":
            want = wl.bf16_bits_to_f32(wl.f32_to_bf16_bits(want))
        assert np.array_equal(got[2].float().cpu().numpy(), want)


@pytest.mark.parametrize("alias", ["residual", "x"])
@pytest.mark.parametrize("M,N", [(3, 100), (65, 5120), (2, 20484)])
def test_norm_quant_sum_in_place(alias, M, N):
    """h_out on the residual, or on x: the same bits as with rows of its own, and guards kept."""
    import torch

    rng = np.random.default_rng(N)
    x, r = rows_of(rng, M, N, True), rows_of(rng, M, N, True)
    g = torch.from_numpy((1 + 0.25 * rng.standard_normal(N)).astype(np.float32)).cuda()
    q0, s0, h0 = B.dit_rms_norm_quant_forward(dev_rows(x, True), g, residual=dev_rows(r, True))
    xd, rd = dev_rows(x, True, pad=1), dev_rows(r, True, pad=1)
    into = rd if alias == "residual" else xd
    q1, s1, h1 = B.dit_rms_norm_quant_forward(xd, g, residual=rd, h_out=into)
    assert h1.data_ptr() == into.data_ptr()
    assert torch.equal(q0, q1) and torch.equal(s0, s1) and torch.equal(h0, h1)
    assert torch.all(into.as_strided((M, 8), (into.stride(0), 1), (N + 7) // 8 * 8) == 999.0)


@pytest.mark.parametrize("M,N", [(1, 1), (3, 17), (1560, 1537), (4, 4096), (5, 70001), (769, 5120)])
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_dequant_rows(M, N, out):
    """One product, rounded once: bit for bit."""
    import torch

    rng = np.random.default_rng(N)
    q = rng.integers(-128, 128, size=(M, N)).astype(np.int8)
    scale = np.exp(rng.standard_normal(M)).astype(np.float32)
    qd, _ = guarded_q(M, N)
    qd.copy_(torch.from_numpy(q))
    per = 8 if out == "bf16" else 4
    buf = torch.full((M + 1, (N + per - 1) // per * per + per), -5.0, dtype=torch.bfloat16 if out == "bf16" else torch.float32,
                     device="cuda")
    B.dit_dequant_rows_forward(qd, torch.from_numpy(scale).cuda(), out=buf[:M, :N])
    want = q.astype(np.float32) * scale[:, None]
    if out == "bf16":
        want = wl.bf16_bits_to_f32(wl.f32_to_bf16_bits(want))
    assert np.array_equal(buf[:M, :N].float().cpu().numpy(), want)
    assert torch.all(buf[M] == -5.0) and torch.all(buf[:, N:] == -5.0)


@pytest.mark.parametrize("N", [40, 5120, 20481])
@pytest.mark.parametrize("norm", [False, True])
def test_rows_that_cannot_be_quantised(N, norm):
    """Rows of zeros, of numbers too small to count, with a NaN or an infinity: scale 0 or NaN and integers 0; the rows
    between them are what they are without these neighbours."""
    import torch

    rng = np.random.default_rng(N)
    x = rows_of(rng, 12, N, False, gain=np.float32(1))
    good = [0, 3, 6, 8, 11]
    x[1] = 0
    x[2, N // 2] = np.nan
    x[4, N - 1] = np.inf
    x[5, 0] = -np.inf
    x[7] = 1e-38
    x[9] = -0.0
    x[10, :] = np.nan
    xd = dev_rows(x, False)

    def call(t):
        return B.dit_rms_norm_quant_forward(t, None, 1e-6) if norm else B.dit_quant_rows_forward(t)

    q, scale = (t.cpu().numpy() for t in call(xd))
    q1, scale1 = (t.cpu().numpy() for t in call(xd[good].contiguous() if N % 4 == 0 else dev_rows(x[good], False)))
    assert np.array_equal(q[good], q1) and np.array_equal(scale[good], scale1)
    bad = [1, 2, 4, 5, 7, 9, 10]
    assert not q[bad].any()
    assert np.all(scale[[1, 7, 9]] == 0) and np.all(np.isnan(scale[[2, 4, 5, 10]]))
    back = B.dit_dequant_rows_forward(torch.from_numpy(q).cuda()[:, :N // 8 * 8], torch.from_numpy(scale).cuda(),
                                      out_dtype=torch.float32) if N % 16 == 0 else None
    if back is not None:
        assert torch.all(torch.isnan(back[[2, 4, 5, 10]])) and torch.all(back[[1, 7, 9]] == 0)


def test_norm_of_huge_rows():
    """Squares that overflow fp32 make the row one with an infinity, never one of zeros."""
    x = np.full((2, 64), 1e25, dtype=np.float32)
    x[1] = 1e15
    q, scale = B.dit_rms_norm_quant_forward(dev_rows(x, False), None, 1e-6)
    assert np.isnan(scale[0].item()) and not q[0].any().item()
    assert abs(scale[1].item() * 127 - 1) < 1e-6 and (q[1] == 127).all().item()


def test_quantised_values_do_not_depend_on_the_sum_of_squares():
    """The norm's factor is common to a row: the integers are those of the plain quantisation of h * gamma."""
    import torch

    rng = np.random.default_rng(5)
    x = rows_of(rng, 40, 3001, False)
    g = torch.from_numpy((1 + 0.25 * rng.standard_normal(3001)).astype(np.float32)).cuda()
    q, _ = B.dit_rms_norm_quant_forward(dev_rows(x, False), g)
    t = B._empty_rows(40, 3001, torch.float32, "cuda")
    t.copy_(torch.from_numpy(x).cuda() * g)
    assert torch.equal(q, B.dit_quant_rows_forward(t)[0])


def test_offsets_beyond_32_bits():
    """Rows 2^17 elements apart: the last ones start beyond 2^32 bytes, and beyond 2^32 elements of x."""
    import torch

    M, N, ld = 33000, 72, 1 << 17
    gen = torch.Generator(device="cuda").manual_seed(3)
    dense = torch.randn((M, N), generator=gen, device="cuda").bfloat16()
    x = torch.empty((M, ld), dtype=torch.bfloat16, device="cuda")[:, :N]
    q = torch.empty((M, ld), dtype=torch.int8, device="cuda")[:, :N]
    x.copy_(dense)
    q.fill_(99)
    _, scale = B.dit_quant_rows_forward(x, q=q)
    q1, scale1 = B.dit_quant_rows_forward(dense)
    assert torch.equal(q, q1) and torch.equal(scale, scale1)
    q.fill_(99)
    _, scale, h = B.dit_rms_norm_quant_forward(x, residual=x, h_out=x, q=q)
    q1, scale1, h1 = B.dit_rms_norm_quant_forward(dense, residual=dense)
    assert torch.equal(q, q1) and torch.equal(scale, scale1) and torch.equal(h, h1)
    B.dit_dequant_rows_forward(q, scale, out=x)
    assert torch.equal(x, B.dit_dequant_rows_forward(q1, scale1))


def test_own_stream_and_graph():
    """On a stream that is not the current one, then captured and replayed on new inputs, other work between replays."""
    import torch

    rng = np.random.default_rng(9)
    M, N = 130, 2052
    xs = [torch.from_numpy(rows_of(rng, M, N, True)).cuda().bfloat16() for _ in range(4)]
    g = torch.from_numpy((1 + 0.25 * rng.standard_normal(N)).astype(np.float32)).cuda()
    ld = (N + 7) // 8 * 8

    def rows(dt):
        return torch.zeros((M, ld if dt != torch.int8 else (N + 15) // 16 * 16), dtype=dt, device="cuda")[:, :N]

    x, r, h, y = (rows(torch.bfloat16) for _ in range(4))
    q, scale = rows(torch.int8), torch.zeros(M, device="cuda")
    q2, scale2 = rows(torch.int8), torch.zeros(M, device="cuda")

    def calls(stream=None):
        B.dit_rms_norm_quant_forward(x, g, residual=r, h_out=h, q=q, scale=scale, stream=stream)
        B.dit_dequant_rows_forward(q, scale, out=y, stream=stream)
        B.dit_quant_rows_forward(y, act="gelu", q=q2, scale=scale2, stream=stream)

    def results():
        torch.cuda.synchronize()
        return [t.clone() for t in (h, q, scale, y, q2, scale2)]

    want = []
    for i in range(3):
        x.copy_(xs[i])
        r.copy_(xs[i + 1])
        calls()
        want.append(results())
    x.copy_(xs[0])
    r.copy_(xs[1])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    calls(side)
    assert all(torch.equal(a, b) for a, b in zip(results(), want[0]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for i in (1, 2, 0, 2):
        x.copy_(xs[i])
        r.copy_(xs[i + 1])
        for t in (h, q, scale, y, q2, scale2):
            t.zero_()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(results(), want[i]))


# rows enough that a lane takes several chunks and a workgroup several rows, the last workgroup not full
MANY = [(1101, 203), (1027, 520), (1030, 1001), (1050, 1537), (1026, 2567), (1025, 3333), (1041, 4999), (1024, 5120),
        (521, 7777), (1100, 5121)]


@pytest.mark.parametrize("M,N", MANY)
@pytest.mark.parametrize("bf16", [True, False])
def test_quant_many_rows(M, N, bf16):
    test_quant_rows(M, N, bf16)
    test_quant_rows_gelu(M, N, bf16)


@pytest.mark.parametrize("M,N", MANY)
@pytest.mark.parametrize("x_bf16,residual,gamma", [(True, "bf16", True), (True, "f32", True), (False, "f32", True),
                                                   (False, "bf16", True), (True, "none", True), (False, "none", True)])
def test_norm_quant_many_rows(M, N, x_bf16, residual, gamma):
    test_norm_quant(M, N, x_bf16, residual, gamma)


@pytest.mark.parametrize("N", [5120, 5121])
@pytest.mark.parametrize("residual", ["none", "bf16", "f32"])
def test_rows_larger_than_the_caches(N, residual):
    """61 rows over and over, more than the caches hold: the results of a call on the 61 alone, but for the order in which
    a row's squares are added up, which is in the scale."""
    import torch

    M, base = 27500, 61  # 282 MB of x
    gen = torch.Generator(device="cuda").manual_seed(N)
    of = torch.arange(M, device="cuda") % base

    def rows(dt):
        r = torch.empty((M, (N + 15) // 16 * 16), dtype=dt, device="cuda")[:, :N]
        few = torch.empty((base, (N + 15) // 16 * 16), dtype=dt, device="cuda")[:, :N]
        few.copy_(torch.randn((base, N), generator=gen, device="cuda"))
        r.copy_(few[of])
        return r, few

    x, x0 = rows(torch.bfloat16)
    g = 1 + 0.25 * torch.randn(N, generator=gen, device="cuda")
    r, r0 = (None, None) if residual == "none" else rows(torch.bfloat16 if residual == "bf16" else torch.float32)
    got = B.dit_rms_norm_quant_forward(x, g, residual=r)
    want = B.dit_rms_norm_quant_forward(x0, g, residual=r0)
    assert torch.equal(got[0], want[0][of])
    rel = ((got[1].double() - want[1].double()[of]) / want[1].double()[of]).abs().max().item()
    assert rel <= 2 * (6 * R.U + R.norm_scale_rel(N)), rel
    if r is not None:
        assert torch.equal(got[2], want[2][of])
    for act in ("none", "gelu"):
        q, scale = B.dit_quant_rows_forward(x, act=act)
        q0, scale0 = B.dit_quant_rows_forward(x0, act=act)
        assert torch.equal(q, q0[of]) and torch.equal(scale, scale0[of])
    for dt in (torch.bfloat16, torch.float32):
        y = B.dit_dequant_rows_forward(q, scale, out_dtype=dt)
        assert torch.equal(y, B.dit_dequant_rows_forward(q0, scale0, out_dtype=dt)[of])
