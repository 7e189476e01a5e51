"""The paged-cache operators together, as a program that generates chunk by chunk uses them."""
import numpy as np
import pytest

import paged_ref as R
from paged_util import Cache, host, ints, randn
from paper_2601_20655_amd import binding as B

pytestmark = pytest.mark.gpu
SPLIT = {128: (44, 42, 42), 64: (22, 20, 22)}


def lattice(first, n, hw=(3, 5)):
    at = np.arange(first, first + n)
    return np.stack([at // (hw[0] * hw[1]), at // hw[1] % hw[0], at % hw[1]], 1).astype(np.int32)


@pytest.mark.parametrize("D,H,Hk,kind,page", [(128, 4, 2, "bf16", 64), (64, 3, 3, "f16", 20)])
@pytest.mark.parametrize("norm", [None, "head", "token"])
def test_generation(D, H, Hk, kind, page, norm):
    """Three requests that grow by frames of 15 tokens, one or two at a time, one of which drops pages as it goes; then token by
    token.  Every chunk's rows against the attention over what the cache then holds, the cache against the rows."""
    import torch

    frame, R_ = 15, 3
    total = np.array([75, 60, 92])
    c = Cache(list(total), Hk, D, page, kind, "head", 1)
    c.k.zero_()
    c.v.zero_()
    rng = np.random.default_rng(0)
    gamma = [(1 + 0.25 * rng.standard_normal(h * D)).astype(np.float32) for h in (H, Hk)]
    args = None if norm is None else (norm, 1e-6) + tuple(torch.from_numpy(g).cuda() for g in gamma)
    have = np.zeros(R_, int)
    keys = [np.zeros((n, Hk, D)) for n in total]
    steps = [(15, 30, 15), (15, 0, 45), (30, 15, 30), (15, 15, 0), (0, 0, 1), (0, 0, 1)]
    for step, new in enumerate(steps):
        N = sum(new)
        rows = randn([step, 1], (N, H + 2 * Hk, D), "bf16")
        q, k, v = rows[:, :H], rows[:, H:H + Hk], rows[:, H + Hk:]
        pos = np.concatenate([lattice(have[r], new[r]) for r in range(R_)])
        have = have + new
        c.lens = have
        if step == 3:
            c.table[1, 0] = -1
        call = c.args(new)
        q_out = B.dit_kv_append_forward(k, v, *call, pos=ints(pos), split=SPLIT[D], q=q, norm=args, out_dtype=torch.float32)
        out, lse = B.dit_attn_paged_forward(q_out, *call, frame=frame, max_q=max(new), max_kv=int(max(have)), out_dtype=torch.bfloat16,
                                            want_lse=True)
        # the rows
        y, mag = R.rows(host(k), pos, SPLIT[D], 1e4, norm, gamma[1], 1e-6)
        for r in range(R_):
            at = slice(c.q_start[r], c.q_start[r + 1])
            keys[r][have[r] - new[r]:have[r]] = y[at]
        for r in range(R_):
            got, there = R.gather(host(c.k), c.table, r, have[r])
            tol = R.HALF[kind] * np.abs(keys[r][:have[r]]) + 60 * 2.0 ** -22
            assert np.all((np.abs(got - keys[r][:have[r]]) <= tol)[there]), (step, r)
        # the attention, over what the cache and the q rows hold
        x = host(q_out)
        x = torch.from_numpy(x).to(c.k.dtype).float().numpy()
        ref = R.attend(x, host(c.k), host(c.v), c.table, c.q_start, have, frame, 0, None, R.HALF[kind])
        R.check_attn(host(out), host(lse), ref, "bf16", "step %d" % step)


@pytest.mark.parametrize("grid,H,D", [((3, 5, 7), 2, 128), ((2, 9, 20), 3, 64), ((1, 1, 1), 2, 128)])
@pytest.mark.parametrize("norm", [None, "head", "token"])
def test_one_chunk_is_self_attention(grid, H, D, norm):
    """All tokens of a lattice as one chunk in an fp16 cache: the rows of dit_attn_forward."""
    import torch

    L = grid[0] * grid[1] * grid[2]
    c = Cache([L], H, D, 32, "f16", "head", 1)
    rows = randn(L, (L, 3 * H, D), "bf16")
    q, k, v = (rows[:, i * H:(i + 1) * H] for i in range(3))
    g = [(1 + 0.25 * randn(i, (H * D,), "f32")).contiguous() for i in (7, 8)]
    args = None if norm is None else (norm, 1e-6, g[0], g[1])
    pos = lattice(0, L, grid[1:])
    call = c.args([L])
    q_out = B.dit_kv_append_forward(k, v, *call, pos=ints(pos), split=SPLIT[D], q=q, norm=args, out_dtype=torch.float16)
    out, lse = B.dit_attn_paged_forward(q_out, *call, want_lse=True, out_dtype=torch.float32)
    want, want_lse = B.dit_attn_forward(q[None], k[None], v[None], grid, SPLIT[D], norm=args, want_lse=True, out_dtype=torch.float32)
    # Each side is off by the roundings of q, k (2^-11 each of a score's terms, sum |q k| scale up to 3 D^(1/2)) and of P; q is
    # rounded before the scale is applied here, and after it there.
    rms = float(want.square().mean().sqrt())
    assert float((out - want[0]).abs().max()) <= 2e-2 * max(rms, 0.1)
    assert float((lse - want_lse[0]).abs().max()) <= 4 * 2.0 ** -11 * 3 * D ** 0.5


def test_captured_and_replayed():
    """append and attention in one graph on fixed buffers; counts, tables and rows change between replays, with eager calls of other
    sizes and synchronisations in between.  Every replay against the same calls made eagerly."""
    import torch

    H, Hk, D, page, N = 4, 2, 128, 16, 70
    c = Cache([200, 180, 150], Hk, D, page, "bf16", "head", 1, spare=6)
    rows = randn(1, (N, H + 2 * Hk, D), "bf16")
    q, k, v = rows[:, :H], rows[:, H:H + Hk], rows[:, H + Hk:]
    kc, vc, table, q_start, kv_len = c.args([64, 5, 1])
    pos = ints(lattice(0, N))
    q_out = torch.empty((N, H, D), dtype=torch.bfloat16, device="cuda")
    out, lse = torch.zeros((N, H, D), dtype=torch.bfloat16, device="cuda"), torch.zeros((H, N), device="cuda")
    gamma = (1 + 0.25 * randn(9, (H * D,), "f32"), 1 + 0.25 * randn(10, (Hk * D,), "f32"))
    ws = {}

    def step(kc, vc, q_out, out, lse, key):
        B.dit_kv_append_forward(k, v, kc, vc, table, q_start, kv_len, pos=pos, split=SPLIT[D], q=q, q_out=q_out,
                                norm=("token", 1e-6) + gamma)
        if key not in ws:
            p = B.dit_paged_attn_params(N, H, 15, 0, 64, 200, 0.0, 0, 0, 0, B.dit_strides(0, H * D, D), B.dit_strides(0, H * D, D),
                                        B.kv_cache(kc, vc, table, q_start, kv_len))
            ws[key] = torch.empty(B.dit_attn_paged_workspace_bytes(p), dtype=torch.uint8, device="cuda")
        B.dit_attn_paged_forward(q_out, kc, vc, table, q_start, kv_len, frame=15, max_q=64, max_kv=200, out=out, lse=lse,
                                 workspace=ws[key])

    step(kc, vc, q_out, out, lse, "graph")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step(kc, vc, q_out, out, lse, "graph")
    torch.cuda.synchronize()
    for it, (starts, lens) in enumerate([([0, 64, 69, 70], [200, 180, 150]), ([0, 1, 2, 3], [199, 20, 3]), ([0, 0, 64, 64], [90, 64, 0]),
                                         ([0, 5, 5, 70], [5, 0, 150]), ([0, 0, 0, 0], [3, 4, 5])]):
        rows.copy_(randn([it, 3], tuple(rows.shape), "bf16"))
        pos.copy_(ints(lattice(it * 100, N)))
        q_start.copy_(ints(starts))
        kv_len.copy_(ints(lens))
        table.copy_(ints(np.roll(c.table, it, 1)))
        for t in (q_out, out, lse):
            t.fill_(-7)
        other = [t.clone() for t in (kc, vc, q_out, out, lse)]
        graph.replay()
        if it % 2:
            torch.cuda.synchronize()
        step(*other, "eager")
        B.dit_attn_paged_forward(q[:3], kc, vc, table, ints([0, 1, 1, 3]), kv_len)
        torch.cuda.synchronize()
        for a, b in zip((kc, vc, q_out, out, lse), other):
            assert torch.equal(a, b), it


def test_two_streams():
    """Two steps of other sizes at once on two streams, each with buffers of its own."""
    import torch

    jobs = []
    for seed, (new, lens) in enumerate([([3, 200], [300, 900]), ([1, 1, 1], [700, 70, 7])]):
        c = Cache(lens, 2, 128, 64, "bf16", "head", seed)
        rows = randn(seed, (sum(new), 8, 128), "bf16")
        jobs.append((c, rows, c.args(new), torch.cuda.Stream()))

    def step(c, rows, call, stream):
        q = B.dit_kv_append_forward(rows[:, 4:6], rows[:, 6:], *call, q=rows[:, :4], stream=stream)
        return B.dit_attn_paged_forward(q, *call, frame=1, stream=stream)

    want = []
    for c, rows, call, _ in jobs:
        want.append(host(step(c, rows, call, None)))
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for c, rows, call, stream in jobs:
            with torch.cuda.stream(stream):
                got.append(step(c, rows, call, stream))
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert np.array_equal(host(a), b)


def test_memory_of_another_stream():
    """What a call on another stream allocates is none that work queued on the current stream still writes."""
    import torch

    c = Cache([5000], 2, 128, 64, "bf16", "head", 4)
    q = randn(5, (4, 8, 128), "bf16")
    call = c.args([4])
    want, want_lse = B.dit_attn_paged_forward(q, *call, frame=1, want_lse=True)  # (in pieces: a workspace)
    need = 64 << 20
    side = torch.cuda.Stream()
    busy = torch.randn((4096, 4096), device="cuda")
    torch.cuda.synchronize()
    for _ in range(3):
        for _ in range(20):
            busy = busy @ busy * 1e-3
        late = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in (need, want.numel() * 2, want_lse.numel() * 4)]
        for x in late:
            x.fill_(255)  # runs when the products have
        del late, x
        got, lse = B.dit_attn_paged_forward(q, *call, frame=1, want_lse=True, stream=side)
        side.synchronize()
        kept = got.clone(), lse.clone()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(kept + (got, lse), (want, want_lse) * 2))
