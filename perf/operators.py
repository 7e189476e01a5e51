"""The operators of a transformer block in 8 bits, as a list of measurable cases.

A program that serves a video diffusion transformer with 8-bit weights and activations runs four operators around
attention.  Rows are symmetric 8-bit integers with one 32-bit scale each: the values they stand for are q * scale.

  norm    h = x + residual; y = h * gamma / sqrt(mean(h^2) + eps); y to 8-bit rows.  Ahead of each projection; h is the
          new residual stream.
  quant   rows (of attention's output, of a weight matrix), through a GELU or not, to 8-bit rows.
  dequant 8-bit rows read back as 16- or 32-bit numbers.
  linear  y[m, n] = sum_k xq[m, k] wq[n, k] * x_scale[m] * w_scale[n] + bias[n]: the projection itself.

8-bit rows are returned as the values they stand for: the cases of norm and quant read them back with dequant, rounded to
16 bits.  Widths are those of 12 and 40 heads of 128 channels, and four times as much inside the feed-forward layer; token
counts are those of the repository's clips, conditioning sequences and single tokens.

Values: activations are N(0, 1) times a gain for each token, with some channels twenty times as large (what the rows of a
residual stream look like); weights are N(0, 1/K) before they are quantised; normalisation weights 1 + N(0, 0.25^2).
"""
import math

import torch

own = False

DEVICE = "cuda"
EPS = 1e-6


def listed():
    return [
        # One token of the residual stream ahead of its projection: all latency.
        dict(name="norm_token", kind="norm", M=1, N=5120, x="bf16", residual="bf16", gamma=True),
        # The conditioning tokens of a request, odd width, a residual stream kept in 32 bits.
        dict(name="norm_cond_odd", kind="norm", M=769, N=4999, x="bf16", residual="f32", gamma=True),
        # A full clip at 40 heads, between attention and the feed-forward layer.
        dict(name="norm_clip_14b", kind="norm", M=32760, N=5120, x="bf16", residual="bf16", gamma=True),
        # Attention's output of a few image tokens ahead of the output projection, 32-bit rows.
        dict(name="quant_image", kind="quant", M=257, N=5120, x="f32", act="none"),
        # Inside the feed-forward layer of a full clip at 40 heads: GELU, then 8 bits.  The longest rows.
        dict(name="quant_clip_14b", kind="quant", M=32760, N=20480, x="bf16", act="gelu"),
        # 8-bit rows of a short clip at 12 heads read back in 32 bits, an odd number of columns.
        dict(name="dequant_short_odd", kind="dequant", M=1560, N=1537, out="f32"),
        # 8-bit rows of a full clip at 40 heads read back in 16 bits.
        dict(name="dequant_clip_14b", kind="dequant", M=32760, N=5120, out="bf16"),
        # The q/k/v projection of one token at 40 heads: a pass over the weights.
        dict(name="linear_token_14b", kind="linear", M=1, N=15360, K=5120, bias=True, out="bf16"),
        # The way back out of the feed-forward layer for 16 tokens: few rows, a long sum.
        dict(name="linear_few_14b", kind="linear", M=16, N=5120, K=20480, bias=True, out="bf16"),
        # No dimension a multiple of anything, 32-bit rows.
        dict(name="linear_odd", kind="linear", M=769, N=2311, K=1001, bias=True, out="f32"),
        # The q/k/v projection of a short clip at 12 heads.
        dict(name="linear_short_1p3b", kind="linear", M=7800, N=4608, K=1536, bias=True, out="bf16"),
        # The q/k/v projection of a full clip at 40 heads: the largest.
        dict(name="linear_clip_14b", kind="linear", M=32760, N=15360, K=5120, bias=True, out="bf16"),
    ]


# ---- drawn cases ----

def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A row length: whole heads' worth half of the time, any number the other half."""
    n = _log_int(rng, lo, hi)
    return max(128, n // 128 * 128) if rng.random() < 0.5 else n


def _draw_once(rng):
    kind = rng.choice(["norm", "norm", "quant", "dequant", "linear", "linear", "linear"])
    M = _log_int(rng, 1, 32760)
    if kind == "norm":
        return dict(kind=kind, M=M, N=_width(rng, 64, 8192), x=rng.choice(["bf16", "bf16", "f32"]),
                    residual=rng.choice(["none", "bf16", "f32"]), gamma=rng.random() < 0.75)
    if kind == "quant":
        return dict(kind=kind, M=M, N=_width(rng, 64, 20480), x=rng.choice(["bf16", "bf16", "f32"]),
                    act=rng.choice(["none", "gelu"]))
    if kind == "dequant":
        return dict(kind=kind, M=M, N=_width(rng, 64, 20480), out=rng.choice(["bf16", "f32"]))
    return dict(kind=kind, M=M, N=_width(rng, 32, 20480), K=_width(rng, 32, 20480), bias=rng.random() < 0.75,
                out=rng.choice(["bf16", "bf16", "f32"]))


def draw(rng):
    top = [work(c) for c in listed()]
    while True:
        case = _draw_once(rng)
        w = work(case)
        if all(w[k] <= max(t[k] for t in top) for k in w):
            return case


# ---- helpers on a case ----

def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _esize(name):
    return {"none": 0, "f32": 4, "bf16": 2}[name]


def work(case):
    kind, M, N = case["kind"], case["M"], case["N"]
    if kind == "linear":
        K = case["K"]
        return {"bytes": M * K + N * K + 4 * (M + N) + (2 * N if case["bias"] else 0) + _esize(case["out"]) * M * N,
                "flops": 2 * M * N * K}
    if kind == "dequant":
        return {"bytes": M * N * (1 + _esize(case["out"])) + 4 * M, "flops": M * N}
    # the values come back in 16 bits, with the scales
    if kind == "quant":
        return {"bytes": M * N * (_esize(case["x"]) + 2) + 4 * M, "flops": (10 if case["act"] == "gelu" else 3) * M * N}
    return {"bytes": M * N * (_esize(case["x"]) + 2 * _esize(case["residual"]) + 2) + 4 * M + (4 * N if case["gamma"] else 0),
            "flops": 7 * M * N}


# ---- inputs ----

def _rows(M, N, dtype):
    """An [M, N] tensor whose rows start on multiples of 16 bytes."""
    per = 16 // torch.empty(0, dtype=dtype).element_size()
    return torch.empty((M, (N + per - 1) // per * per), dtype=dtype, device=DEVICE)[:, :N]


def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.float32)


def _activations(gen, M, N, dtype):
    x = _randn(gen, M, N)
    x *= torch.exp(0.3 * _randn(gen, M, 1))
    x *= torch.where(torch.rand(N, generator=gen, device=DEVICE) < 0.005, 20.0, 1.0)
    rows = _rows(M, N, dtype)
    rows.copy_(x)
    return rows


def _quantised(gen, M, N, gain):
    """8-bit rows of N(0, gain^2) numbers, and their scales."""
    x = _randn(gen, M, N)
    scale = x.abs().amax(1) / 127
    rows = _rows(M, N, torch.int8)
    rows.copy_(torch.round(x / scale.clamp_min(1e-30)[:, None]))
    return rows, scale * gain


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    s, kind, M, N = {"case": case}, case["kind"], case["M"], case["N"]
    if kind == "linear":
        K = case["K"]
        s["x"], s["x_scale"] = _quantised(gen, M, K, 1.0)
        s["w"], s["w_scale"] = _quantised(gen, N, K, K ** -0.5)
        s["bias"] = (0.1 * _randn(gen, N)).to(torch.bfloat16) if case["bias"] else None
        s["out"] = _rows(M, N, _dtype(case["out"]))
        return s
    if kind == "dequant":
        s["q"], s["scale"] = _quantised(gen, M, N, 1.0)
        s["out"] = _rows(M, N, _dtype(case["out"]))
        return s
    s["x"] = _activations(gen, M, N, _dtype(case["x"]))
    s["gamma"] = s["residual"] = s["h"] = None
    if kind == "norm":
        if case["residual"] != "none":
            s["residual"] = _activations(gen, M, N, _dtype(case["residual"]))
            s["h"] = _rows(M, N, _dtype(case["residual"]))
        if case["gamma"]:
            s["gamma"] = 1.0 + 0.25 * _randn(gen, N)
    s["q"] = _rows(M, N, torch.int8)
    s["scale"] = torch.empty(M, dtype=torch.float32, device=DEVICE)
    s["out"] = _rows(M, N, torch.bfloat16)
    return s


# ---- one pass ----

def _run_own(s):
    from paper_2601_20655_amd import binding as dit

    case = s["case"]
    kind = case["kind"]
    if kind == "linear":
        return dit.dit_linear_quant_forward(s["x"], s["x_scale"], s["w"], s["w_scale"], s["bias"], out=s["out"])
    if kind == "dequant":
        return dit.dit_dequant_rows_forward(s["q"], s["scale"], out=s["out"])
    if kind == "quant":
        dit.dit_quant_rows_forward(s["x"], act=case["act"], q=s["q"], scale=s["scale"])
        return dit.dit_dequant_rows_forward(s["q"], s["scale"], out=s["out"]), s["scale"]
    dit.dit_rms_norm_quant_forward(s["x"], s["gamma"], EPS, residual=s["residual"], h_out=s["h"], q=s["q"],
                                   scale=s["scale"])
    return s["h"], dit.dit_dequant_rows_forward(s["q"], s["scale"], out=s["out"]), s["scale"]


def _gelu(x):
    return 0.5 * x * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (x + 0.044715 * x * x * x)))


def _to_rows(t):
    """t as 8-bit rows (still in 32 bits) and the largest magnitude of each: the row's values are q * amax / 127."""
    amax = t.abs().amax(dim=1)
    inverse = torch.where(amax > 0, 127.0 / amax, 0.0)
    return torch.round(t * inverse[:, None]), amax


def run(s):
    if own:
        return _run_own(s)
    case = s["case"]
    kind = case["kind"]
    if kind == "linear":
        y = s["x"].float() @ s["w"].float().t()
        y = y * (s["x_scale"][:, None] * s["w_scale"][None, :])
        if s["bias"] is not None:
            y = y + s["bias"].float()
        return y.to(_dtype(case["out"]))
    if kind == "dequant":
        return (s["q"].float() * s["scale"][:, None]).to(_dtype(case["out"]))
    if kind == "quant":
        x = s["x"].float()
        q, amax = _to_rows(_gelu(x) if case["act"] == "gelu" else x)
        scale = amax / 127
        return (q * scale[:, None]).to(torch.bfloat16), scale
    h = s["x"].float()
    if s["residual"] is not None:
        h = h + s["residual"].float()
    # the factor 1 / sqrt(mean + eps) is common to a row: it changes the scale and not the 8-bit numbers
    q, amax = _to_rows(h * s["gamma"] if s["gamma"] is not None else h)
    scale = amax * torch.rsqrt((h * h).mean(dim=1) + EPS) / 127
    return None if s["residual"] is None else h.to(s["residual"].dtype), (q * scale[:, None]).to(torch.bfloat16), scale


# ---- the same in 64 bits ----

def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "linear":
        x = s["x"].double() * s["x_scale"].double()[:, None]
        w = s["w"].double() * s["w_scale"].double()[:, None]
        y = torch.mm(x, w.t().contiguous())
        return y if s["bias"] is None else y.add_(s["bias"].double())
    if kind == "dequant":
        return s["q"].double().mul_(s["scale"].double()[:, None])
    y, h = s["x"].double(), None
    if kind == "quant" and case["act"] == "gelu":
        u = y.pow(3).mul_(0.044715).add_(y).mul_((2.0 / math.pi) ** 0.5)
        y = u.tanh_().add_(1.0).mul_(y).mul_(0.5)
    if kind == "norm":
        if s["residual"] is not None:
            h = y = y + s["residual"].double()
        y = y / ((y * y).mean(dim=1, keepdim=True) + EPS).sqrt()
        if s["gamma"] is not None:
            y = y * s["gamma"].double()
    scale = y.abs().amax(dim=1, keepdim=True) / 127
    values = (y / scale).nan_to_num_(0.0).round_().mul_(scale)
    return (values, scale[:, 0]) if kind == "quant" else (h, values, scale[:, 0])
