"""The operators of the paged cache in 64 bits (numpy), and how far a 32-bit computation that rounds once may be from them."""
import numpy as np

HALF = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}  # half a step, relative
TINY = {"bf16": 2.0 ** -134, "f16": 2.0 ** -25, "f32": 2.0 ** -150}  # and absolute, where numbers are subnormal


def turns(pos, split, base):
    """Rotation angle of every pair in turns, reduced to (-1/2, 1/2]: [N, D/2], formed in extended precision."""
    out = []
    two_pi = np.longdouble("6.283185307179586476925286766559")
    for axis, d in enumerate(split):
        for i in range(d // 2):
            t = pos[:, axis].astype(np.longdouble) * (np.longdouble(base) ** (np.longdouble(-2 * i) / d) / two_pi)
            out.append((t - np.rint(t)).astype(np.float64))
    return np.stack(out, 1)


def angle_bound(pos, split, base):
    """What is lost of an angle, radians: 2^-22, and 2^-51 of the angle."""
    out = []
    for axis, d in enumerate(split):
        for i in range(d // 2):
            out.append(2.0 ** -22 + 2.0 ** -51 * np.abs(pos[:, axis].astype(np.float64)) * float(base) ** (-2.0 * i / d))
    return np.stack(out, 1)


def rows(x, pos, split, base, norm=None, gamma=None, eps=0.0):
    """x [N, H, D] normalised (norm: None, "head", "token") and rotated (pos None: not)."""
    x = x.astype(np.float64)
    if norm is not None:
        axes = (2,) if norm == "head" else (1, 2)
        x = x / np.sqrt(np.mean(x * x, axis=axes, keepdims=True) + np.float64(np.float32(eps)))
        if gamma is not None:
            x = x * gamma.astype(np.float64).reshape(1, x.shape[1], x.shape[2])
    if pos is None:
        return x, np.abs(x)
    phi = 2 * np.pi * turns(pos, split, base)[:, None, :]
    a, b = x[..., 0::2], x[..., 1::2]
    y = np.empty_like(x)
    y[..., 0::2] = a * np.cos(phi) - b * np.sin(phi)
    y[..., 1::2] = a * np.sin(phi) + b * np.cos(phi)
    return y, np.repeat(np.hypot(a, b), 2, axis=-1)


def rows_tolerance(y, mag, kind, norm, bound=0.0):
    """mag: magnitude of the pair.  Rotation: two products and a sum, 4 roundings of mag at the most, and the angle's error.
    Normalisation: a sum of squares of at most 64 terms a lane, 6 steps over the lanes and 16 over the wavefronts is off by 86
    roundings, its root by half of them; mean, eps, root, reciprocal, product and weight are 7 more: 50."""
    r = (4 + (50 if norm is not None else 0)) * 2.0 ** -24
    if not np.isscalar(bound):
        bound = np.repeat(bound, 2, axis=-1)[:, None, :]
    return mag * (r + bound) * (1 + HALF[kind]) + np.abs(y) * HALF[kind] + TINY[kind]


def check_rows(got, y, mag, kind, norm, bound=0.0, what=""):
    got = got.astype(np.float64)
    assert np.all(np.isfinite(got)), what
    over = np.abs(got - y) - rows_tolerance(y, mag, kind, norm, bound)
    assert over.max() <= 0, "%s: beyond tolerance by %g at %s" % (what, over.max(), np.unravel_index(over.argmax(), over.shape))


def seen(p, keys, frame, window):
    """First and one past the last key that the token at place p sees of `keys`."""
    if not frame:
        return 0, keys
    f = p // frame
    return (max(0, (f - window + 1) * frame) if window else 0), max(0, min(keys, (f + 1) * frame))


def gather(cache, table, r, keys):
    """Rows [keys, Hk, D] of request r in cache [pages, page_size, Hk, D], and whether they are there."""
    n = np.arange(keys)
    page = table[r][n // cache.shape[1]]
    there = (page >= 0) & (page < cache.shape[0])
    return cache[np.where(there, page, 0), n % cache.shape[1]], there


def attend(q, k_cache, v_cache, table, q_start, kv_len, frame=0, window=0, scale=None, p_half=0.0):
    """(out [N, H, D], lse [H, N], tolerance of out without its own rounding, of lse); rows of no request: NaN.

    Tolerances: the products of a score are exact and summed in fp32, D + 8 roundings of sum |q k|; a probability is off by
    that much and rounded to p_half; sums over n keys take n + 64 roundings.  Numerator and denominator each."""
    N, H, D = q.shape
    Hk = k_cache.shape[2]
    G = H // Hk
    scale = D ** -0.5 if scale is None else scale
    out = np.full((N, H, D), np.nan)
    lse = np.full((H, N), np.nan)
    tol, ltol = np.zeros((N, H, D)), np.zeros((H, N))
    for r in range(len(kv_len)):
        new, keys = int(q_start[r + 1] - q_start[r]), int(kv_len[r])
        if new <= 0:
            continue
        k, there = gather(k_cache, table, r, keys)
        v, _ = gather(v_cache, table, r, keys)
        for i in range(new):
            t = q_start[r] + i
            lo, hi = seen(keys - new + i, keys, frame, window)
            at = np.arange(keys)
            at = at[(at >= lo) & (at < hi) & there]
            if len(at) == 0:
                out[t], lse[:, t] = 0, -np.inf
                continue
            for h in range(H):
                kk, vv = k[at, h // G].astype(np.float64), v[at, h // G].astype(np.float64)
                x = q[t, h].astype(np.float64)
                s = scale * (kk @ x)
                top = s.max()
                w = np.exp(s - top)
                total = w.sum()
                out[t, h] = w @ vv / total
                lse[h, t] = top + np.log(total)
                err = scale * (np.abs(kk) @ np.abs(x)).max() * (D + 8) * 2.0 ** -24 + (len(at) + 64) * 2.0 ** -24
                ltol[h, t] = err + 2.0 ** -22 * (1 + np.abs(lse[h, t]))
                tol[t, h] = (p_half + 2 * err + 2.0 ** -20) * (w @ np.abs(vv) / total)
    return out, lse, tol, ltol


def check_attn(got, lse, ref, kind, what=""):
    out, ref_lse, tol, ltol = ref
    got = got.astype(np.float64)
    live = ~np.isnan(out)
    assert np.all(np.isfinite(got[live])), "%s: not finite" % what
    over = np.where(live, np.abs(got - out) - tol * (1 + HALF[kind]) - np.abs(out) * HALF[kind] - TINY[kind], -1.0)
    assert over.max() <= 0, "%s: out beyond tolerance by %g at %s" % (what, over.max(), np.unravel_index(over.argmax(), over.shape))
    if lse is not None:
        some = np.isfinite(ref_lse)
        assert np.array_equal(np.isneginf(lse) & ~np.isnan(ref_lse), np.isneginf(ref_lse)), what
        over = np.abs(lse[some].astype(np.float64) - ref_lse[some]) - ltol[some]
        assert over.max(initial=-1.0) <= 0, "%s: lse beyond tolerance by %g" % (what, over.max())
