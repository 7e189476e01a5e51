"""The 8-bit row operators in 64 bits with numpy, and how far the library's 32-bit arithmetic may be from them."""
import numpy as np

U = 2.0 ** -24  # largest relative error of one fp32 operation
TOP = 127.0


def gelu(x):
    return 0.5 * x * (1.0 + np.tanh(np.sqrt(2.0 / np.pi) * (x + 0.044715 * x ** 3)))


def norm_rows(x, gamma, residual, eps):
    """(h, t, factor): rows y = t * factor[:, None], the factor of a row being 1 / sqrt(mean(h^2) + eps)."""
    h = x.astype(np.float64)
    if residual is not None:
        h = h + residual.astype(np.float64)
    t = h if gamma is None else h * gamma.astype(np.float64)
    return h, t, 1.0 / np.sqrt(np.mean(h * h, axis=1) + eps)


def check_rows(q, scale, t, factor, q_slack=0.0, scale_rel=0.0, what=""):
    """8-bit rows against t (numbers that are quantised, but for a positive factor of the row, which is in the scale alone).

    q = rint(t * (127 * (1 / amax))): t carries at most two roundings (the sum, the product with the weight), amax the same
    two, the quotient and the products one each: seven units of 2^-24 of at most 127, 5.3e-5, by which a number next to a tie
    may fall to the other side.  So q is within 1/2 + 1e-4 (+ q_slack, one number a row) of the unrounded 64-bit number.
    scale = amax * factor / 127: the two roundings of amax and three of its own, and scale_rel for the factor."""
    amax = np.abs(t).max(axis=1)
    with np.errstate(divide="ignore", invalid="ignore"):
        v = np.where(amax[:, None] > 0, t * (TOP / amax)[:, None], 0.0)
    off = np.abs(q.astype(np.float64) - v) - np.broadcast_to(np.asarray(q_slack, dtype=np.float64).reshape(-1, 1), v.shape)
    assert off.max() <= 0.5 + 1e-4, "%s: an integer is %.6f off" % (what, off.max())
    want = amax * factor / TOP
    rel = np.abs(scale.astype(np.float64) - want) / np.where(want > 0, want, 1.0)
    bound = 6 * U + scale_rel
    assert np.all(rel <= bound), "%s: a scale is %.2e off, %.2e allowed" % (what, rel.max(), bound)
    nonzero = amax > 0
    assert np.all(np.abs(q).max(axis=1)[nonzero] == 127), "%s: the largest number of a row is kept" % what


def norm_scale_rel(N):
    """The sum of N squares in fp32: at most N / 64 terms one after the other in a lane, one rounding each (the square is
    fused), a dozen levels of partial sums, half of it after the square root; and the mean, eps, the root, the quotient."""
    return 0.5 * (N / 64.0 + 16) * U + 4 * U


def half_ulp_bf16(x):
    ax = np.maximum(np.abs(x), 1e-38)
    return 2.0 ** (np.floor(np.log2(ax)) - 8)


def check_linear(y, xq, xs, wq, ws, bias, bf16_out, what=""):
    """The sum of products is an integer below 2^53: exact in float64, whatever the order.  fp32 rounds it once, its product
    with the token's scale once, and that times the channel's scale plus the bias once: three of the four units."""
    acc = xq.astype(np.float64) @ wq.astype(np.float64).T
    part = acc * (xs.astype(np.float64)[:, None] * ws.astype(np.float64)[None, :])
    ref = part if bias is None else part + bias.astype(np.float64)[None, :]
    allow = 4 * U * (np.abs(part) + (0.0 if bias is None else np.abs(bias.astype(np.float64))[None, :])) * (1 + 1e-3)
    if bf16_out:
        allow = allow + half_ulp_bf16(ref) * (1 + 2.0 ** -7)
    bad = ~(np.abs(y.astype(np.float64) - ref) <= allow)
    assert not bad.any(), "%s: %d of %d elements beyond the bound, first at %s" % (
        what, int(bad.sum()), bad.size, tuple(np.argwhere(bad)[0]))


# Every kernel of the projection, with at least twice as many blocks of K as a ring of LDS stages holds: few rows (groups of 8
# rows / groups of 8 features of a workgroup), that kernel with several row blocks ("blocks"), the small tiles (10 x 32-row blocks
# + 64-feature blocks; "any": N cut, or K), tiles of 192 ("64") and 256 ("big") rows x 256 features ("tail": K cut; "rest":
# the last N % 8 features in a call of their own).
KERNELS = [
    ("few1/1", 3, 173, 6423), ("few1/2", 6, 2873, 3146), ("few1/3", 7, 4146, 2067), ("few1/4", 5, 7952, 1664),
    ("few2/1", 14, 605, 6528), ("few2/2", 15, 3164, 2124), ("few2/3", 10, 4512, 3456), ("few2/4", 11, 7456, 2304),
    ("few4/2", 23, 3384, 2192), ("few4/3", 21, 4369, 3247), ("few4/4", 18, 7699, 2207), ("few8/3", 34, 4312, 3164),
    ("few8/4", 34, 6252, 3013), ("blocks2/1", 54, 350, 6401), ("blocks2/2", 30, 1395, 3534),
    ("blocks4/1", 4361, 8, 2304), ("blocks4/2", 2602, 31, 3029), ("blocks4/3", 7007, 19, 2258),
    ("blocks4/4", 5478, 31, 1787), ("blocks8/1", 10337, 8, 3200), ("blocks8/2", 8425, 10, 3565),
    ("blocks8/3", 8267, 17, 3187), ("blocks8/4", 8337, 25, 3069), ("11", 33, 5128, 1792), ("11 any", 36, 4408, 1898),
    ("21", 10472, 16, 1792), ("21 any", 8227, 19, 1944), ("22", 8498, 72, 1664), ("22 any", 8394, 66, 1706),
    ("42", 9519, 136, 1792), ("42 any", 9628, 139, 1691), ("34", 11202, 264, 1664), ("34 any", 11084, 281, 1774),
    ("44", 12301, 264, 1664), ("44 any", 12247, 269, 1791), ("54", 8218, 784, 1664), ("54 any", 1418, 5465, 1792),
    ("64", 11060, 536, 1792), ("64 tail", 8497, 784, 1708), ("64 rest", 8205, 871, 1792),
    ("64 tail rest", 10901, 551, 1667), ("big", 12594, 800, 1664), ("big tail", 13681, 808, 1683),
    ("big rest", 12405, 1101, 1664), ("big tail rest", 12403, 769, 1678),
]
