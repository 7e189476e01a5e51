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
    """The sum of products is an integer below 2^53: exact in float64, whatever the order.  fp32 rounds it once, the product
    of the scales once, their product once and the sum with the bias once."""
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
# rows / groups of 8 features of a workgroup), that kernel in blocks of 32 rows (/ groups of 8 features), the small tiles (10 x
# 32-row blocks + 64-feature blocks; "any": N cut, or K), tiles of 192 ("64") and 256 ("big") rows x 256 features ("tail": K
# cut; "rest": the last N % 8 features in a call of their own).
KERNELS = [
    ("few1/1", 3, 173, 1959), ("few1/2", 2, 3116, 2259), ("few1/3", 7, 4146, 1738), ("few1/4", 4, 7456, 1920),
    ("few2/1", 14, 605, 2141), ("few2/2", 14, 2376, 1664), ("few2/3", 12, 8960, 1920), ("few2/4", 13, 7840, 2432),
    ("few4/1", 28, 8, 2432), ("few4/2", 30, 3234, 1729), ("few4/3", 21, 4368, 2304), ("few4/4", 17, 7752, 1664),
    ("few8/1", 47, 48, 1664), ("few8/2", 52, 2396, 1860), ("few8/3", 33, 4169, 2196), ("few8/4", 33, 6220, 1706),
    ("blocks/1", 634, 8, 2176), ("blocks/2", 1957, 16, 2048), ("blocks/3", 1149, 24, 1795),
    ("blocks/4", 95, 432, 1792), ("11", 19, 8360, 1920), ("11 any", 18, 8839, 1919), ("21", 34, 8512, 1664),
    ("21 any", 4332, 66, 1675), ("22", 5738, 136, 1664), ("22 any", 5445, 143, 1687), ("42", 5785, 296, 1664),
    ("42 any", 5782, 261, 1708), ("34", 544, 6536, 1664), ("34 any", 513, 6555, 1801), ("44", 581, 9344, 1536),
    ("44 any", 4055, 1300, 1732), ("54", 5409, 1296, 1664), ("54 any", 1051, 7375, 2048), ("64", 5742, 1304, 1792),
    ("64 tail", 5433, 1352, 1845), ("64 rest", 3654, 2301, 1792), ("64 tail rest", 5405, 1313, 1686),
    ("big", 2819, 4360, 1536), ("big tail", 1231, 9376, 1800), ("big rest", 1383, 8357, 1664),
    ("big tail rest", 1177, 9455, 1694),
]
