"""Plain 64-bit forms of the operators around the 4-bit products, and the errors that
fp32 arithmetic may make in them (test side; no code of the library).

u = 2^-24 is the unit roundoff of fp32: a sum of n terms, in whatever order, is off by at
most n u times the sum of their magnitudes to first order, and by d u for d additions in a
row on the way to the result.  A bf16 result (8 significant bits) adds up to 2^-8 of itself.
"""
import numpy as np

U = 2.0 ** -24
BF16 = 2.0 ** -8


def group_ids(ids, groups):
    ids = np.asarray(ids, dtype=np.int64)
    key = np.where((ids >= 0) & (ids < groups), ids, groups)
    order = np.argsort(key, kind="stable")
    return order.astype(np.int32), np.searchsorted(key[order], np.arange(groups + 1)).astype(np.int32)


def embedding_grad(dout, ids, vocab, scale):
    """(gradient, bound of its fp32 error)."""
    d = np.asarray(dout, dtype=np.float64)
    grad, mag = np.zeros((vocab, d.shape[1])), np.zeros((vocab, d.shape[1]))
    count = np.zeros(vocab)
    ok = (ids >= 0) & (ids < vocab)
    np.add.at(grad, ids[ok], d[ok])
    np.add.at(mag, ids[ok], np.abs(d[ok]))
    np.add.at(count, ids[ok], 1)
    return grad * scale, (count[:, None] + 2) * U * mag * abs(scale)


def _depth(cols):
    """Additions in a row of a sum over a row: 64 lanes at least share it, then a tree."""
    return cols / 64 + 16


def layernorm(x, gamma, beta, eps, bf16):
    """((y, mean, rstd), bounds of their errors)."""
    x = np.asarray(x, dtype=np.float64)
    cols = x.shape[1]
    g = np.ones(cols) if gamma is None else np.asarray(gamma, dtype=np.float64)
    b = np.zeros(cols) if beta is None else np.asarray(beta, dtype=np.float64)
    mean = x.mean(1, keepdims=True)
    d = x - mean
    var = (d * d).mean(1, keepdims=True)
    rstd = 1.0 / np.sqrt(var + eps)
    y = d * rstd * g + b
    k = _depth(cols)
    e_mean = (k + 2) * U * np.abs(x).mean(1, keepdims=True)
    # the differences to a mean that is off by e add e^2 to the variance
    rel = 0.5 * (e_mean ** 2 + (k + 6) * U * (var + e_mean ** 2)) / (var + eps) + 3 * U
    e_y = np.abs(g) * rstd * (np.abs(d) * (rel + 4 * U) + e_mean) + 2 * U * (np.abs(b) + np.abs(y))
    if bf16:
        e_y = e_y + BF16 * (np.abs(y) + e_y)
    return (y, mean[:, 0], rstd[:, 0]), (e_y, e_mean[:, 0], (rstd * rel)[:, 0])


def layernorm_grad(dy, x, mean, rstd, gamma, bf16):
    """((dx, dgamma, dbeta), bounds), from the statistics as they were given."""
    dy, x = np.asarray(dy, dtype=np.float64), np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    mean, rstd = np.asarray(mean, dtype=np.float64)[:, None], np.asarray(rstd, dtype=np.float64)[:, None]
    g = np.ones(cols) if gamma is None else np.asarray(gamma, dtype=np.float64)
    xh = (x - mean) * rstd
    a = dy * g
    m1, m2 = a.mean(1, keepdims=True), (a * xh).mean(1, keepdims=True)
    dx = rstd * (a - m1 - xh * m2)
    k = _depth(cols)
    e1 = (k + 3) * U * np.abs(a).mean(1, keepdims=True)
    e2 = (k + 6) * U * np.abs(a * xh).mean(1, keepdims=True)
    e_dx = rstd * (e1 + np.abs(xh) * e2 + 8 * U * (np.abs(a) + np.abs(m1) + np.abs(xh * m2)))
    if bf16:
        e_dx = e_dx + BF16 * (np.abs(dx) + e_dx)
    e_gamma = (rows + 5) * U * np.abs(dy * xh).sum(0)
    e_beta = (rows + 1) * U * np.abs(dy).sum(0)
    return (dx, (dy * xh).sum(0), dy.sum(0)), (e_dx, e_gamma, e_beta)


def within(got, ref, bound, what):
    got = np.asarray(got, dtype=np.float64)
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    bad = ~(np.abs(got - ref) <= bound + 1e-300)
    assert not bad.any(), (what, int(bad.sum()), "worst", float(np.nanmax(np.abs(got - ref) / (bound + 1e-300))),
                           "first", [int(v[0]) for v in np.nonzero(bad)])


# ---- 4-bit codes --------------------------------------------------------------------------


def pack(nibbles):
    n = np.asarray(nibbles).astype(np.uint8) & 15
    return np.ascontiguousarray(n[..., 0::2] | (n[..., 1::2] << 4))


def luq_fields(rng, shape, top=5):
    """LUQ codes as signed fields -top .. top (R = 4: fields up to 5)."""
    return rng.integers(-top, top + 1, shape)


def luq_pack(field):
    return pack(np.where(field < 0, -field + 8, field))


def luq_levels(field):
    return np.where(field == 0, 0, np.sign(field) * (1 << np.maximum(np.abs(field) - 1, 0))).astype(np.int64)


def int4_values(rng, shape, signed):
    return rng.integers(-7, 8, shape) if signed else rng.integers(0, 16, shape)
