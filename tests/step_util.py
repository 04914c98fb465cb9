"""Plain 64-bit forms of the choice of experts, the last layer's loss and AdamW, and the errors that
fp32 and bf16 arithmetic may make in them (test side; no code of the library).

u = 2^-24 is the unit roundoff of fp32; a bf16 term carries 8 bits and is off by 2^-8 of itself at
most, n terms by 2^-8n.  A matrix instruction's additions count as 2u each, should it cut them off.
An exponential of an fp32 argument d is off by |d| u (the argument's rounding) and 4u (its own).
"""
import numpy as np

from lm_util import BF16, U


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


# ---- choice of experts ----------------------------------------------------------------------


def scores(logits, score):
    with np.errstate(all="ignore"):
        if score == "sigmoid":
            return 1.0 / (1.0 + np.exp(-logits))
        top = logits.max(1, keepdims=True)
        e = np.where(logits > -np.inf, np.exp(logits - np.where(np.isfinite(top), top, 0)), 0.0)
        return e / np.maximum(e.sum(1, keepdims=True), 1e-300)


def route(logits, k, score, bias=None, groups=1, top_groups=1, best=1, renorm=True, scale=1.0):
    """(experts, weights, bound of the weights' error), row by row."""
    T, E = logits.shape
    s = scores(logits, score)
    experts, weights, bound = np.full((T, k), -1), np.zeros((T, k)), np.zeros((T, k))
    for t in range(T):
        # without a bias and sums the order of the scores is that of the logits, whose scores may round to 0
        c = logits[t] if bias is None and (groups == 1 or best == 1) else s[t] + (0 if bias is None else bias)
        if np.isnan(logits[t]).any() or np.isposinf(logits[t]).any() or (~(c < np.inf)).any():
            weights[t] = np.nan
            continue
        c = np.where(logits[t] == -np.inf, -np.inf, c)
        if groups > 1:
            size = E // groups
            rank = []
            for g in range(groups):
                top = sorted((v for v in c[g * size:(g + 1) * size] if v > -np.inf), reverse=True)[:best]
                rank.append(sum(top) if top else -np.inf)
            kept = sorted(range(groups), key=lambda g: (-rank[g], g))[:top_groups]
            kept = [g for g in kept if rank[g] > -np.inf]
            c = np.where(np.isin(np.arange(E) // size, kept), c, -np.inf)
        order = sorted((e for e in range(E) if c[e] > -np.inf), key=lambda e: (-c[e], e))[:k]
        experts[t, :len(order)] = order
        if not order:
            continue
        l = logits[t, order]
        if renorm:
            lw = -np.logaddexp(0, -l) if score == "sigmoid" else l
            w = np.exp(lw - lw.max())
            w /= w.sum()
            span = np.abs(l - l.max()).max() + (np.abs(l).max() if score == "sigmoid" else 0)
        else:
            w = s[t, order]
            fin = logits[t][np.isfinite(logits[t])]
            span = min(fin.max() - fin.min(), 104.0) if score == "softmax" else np.abs(l).max()
        weights[t, :len(order)] = w * scale
        # the exponential and those of the sum, a division, the additions in a row of the sum
        bound[t, :len(order)] = np.abs(w * scale) * (2 * span + 30 + E / 64) * U
    return experts, weights, bound


def route_grad(dw, logits, experts, score, renorm, scale, bf16):
    """(gradient of the logits, bound)."""
    T, E = logits.shape
    s = scores(logits, score)
    out, mag = np.zeros((T, E)), np.zeros((T, E))
    span = np.zeros(T)
    for t in range(T):
        at = [(k, e) for k, e in enumerate(experts[t]) if 0 <= e < E]
        if not at:
            continue
        ks, es = [k for k, _ in at], [e for _, e in at]
        d = dw[t, ks] * scale
        l = logits[t]
        fin = l[np.isfinite(l)]
        span[t] = min(fin.max() - fin.min(), 104.0) + (np.abs(l[es]).max() if score == "sigmoid" else 0)
        if renorm:
            lw = -np.logaddexp(0, -l[es]) if score == "sigmoid" else l[es]
            share = np.exp(lw - lw.max())
            share /= share.sum()
            g = share * (d - (d * share).sum())
            m = share * (np.abs(d) + np.abs(d * share).sum())
            if score == "sigmoid":
                rest = 1.0 / (1.0 + np.exp(l[es]))
                g, m = g * rest, m * rest
            np.add.at(out[t], es, g)
            np.add.at(mag[t], es, m)
        else:
            e, a = np.zeros(E), np.zeros(E)
            np.add.at(e, es, d)
            np.add.at(a, es, np.abs(d))
            if score == "sigmoid":
                with np.errstate(all="ignore"):
                    r = np.where(e == 0, 0, e * s[t] * (1.0 / (1.0 + np.exp(l))))
                out[t], mag[t] = r, a * s[t] * np.minimum(1, 1.0 / (1.0 + np.exp(l)))
            else:
                out[t] = s[t] * (e - (e * s[t]).sum())
                mag[t] = s[t] * (a + (a * s[t]).sum())
    bound = mag * (4 * span[:, None] + 60 + E / 32) * U
    if bf16:
        bound = bound + BF16 * np.abs(out) + BF16 * bound
    return out, bound


# ---- cross entropy of the last layer -----------------------------------------------------------


def _pairs(na, nb):
    return sum(1 for i in range(na) for j in range(nb) if i + j <= 2)


def _chain(pairs, k):
    """Additions in a row of a product of `pairs` terms over k, sixteen k an instruction; splits and pieces join."""
    return pairs * (-(-k // 16)) + 16 + 64 + 16


def logits_and_bound(x, w, scale, x_bf16, w_bf16):
    nx, nw = (1 if x_bf16 else 3), (1 if w_bf16 else 3)
    z = scale * (x @ w.T)
    mag = abs(scale) * (np.abs(x) @ np.abs(w).T)
    return z, mag * (_chain(_pairs(nx, nw), x.shape[1]) * 2 * U + 8 * U)


def loss(x, w, targets, scale, eps, x_bf16, w_bf16):
    """((loss, lse), bounds)."""
    z, ez = logits_and_bound(x, w, scale, x_bf16, w_bf16)
    T, V = z.shape
    top = z.max(1)
    e = np.exp(z - top[:, None])
    lse = top + np.log(e.sum(1))
    # every exponential by its logit's error and its argument's rounding; the sums' additions in a row; the logarithm
    p = e / e.sum(1, keepdims=True)
    e_lse = (p * (ez + (np.abs(z) + 2 * np.abs(z - top[:, None]) + 8) * 2 * U)).sum(1) + (64 + V / 512) * U + 6 * U * (
        np.abs(lse) + np.abs(top) + np.log(V) + 1)
    ok = (targets >= 0) & (targets < V)
    y = np.where(ok, targets, 0)
    row = np.arange(T)
    zy, ezy = z[row, y], ez[row, y]
    value = lse - (1 - eps) * zy - eps / V * z.sum(1)
    e_loss = e_lse + ezy + 4 * U * (np.abs(lse) + np.abs(zy)) + eps * (ez.mean(1) + (96 + V / 512) * U * np.abs(z).mean(1))
    value = np.where(targets < 0, 0.0, np.where(ok, value, np.nan))
    return (value, np.where(ok, lse, 0.0)), (np.where(ok, e_loss, 0.0), np.where(ok, e_lse, 0.0))


def loss_grad(dloss, x, w, targets, lse, scale, eps, x_bf16, w_bf16, g_bf16, before=None):
    """((dx, dtable), bounds), from the lse as it was given."""
    T, V = x.shape[0], w.shape[0]
    ok = (targets >= 0) & (targets < V)
    x = np.where(ok[:, None], x, 0.0)
    z, ez = logits_and_bound(x, w, scale, x_bf16, w_bf16)
    p = np.exp(z - np.where(ok, lse, 0.0)[:, None])
    hot = np.zeros((T, V))
    hot[np.arange(T)[ok], targets[ok]] = 1 - eps
    up = np.where(ok, dloss * scale, 0.0)[:, None]
    g = up * (p - hot - eps / V)
    eg = np.abs(up) * (p * (ez + (np.abs(z) + 2 * np.abs(z - np.where(ok, lse, 0.0)[:, None]) + 8) * 2 * U)
                       + 4 * U * (p + hot + eps / V))
    nx, nw = (1 if x_bf16 else 3), (1 if w_bf16 else 3)
    rows, cols = (1 if x_bf16 else 3), (1 if g_bf16 else 3)
    tx, xt = (2 if x_bf16 and nw > 2 else nw), (2 if g_bf16 and nx > 2 else nx)
    ag, ax, aw = np.abs(g), np.abs(x), np.abs(w)

    def product(a, e, b, terms_a, terms_b, exact_b, k):
        """|a| |b| times: a's error, both roundings to terms, the additions."""
        terms = BF16 ** terms_a + (0 if exact_b else BF16 ** terms_b) + 4 * U
        chain = _chain(_pairs(terms_a, terms_b), k) * 2 * U
        return e @ b + (terms + chain) * (a @ b)
    dx, e_dx = g @ w, product(ag, eg, aw, rows, tx, w_bf16, V)
    dw, e_dw = g.T @ x, product(ag.T, eg.T, ax, cols, xt, x_bf16, T)
    if before is not None:
        dw = dw + before
        e_dw = e_dw + 2 * U * np.abs(dw)
    if x_bf16:
        e_dx = e_dx + BF16 * (np.abs(dx) + e_dx)
    if g_bf16:
        e_dw = e_dw + BF16 * (np.abs(dw) + e_dw)
    return (dx, dw), (e_dx + 1e-37, e_dw + 1e-37)


# ---- AdamW -----------------------------------------------------------------------------------

GRID = np.array([m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)])[:127]


def decode(codes, scale):
    """Values of e4m3 codes (OCP), 32 of them over a power of two."""
    codes = codes.astype(np.int64)
    v = np.where(codes & 127 == 127, np.nan, GRID[np.minimum(codes & 127, 126)])
    return np.where(codes & 128, -v, v) * np.repeat(2.0 ** (scale.astype(np.float64) - 127), 32)[:codes.size]


def adamw(p, g, m, v, t, lr, wd, b1, b2, eps, gs=1.0):
    """((p, m, v), bounds)."""
    g = g * gs
    m1, v1 = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    step = lr / (1 - b1 ** t) * m1 / (np.sqrt(v1) / np.sqrt(1 - b2 ** t) + eps)
    e_m = 4 * U * (np.abs(b1 * m) + np.abs((1 - b1) * g))
    with np.errstate(all="ignore"):
        e_step = np.abs(step) * 16 * U + np.where(m1 == 0, 0, np.abs(step / np.where(m1 == 0, 1, m1))) * e_m
    p1 = p - lr * wd * p - step
    return (p1, m1, v1), (3 * U * (np.abs(p) + np.abs(p1)) + e_step, e_m + 1e-44, 6 * U * v1 + 1e-44)


def uniforms(n, tensor, t, seed):
    """16-bit uniforms of n elements: (for m, for the root of v)."""
    from oracle.philox import philox4x32_10
    quad = np.arange(-(-n // 4))
    ctr = np.stack([quad & 0xFFFFFFFF, quad >> 32, np.full_like(quad, tensor), np.full_like(quad, t & 0xFFFFFFFF)], -1)
    words = philox4x32_10(ctr.astype(np.uint32), (seed & 0xFFFFFFFF, seed >> 32)).reshape(-1)[:n].astype(np.int64)
    return words & 0xFFFF, words >> 16


def check_codes(codes, scale, value, err, u, positive, what):
    """Codes of the values (known to within err): the code below, or the one above by the fraction and the uniform."""
    n = value.size
    if n == 0:
        return
    a, blocks = np.abs(value), -(-n // 32)
    top = np.array([a[i * 32:(i + 1) * 32].max() for i in range(blocks)])
    slack = np.array([err[i * 32:(i + 1) * 32].max() for i in range(blocks)])

    def field(x):
        with np.errstate(all="ignore"):
            return np.maximum(np.where(x > 0, np.floor(np.log2(np.where(x > 0, x, 1.0))) + 120, 0), 0)
    assert ((field(np.maximum(top - slack, 0)) <= scale) & (scale <= field(top + slack))).all(), (what, "scales")
    unit = np.repeat(2.0 ** (scale.astype(np.float64) - 127), 32)[:n]
    y, e = a / unit, err / unit
    mag = codes.astype(np.int64) & 127
    low = np.minimum(np.searchsorted(GRID, y, side="right") - 1, 125)
    width = GRID[low + 1] - GRID[low]
    frac, tol = (y - GRID[low]) / width, e / width + 2.0 ** -16
    want = low + (frac + u / 65536 >= 1)
    if positive:     # a root above 0 does not become 0
        want = np.where(a > 0, np.maximum(want, 1), want)
    near = np.abs(frac + u / 65536 - 1) <= tol
    # at a border the value may also lie on the other side of a code
    fine = (mag == want) | (near & ((mag == low) | (mag == low + 1))) | ((frac <= tol) & (mag == low - 1)) | (
        (frac >= 1 - tol) & (mag >= low) & (mag <= low + 2))
    if positive:
        fine &= ~((a > err) & (mag == 0))
    else:
        fine &= (mag == 0) | (a <= err) | ((codes >= 128) == (value < 0))
    assert fine.all(), (what, int((~fine).sum()), np.nonzero(~fine)[0][:5])
    # and hardly any of those known to a thousandth of a step is at a border
    known = tol < 2.0 ** -10
    assert (mag != want)[known].sum() <= 0.01 * known.sum() + 3, (what, "share off")
