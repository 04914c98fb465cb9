"""luq_cross_entropy_fwd and luq_cross_entropy_bwd against plain forms in 64 bits, through the C ABI."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from gpu_util import announce, host  # noqa: E402
import lm_util  # noqa: E402
import step_util as S  # noqa: E402

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
TYPES = [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")]
SHAPES = [(1, 1, 1), (1, 100, 64), (2, 5, 8), (3, 129, 65), (16, 127, 40), (33, 500, 96), (64, 128, 128), (65, 1000, 72),
          (128, 256, 64), (130, 257, 200), (257, 1030, 136), (300, 2100, 31), (5, 20000, 24), (700, 130, 520), (1, 3000, 1030)]


@pytest.fixture(scope="module")
def L():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2112_10769_amd as lib
    return lib


def _inputs(T, V, D, xt, tt, seed=0, pad=0.15, idt=torch.int64):
    gen = torch.Generator(device="cuda").manual_seed(seed + T * 7 + V * 3 + D)
    w = torch.randn(V, D, device="cuda", generator=gen) * D ** -0.5
    y = torch.randint(0, V, (T,), device="cuda", generator=gen)
    x = torch.randn(T, D, device="cuda", generator=gen) + 4.0 * torch.rand(T, 1, device="cuda", generator=gen) * w[y] / (
        (w[y] ** 2).sum(1, keepdim=True) + 0.1)
    y[torch.rand(T, device="cuda", generator=gen) < pad] = -1
    dloss = (torch.rand(T, device="cuda", generator=gen) + 0.5) / T
    return x.to(DT[xt]), w.to(DT[tt]), y.to(idt), dloss


def _forward(L, x, w, y, scale, eps, what):
    announce("cross_entropy_fwd", what)
    loss, lse = L.luq_cross_entropy_fwd(x, w, y, scale, eps)
    ref, bound = S.loss(S.f64(x), S.f64(w), host(y), scale, eps, x.dtype == torch.bfloat16, w.dtype == torch.bfloat16)
    for got, r, b, name in zip((loss, lse), ref, bound, ("loss", "lse")):
        g = host(got)
        assert np.array_equal(np.isnan(g), np.isnan(r)), (what, name)
        lm_util.within(np.nan_to_num(g), np.nan_to_num(r), b, (what, name))
    return lse


def _backward(L, x, w, y, dloss, lse, scale, eps, gt, before, what):
    announce("cross_entropy_bwd", what)
    dtable = torch.full(w.shape, float("nan"), dtype=DT[gt], device="cuda") if before is None else before.clone()
    dx, dw = L.luq_cross_entropy_bwd(dloss, x, w, y, lse, scale, eps, before is not None, dtable=dtable)
    ref, bound = S.loss_grad(S.f64(dloss), S.f64(x), S.f64(w), host(y), S.f64(lse), scale, eps, x.dtype == torch.bfloat16,
                             w.dtype == torch.bfloat16, gt == "bf16", None if before is None else S.f64(before))
    lm_util.within(host(dx.float()), ref[0], bound[0], (what, "dx"))
    lm_util.within(host(dw.float()), ref[1], bound[1], (what, "dtable"))
    return dx, dw


@pytest.mark.parametrize("T,V,D", SHAPES)
@pytest.mark.parametrize("xt,tt", TYPES)
def test_loss_and_gradients(L, T, V, D, xt, tt):
    for eps, scale, idt in ((0.0, 1.0, torch.int64), (0.1, -0.7, torch.int32)):
        x, w, y, dloss = _inputs(T, V, D, xt, tt, idt=idt)
        what = (T, V, D, xt, tt, eps)
        lse = _forward(L, x, w, y, scale, eps, what)
        for gt in ("f32", "bf16") if tt == "bf16" else ("f32",):
            got = _backward(L, x, w, y, dloss, lse, scale, eps, gt, None, (*what, gt))
            again = L.luq_cross_entropy_bwd(dloss, x, w, y, lse, scale, eps, dtable=torch.empty_like(got[1]))
            assert all(torch.equal(a, b) for a, b in zip(got, again)), "the order of the sums is fixed"


@pytest.mark.parametrize("gt", ["f32", "bf16"])
def test_accumulate(L, gt):
    """Added to what is there, in one product and in split ones."""
    for T, V, D in ((200, 300, 64), (2000, 100, 40), (70, 9000, 24)):
        x, w, y, dloss = _inputs(T, V, D, "bf16", "bf16")
        lse = _forward(L, x, w, y, 1.0, 0.0, (T, V, D))
        before = (0.01 * torch.randn(V, D, device="cuda")).to(DT[gt])
        _backward(L, x, w, y, dloss, lse, 1.0, 0.0, gt, before, (T, V, D, gt))


def test_padding_and_bad_targets(L):
    """Padding rows may hold anything: NaN and infinities in them reach nothing.  A target beyond the table is NaN in the
    loss and has no gradient.  A batch that is padding throughout."""
    x, w, y, dloss = _inputs(150, 260, 72, "bf16", "bf16", pad=0.0)
    y[5], y[77], y[149] = -1, -100, -1
    clean = x.clone()
    for rows in (5, 77, 149):
        clean[rows] = 0.0
    x[5], x[77, 3], x[149] = float("nan"), float("inf"), -float("inf")
    dloss[5] = float("nan")
    loss, lse = L.luq_cross_entropy_fwd(x, w, y, smoothing=0.1)
    assert (loss[[5, 77, 149]] == 0).all() and (lse[[5, 77, 149]] == 0).all() and torch.isfinite(loss).all()
    good = dloss.clone()
    good[5] = 0.0
    want = L.luq_cross_entropy_bwd(good, clean, w, y, lse, smoothing=0.1)
    got = L.luq_cross_entropy_bwd(dloss, x, w, y, lse, smoothing=0.1)
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and (got[0][[5, 77, 149]] == 0).all()
    y[9], y[10] = 260, 2**31 + 5
    loss, lse = L.luq_cross_entropy_fwd(clean, w, y)
    assert torch.isnan(loss[[9, 10]]).all() and torch.isfinite(loss[11:]).all() and (lse[[9, 10]] == 0).all()
    dx, dw = L.luq_cross_entropy_bwd(good, clean, w, y, lse)
    assert (dx[[9, 10]] == 0).all() and torch.isfinite(dw).all()
    y[:] = -1
    loss, lse = L.luq_cross_entropy_fwd(x, w, y)
    dx, dw = L.luq_cross_entropy_bwd(dloss, x, w, y, lse)
    assert (loss == 0).all() and (lse == 0).all() and (dx == 0).all() and (dw == 0).all()


def test_non_finite_table_reaches_no_padding(L):
    """A NaN in the table is everyone's, but for padding rows."""
    x, w, y, dloss = _inputs(70, 130, 64, "f32", "f32", pad=0.0)
    y[3] = -1
    w[7, 7] = float("nan")
    loss, lse = L.luq_cross_entropy_fwd(x, w, y)
    assert loss[3] == 0 and torch.isnan(loss[:3]).all()
    dx, _ = L.luq_cross_entropy_bwd(dloss, x, w, y, lse)
    assert (dx[3] == 0).all()


@pytest.mark.parametrize("xt,tt", TYPES)
def test_large_and_small_values(L, xt, tt):
    """Logits far from zero and far apart, rows of zeros, subnormal and near-largest fp32 elements."""
    x, w, y, dloss = _inputs(40, 300, 64, xt, tt, pad=0.0)
    x[:10] *= 40.0
    x[10:12] = 0.0
    lse = _forward(L, x, w, y, 1.0, 0.0, ("far", xt, tt))
    _backward(L, x, w, y, dloss, lse, 1.0, 0.0, "f32", None, ("far", xt, tt))
    x, w = torch.zeros(2, 8, device="cuda"), torch.zeros(3, 8, device="cuda")
    x[:, 0] = 3.4e38
    w[0, 0], w[1, 0] = 1e-38, -1e-38
    loss, lse = L.luq_cross_entropy_fwd(x, w, torch.tensor([0, 1], device="cuda"))
    z = torch.tensor([3.4, -3.4, 0.0], dtype=torch.float64)
    want = torch.logsumexp(z, 0) - z[:2]
    # 1e-38 is below the normal numbers, where a bf16 term is a multiple of 2^-133: z is off by 3.4e38 * 2^-134
    assert torch.allclose(loss.cpu().double(), want, rtol=1e-5, atol=2 * 3.4e38 * 2.0 ** -134)


def test_gradient_against_differences(L):
    """Central differences of the 64-bit loss along a random direction: h^2 times the third derivative, below 1e-6."""
    x, w, y, dloss = _inputs(20, 90, 16, "f32", "f32")
    _, lse = L.luq_cross_entropy_fwd(x, w, y, 0.9, 0.1)
    dx, dw = L.luq_cross_entropy_bwd(dloss, x, w, y, lse, 0.9, 0.1)
    rng = np.random.default_rng(0)
    x64, w64, d64, t = S.f64(x), S.f64(w), S.f64(dloss), host(y)

    def value(a, b):
        return (S.loss(a, b, t, 0.9, 0.1, False, False)[0][0] * d64).sum()
    for _ in range(4):
        u, v, h = rng.standard_normal(x64.shape), rng.standard_normal(w64.shape), 1e-4
        num = (value(x64 + h * u, w64 + h * v) - value(x64 - h * u, w64 - h * v)) / (2 * h)
        assert abs(num - (S.f64(dx) * u).sum() - (S.f64(dw) * v).sum()) <= 2e-5


def test_pieces_of_the_vocabulary(L):
    """A batch long enough for several pieces and a table wide enough for whole tiles of each."""
    x, w, y, dloss = _inputs(40000, 5000, 8, "bf16", "bf16")
    loss, lse = L.luq_cross_entropy_fwd(x, w, y)
    dx, dw = L.luq_cross_entropy_bwd(dloss, x, w, y, lse)
    z = x.double() @ w.double().t()
    want = torch.logsumexp(z, 1)
    ok = y >= 0
    assert (lse[ok] - want[ok]).abs().max() < 1e-5
    p = torch.exp(z - lse.double()[:, None])
    p[torch.arange(40000, device="cuda")[ok], y[ok]] -= 1.0
    p *= (dloss.double() * ok)[:, None]
    for got, ref, bound in ((dx, p @ w.double(), p.abs() @ w.double().abs()),
                            (dw, p.t() @ x.double(), p.abs().t() @ x.double().abs())):
        # a term of g and the output's rounding (dx), three terms of g and 40000 / 16 additions in a row (dtable)
        tol = 2 * 2.0 ** -8 if got.dtype == torch.bfloat16 else 2.0 ** -24 + 3000 * 2.0 ** -23
        assert ((got.double() - ref).abs() <= tol * bound + 1e-30).all()


def test_outputs_stay_in_their_rows(L):
    x, w, y, dloss = _inputs(37, 203, 51, "bf16", "bf16")
    out = {n: torch.full(s, 7.0, device="cuda", dtype=d) for n, s, d in (
        ("loss", (39,), torch.float32), ("lse", (39,), torch.float32), ("dx", (39, 51), torch.bfloat16), ("dt", (205, 51), torch.float32))}
    L.luq_cross_entropy_fwd(x, w, y, loss=out["loss"][:37], lse=out["lse"][:37])
    L.luq_cross_entropy_bwd(dloss, x, w, y, out["lse"][:37], dx=out["dx"][:37], dtable=out["dt"][:203])
    assert all((out[n][k:] == 7).all() for n, k in (("loss", 37), ("lse", 37), ("dx", 37), ("dt", 203)))


def test_empty_batch(L):
    w = torch.randn(11, 3, device="cuda").to(torch.bfloat16)
    x, y, none = torch.empty(0, 3, dtype=torch.bfloat16, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda"), torch.empty(0, device="cuda")
    assert L.luq_cross_entropy_fwd(x, w, y)[0].shape == (0,)
    for dt in (torch.float32, torch.bfloat16):
        dw = torch.full((11, 3), 5.0, dtype=dt, device="cuda")
        L.luq_cross_entropy_bwd(none, x, w, y, none, accumulate=True, dtable=dw)
        assert (dw == 5).all()
        L.luq_cross_entropy_bwd(none, x, w, y, none, dtable=dw)
        assert (dw == 0).all()


def test_views_and_streams(L):
    """Operands that are transposed, unaligned or on another stream than the current one."""
    x, w, y, dloss = _inputs(60, 150, 64, "bf16", "bf16")
    want = L.luq_cross_entropy_fwd(x, w, y)
    grads = L.luq_cross_entropy_bwd(dloss, x, w, y, want[1])
    flat = torch.zeros(1 + x.numel(), dtype=torch.bfloat16, device="cuda")
    flat[1:] = x.view(-1)
    for a, b in ((flat[1:].view(60, 64), w), (x, w.t().contiguous().t())):
        got = L.luq_cross_entropy_fwd(a, b, y)
        assert all(torch.equal(p, q) for p, q in zip(got, want))
        got = L.luq_cross_entropy_bwd(dloss, a, b, y, want[1])
        assert all(torch.equal(p, q) for p, q in zip(got, grads))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = L.luq_cross_entropy_fwd(x, w, y)
        back = L.luq_cross_entropy_bwd(dloss, x, w, y, got[1])
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip((*got, *back), (*want, *grads)))


@pytest.mark.parametrize("T,V,D,xt,tt,gt", [(1500, 9100, 72, "bf16", "bf16", "bf16"), (2100, 4300, 1032, "bf16", "bf16", "f32"),
                                            (1111, 6007, 333, "f32", "f32", "f32"), (4100, 2050, 1033, "bf16", "f32", "f32")])
def test_large_tiles(L, T, V, D, xt, tt, gt):
    """Sizes that take the 256 x 256 tiles in every product, with edges in both directions (the references on the GPU, in
    64 bits)."""
    x, w, y, dloss = _inputs(T, V, D, xt, tt)
    announce("cross entropy, large tiles", T, V, D, xt, tt)
    loss, lse = L.luq_cross_entropy_fwd(x, w, y, 1.0, 0.1)
    x64, w64, ok = x.double(), w.double(), y >= 0
    z = x64 @ w64.t()
    want = torch.logsumexp(z, 1)
    row, at = torch.arange(T, device="cuda"), y.clamp(min=0)
    ref = want - 0.9 * z[row, at] - 0.1 * z.mean(1)
    # additions in a row of a logit, of like magnitude as its largest terms' sum
    nx, nw = (1 if xt == "bf16" else 3), (1 if tt == "bf16" else 3)
    ez = (x64.abs() @ w64.abs().t()).amax(1) * (S._chain(S._pairs(nx, nw), D) * 2 + 8) * 2.0 ** -24
    e = 3 * ez + (200 + V / 128) * 2.0 ** -24 * (1 + want.abs())
    assert ((lse - want).abs()[ok] <= e[ok]).all() and ((loss - ref).abs()[ok] <= 2 * e[ok]).all() and (loss[~ok] == 0).all()
    dx, dw = L.luq_cross_entropy_bwd(dloss, x, w, y, lse, 1.0, 0.1, dtable=torch.empty(V, D, dtype=DT[gt], device="cuda"))
    g = torch.exp(z - lse.double()[:, None])
    g -= 0.1 / V
    g[row, at] -= 0.9
    g *= (dloss.double() * ok)[:, None]
    # every g by its logit's error and its roundings to terms
    rel = (ez + 60 * 2.0 ** -24).amax()
    rows, cols = (1 if xt == "bf16" else 3), (1 if gt == "bf16" else 3)
    for got, a, c, terms, k, bf16 in ((dx, g, w64, rows, V, xt == "bf16"), (dw, g.t(), x64 * ok[:, None], cols, T, gt == "bf16")):
        tw = (2 if xt == "bf16" and nw == 3 else nw) if got is dx else (2 if gt == "bf16" and nx == 3 else nx)
        tol = rel + 2.0 ** (-8 * terms) + 2.0 ** (-8 * (tw if (nw if got is dx else nx) > 1 else 9)) + S._chain(S._pairs(terms, tw), k) * 2.0 ** -23
        mag = (a.abs() + 0.1 / V) @ c.abs()   # a g near 0 is off by its parts' errors
        ref = a @ c
        bound = tol * mag + (2.0 ** -8 * ref.abs() * (1 + tol) + 2.0 ** -8 * tol * mag if bf16 else 0)
        assert ((got.double() - ref).abs() <= bound + 1e-30).all(), (got is dx, ((got.double() - ref).abs() / bound).max())


@pytest.mark.parametrize("accumulate", [False, True])
def test_no_tokens_leaves_a_table_of_zeros(L, accumulate):
    """An odd number of bf16 elements on an address of two bytes; its neighbours stay."""
    buf = torch.ones(3 * 5 + 2, dtype=torch.bfloat16, device="cuda")
    dtable = buf[1:16].view(3, 5)
    none = torch.empty(0, device="cuda")
    announce("cross entropy backward without tokens", accumulate)
    dx, _ = L.luq_cross_entropy_bwd(none, torch.empty(0, 5, dtype=torch.bfloat16, device="cuda"), torch.ones(3, 5, dtype=torch.bfloat16, device="cuda"),
                                    torch.empty(0, dtype=torch.int32, device="cuda"), none, accumulate=accumulate, dtable=dtable)
    assert dx.shape == (0, 5) and (dtable == (1 if accumulate else 0)).all() and buf[0] == buf[16] == 1


@pytest.mark.parametrize("T,V,D,xt,tt", [(1000, 129, 700, "f32", "f32"), (33, 1000, 1500, "bf16", "bf16"), (513, 65, 1033, "bf16", "f32")])
def test_few_tiles(L, T, V, D, xt, tt):
    """Sizes of few tiles with long reductions: the sums of a row against 64 bits, and the gradient of a row in the batch
    against that of the row alone, whose tiles are others."""
    x, w, y, dloss = _inputs(T, V, D, xt, tt)
    announce("cross entropy, few tiles", T, V, D, xt, tt)
    loss, lse = L.luq_cross_entropy_fwd(x, w, y, 1.0, 0.1)
    z = x.double() @ w.double().t()
    ok = y >= 0
    want = torch.logsumexp(z, 1)
    ez = (x.double().abs() @ w.double().abs().t()).amax(1) * (S._chain(S._pairs(1 if xt == "bf16" else 3, 1 if tt == "bf16" else 3), D) * 2 + 8) * 2.0 ** -24
    assert ((lse - want).abs()[ok] <= (3 * ez + (200 + V / 128) * 2.0 ** -24 * (1 + want.abs()))[ok]).all()
    dx, dw = L.luq_cross_entropy_bwd(dloss, x, w, y, lse, 1.0, 0.1)
    for r in (0, T // 2, T - 1):
        one, _ = L.luq_cross_entropy_bwd(dloss[r:r + 1], x[r:r + 1].clone(), w, y[r:r + 1], lse[r:r + 1], 1.0, 0.1)
        far = (one.double() - dx[r:r + 1].double()).norm()
        # two results, each off by a rounding of g and the output (2^-8 each in bf16) or by 3 ez of its g and 100 roundings
        size = dx[r:r + 1].double().norm() + dloss[r].abs().double() * w.double().norm(dim=1).amax()
        assert far <= size * (4 * 2.0 ** -8 if xt == "bf16" else 2 * (3 * ez[r] + 100 * 2.0 ** -24)), (r, far, size)


@pytest.mark.parametrize("scale", [1.0, -0.7, 3.0])
@pytest.mark.parametrize("xt,tt", [("bf16", "bf16"), ("f32", "f32")])
def test_one_class_loses_nothing(L, xt, tt, scale):
    """A table of one row: the loss is 0, not the rounding of its logit."""
    x, w, _, _ = _inputs(300, 1, 72, xt, tt)
    loss, lse = L.luq_cross_entropy_fwd(x * 50.0, w, torch.zeros(300, dtype=torch.int64, device="cuda"), scale)
    assert (loss == 0).all() and (lse.abs() > 1).any()


@pytest.mark.parametrize("T,V,D,xt,tt", [(40, 300, 64, "f32", "f32"), (40, 300, 64, "bf16", "bf16"), (509, 8000, 510, "f32", "f32"),
                                         (1500, 9100, 72, "bf16", "bf16")])
def test_losses_of_far_logits(L, T, V, D, xt, tt):
    """Rows predicted well, their target's logit far above the others or not so far: the loss is not below 0, and the
    rounding of the logits' common size is not in it."""
    gen = torch.Generator(device="cuda").manual_seed(T + V)
    w = torch.randn(V, D, device="cuda", generator=gen).to(DT[tt])
    y = torch.randint(0, V, (T,), device="cuda", generator=gen)
    x = w.float()[y] / (w.float()[y] ** 2).sum(1, keepdim=True)
    for size in (5.0, 12.0, 30.0, 1000.0, 1e6, 1e9, 1e30):
        for scale in (1.0, -3.0):
            xs = (x * (size / scale)).to(DT[xt])
            announce("cross entropy, far logits", T, V, D, xt, tt, size, scale)
            loss, lse = L.luq_cross_entropy_fwd(xs, w, y, scale)
            z = scale * (xs.double() @ w.double().t())
            top = z.amax(1)
            row = torch.arange(T, device="cuda")
            rest = torch.logsumexp(z - top[:, None], 1)
            want = rest + (top - z[row, y])
            # every logit is off by its products' additions and its rounding, a row's loss by as much of the others' share twice;
            # the sum, which is 1 at least, and its logarithm by their roundings
            chain = S._chain(S._pairs(1 if xt == "bf16" else 3, 1 if tt == "bf16" else 3), D) * 2 + 8
            ez = abs(scale) * (xs.double().abs() @ w.double().abs().t()).amax(1) * chain * 2.0 ** -24
            off = 1 - torch.exp(z[row, y] - top - rest)
            bound = 2 * ez * torch.clamp(off * torch.exp(torch.clamp(2 * ez, max=700.0)), max=1.0) + (96 + V / 512) * 2.0 ** -24 * (1 + want)
            assert (loss >= 0).all(), (size, scale, loss.min())
            assert ((loss.double() - want).abs() <= bound).all(), (size, scale, ((loss.double() - want).abs() / bound).max())
            assert ((lse.double() - (top + rest)).abs() <= 2 * ez + (96 + V / 512) * 2.0 ** -24 + 2.0 ** -23 * top.abs()).all(), (size, scale)
