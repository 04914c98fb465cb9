"""Every kernel of the cross entropy (its logits' tiles, the tiles of both gradients with a whole and a split
reduction and their epilogues, one and several pieces of the vocabulary, the joins of few and of many parts) against
the plain form in 64 bits on the GPU.  test_cross_entropy_plan_cpu.py holds that the shapes reach them."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from gpu_util import announce  # noqa: E402
from lm_util import BF16, U  # noqa: E402
import step_util as S  # noqa: E402
from test_gpu_cross_entropy import DT, _inputs  # noqa: E402

# T, V, D, types of x, the table and its gradient, whether it is added to
SHAPES = [
    (1, 33, 8, "f32", "bf16", "bf16", 0), (1, 33, 8, "bf16", "bf16", "f32", 1), (1, 33, 8, "bf16", "f32", "f32", 0),
    (151, 38, 8, "bf16", "bf16", "bf16", 1), (1, 32807, 141, "f32", "bf16", "bf16", 0), (1, 35405, 131, "bf16", "f32", "f32", 1),
    (1, 11147, 664, "f32", "bf16", "bf16", 1), (34, 33397, 8, "f32", "f32", "f32", 0), (1815, 521, 11, "bf16", "bf16", "bf16", 1),
    (38, 37983, 8, "bf16", "bf16", "bf16", 0), (130, 8534, 16, "f32", "bf16", "f32", 1), (508, 5727, 8, "f32", "bf16", "bf16", 1),
    (12118, 278, 8, "bf16", "f32", "f32", 0), (136, 32798, 8, "f32", "bf16", "bf16", 1), (137, 45210, 8, "f32", "f32", "f32", 1),
    (7184, 1060, 8, "bf16", "bf16", "bf16", 0), (1, 71469, 928, "f32", "f32", "f32", 0), (17338, 34, 144, "bf16", "bf16", "bf16", 0),
    (4258, 33, 1328, "f32", "bf16", "f32", 0), (19102, 37, 920, "f32", "f32", "f32", 1), (10038, 13431, 8, "f32", "bf16", "f32", 0),
    (9105, 14817, 8, "bf16", "bf16", "f32", 1), (739, 11847, 134, "f32", "bf16", "f32", 0), (23409, 33, 1992, "bf16", "bf16", "bf16", 0),
    (22297, 6062, 24, "bf16", "bf16", "bf16", 1), (1157, 1729, 1672, "f32", "f32", "f32", 1), (1691, 17795, 153, "f32", "bf16", "bf16", 1),
    (5775, 23519, 136, "bf16", "bf16", "bf16", 0), (509, 8000, 510, "f32", "f32", "f32", 0), (1000, 33003, 515, "bf16", "bf16", "f32", 1),
    (16011, 1003, 1032, "bf16", "bf16", "f32", 0), (40011, 3403, 264, "f32", "f32", "f32", 0), (33011, 4099, 1032, "f32", "bf16", "f32", 1),
    (8111, 16561, 4096, "bf16", "bf16", "bf16", 0)]


@pytest.fixture(scope="module")
def L():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2112_10769_amd as lib
    return lib


def _logits(x, w, scale, nx, nw):
    """z and its bound: the additions of a product's terms in a row, and eight roundings."""
    ez = x.abs() @ w.abs().t()
    ez *= abs(scale) * (S._chain(S._pairs(nx, nw), x.shape[1]) * 2 * U + 8 * U)
    return scale * (x @ w.t()), ez


def _loss(z, ez, y, eps):
    """((loss, lse), bounds) of rows with a target; as step_util.loss."""
    V = z.shape[1]
    top = z.amax(1)
    lse = torch.logsumexp(z, 1)
    p = torch.exp(z - lse[:, None])
    e_lse = (p * (ez + (z.abs() + 2 * (z - top[:, None]).abs() + 8) * 2 * U)).sum(1) + (64 + V / 512) * U + 6 * U * (
        lse.abs() + top.abs() + torch.log(torch.tensor(float(V))).item() + 1)
    row = torch.arange(z.shape[0], device="cuda")
    zy = z[row, y]
    e_loss = e_lse + ez[row, y] + 4 * U * (lse.abs() + zy.abs()) + eps * (ez.mean(1) + (96 + V / 512) * U * z.abs().mean(1))
    return (lse - (1 - eps) * zy - eps * z.mean(1), lse), (e_loss, e_lse)


def _product(a, e, b, terms_a, terms_b, exact_b, k):
    """(a b, bound): a's error, both roundings to terms, the additions; as step_util.loss_grad."""
    rel = BF16 ** terms_a + (0 if exact_b else BF16 ** terms_b) + 4 * U + S._chain(S._pairs(terms_a, terms_b), k) * 2 * U
    return a @ b, (e + rel * a.abs()) @ b.abs()


def _within(got, ref, bound, what):
    off = (got.double() - ref).abs()
    assert (off <= bound).all(), (what, (off / bound).nan_to_num(nan=float("inf")).max().item(), int((~(off <= bound)).sum()))


@pytest.mark.parametrize("i", range(len(SHAPES)), ids=["-".join(map(str, s)) for s in SHAPES])
def test_tiles(L, i):
    T, V, D, xt, tt, gt, add = SHAPES[i]
    eps, scale = ((0.0, 1.0), (0.1, -0.7))[i % 2]
    x, w, y, dloss = _inputs(T, V, D, xt, tt)
    y[0] = V // 2
    announce("cross entropy, tiles", SHAPES[i], eps, scale)
    loss, lse = L.luq_cross_entropy_fwd(x, w, y, scale, eps)
    nx, nw = (1 if xt == "bf16" else 3), (1 if tt == "bf16" else 3)
    ok = y >= 0
    x64, w64, at = x.double() * ok[:, None], w.double(), y.clamp(min=0)
    z, ez = _logits(x64, w64, scale, nx, nw)
    ref, bound = _loss(z, ez, at, eps)
    for got, r, b, name in ((loss, ref[0], bound[0], "loss"), (lse, ref[1], bound[1], "lse")):
        assert (got[~ok] == 0).all(), name
        _within(got[ok], r[ok], b[ok], name)

    before = (0.01 * torch.randn(V, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(i))).to(DT[gt])
    out = [before.clone() if add else torch.full((V, D), float("nan"), dtype=DT[gt], device="cuda") for _ in range(2)]
    dx, dw = L.luq_cross_entropy_bwd(dloss, x, w, y, lse, scale, eps, bool(add), dtable=out[0])
    again = L.luq_cross_entropy_bwd(dloss, x, w, y, lse, scale, eps, bool(add), dtable=out[1])
    assert torch.equal(dx, again[0]) and torch.equal(dw, again[1]), "the order of the sums is fixed"
    del again, out
    base = (lse.double() * ok)[:, None]
    up = (dloss.double() * scale * ok)[:, None]
    p = torch.exp(z - base)
    ez += (z.abs() + 2 * (z - base).abs() + 8) * 2 * U
    eg = p * ez + 4 * U * (p + eps / V)
    g = p.sub_(eps / V)
    row = torch.arange(T, device="cuda")
    g[row, at] -= 1 - eps
    eg[row, at] += 4 * U * (1 - eps)
    g *= up
    eg *= up.abs()
    del p, z, ez
    rows, cols = (1 if xt == "bf16" else 3), (1 if gt == "bf16" else 3)
    tx, tw = (2 if xt == "bf16" and nw > 2 else nw), (2 if gt == "bf16" and nx > 2 else nx)
    ref, bound = _product(g, eg, w64, rows, tx, tt == "bf16", V)
    _within(dx, ref, bound + (BF16 * (ref.abs() + bound) if xt == "bf16" else 0) + 1e-37, "dx")
    assert (dx[~ok] == 0).all()
    ref, bound = _product(g.t(), eg.t(), x64, cols, tw, xt == "bf16", T)
    if add:
        ref = ref + before.double()
        bound = bound + 2 * U * ref.abs()
    _within(dw, ref, bound + (BF16 * (ref.abs() + bound) if gt == "bf16" else 0) + 1e-37, "dtable")
